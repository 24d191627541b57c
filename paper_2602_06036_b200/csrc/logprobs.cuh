// Interface of the token log probabilities and their gradient.
#pragma once

#include "dflash_internal.h"

namespace dflash {

constexpr int LP_MAX_TOKENS = 128, LP_MAX_TOP = 128;      // given tokens and alternatives of a row

void token_logprobs_plan(int es, int n_rows, int vocab, int n_tokens, int n_top, int sm_count, int32_t* info);      // threads of a CTA, CTAs of a row, CTAs
int launch_token_logprobs(const Launch& L, const dflash_token_logprobs_args& a);
int launch_token_logprobs_bwd(const Launch& L, const dflash_token_logprobs_bwd_args& a);

}  // namespace dflash
