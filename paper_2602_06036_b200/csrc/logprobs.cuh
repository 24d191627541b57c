// Interface of the token log probabilities and their gradient.
#pragma once

#include "dflash_internal.h"

namespace dflash {

constexpr int LP_MAX_TOKENS = 128, LP_MAX_TOP = 128;      // given tokens and alternatives of a row

int launch_token_logprobs(const Launch& L, const dflash_token_logprobs_args& a);
int launch_token_logprobs_bwd(const Launch& L, const dflash_token_logprobs_bwd_args& a);

}  // namespace dflash
