// Interface of the attention of a batch that shares long prefixes.
#pragma once

#include "dflash_internal.h"

namespace dflash {

bool prefix_attn_supported(const dflash_config& c);
int64_t prefix_attn_workspace_bytes(const dflash_handle* h, int64_t batch, int64_t rows, int64_t groups);
// Walks the split of a call on the host (arrays in host memory); see dflash_prefix_plan_check.
int prefix_plan_check(const dflash_config& c, int sm_count, int S, int R, int n_groups, const int32_t* group_start, const int32_t* prefix_len,
                      const int32_t* ctx_len, int max_ctx_len, int64_t* info);
int launch_prefix_attention(const Launch& L, const dflash_prefix_attn_args& a);

}  // namespace dflash
