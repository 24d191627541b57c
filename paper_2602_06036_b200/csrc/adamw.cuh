// Interface of the AdamW step.
#pragma once

#include "dflash_internal.h"

namespace dflash {

int64_t adamw_workspace_bytes(int sm_count, int n_tensors);
int launch_adamw(const Launch& L, const dflash_adamw_args& a);

}  // namespace dflash
