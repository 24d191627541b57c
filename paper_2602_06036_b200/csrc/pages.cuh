// Interface of the page operations of a paged cache.
#pragma once

#include "dflash_internal.h"

namespace dflash {

int64_t pages_workspace_bytes(int n, int max_pages, int n_pages);
int launch_pages_copy(const Launch& L, const dflash_pages_copy_args& a);
int launch_pages_fork(const Launch& L, const dflash_pages_fork_args& a);
int launch_pages_resize(const Launch& L, const dflash_pages_resize_args& a);
int launch_pages_compact(const Launch& L, const dflash_pages_compact_args& a);

}  // namespace dflash
