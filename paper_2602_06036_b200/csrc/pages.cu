// Pages of a paged K/V cache: copy, fork, resize (grow, truncate, release, copy on write) and compact.
// State: the page table and one reference count per page, in device memory; a page is free when its count is not
// positive. There is no free list to keep in step: a call finds the free pages by scanning the counts (4 bytes a page),
// which also makes the allocation deterministic: lowest free index first, requests in list order.
// Each call is a planning launch, one CTA per request that judges it by the state at the call's start (plus CTAs
// that list the free pages of a stretch of the counts), and an applying launch that changes tables and counts and moves the page
// data. Nothing that the second launch changes is read by it: what it needs of the old state the first one has
// written to the workspace. Page data moves as 16-byte vectors, 32 KB in flight per CTA, which is bound by HBM.
#include "dflash_internal.h"
#include "pages.cuh"
#include "ptx_sm100.cuh"

#include <algorithm>

namespace dflash {
namespace {

constexpr int NT = 256;                  // threads of every kernel here but the compaction plan
constexpr int SEG = 4096;                // counts scanned by one CTA
constexpr int VPT = 8;                   // 16-byte vectors in flight per thread
constexpr int CHUNK = NT * VPT;          // vectors per chunk (32 KB)
constexpr int CTAS_PER_SM = 8;

// The pool as 16-byte vectors. A page of one layer is contiguous: 2 * Hkv tiles of page_size slots.
struct Geometry {
    uint4* pool;
    int64_t layer_vecs;                  // vectors between the layers of a page
    int32_t n_pages, n_layers, page_size, page_vecs, tile_mask, slot_shift, chunks;   // chunks: per page, over all layers
    int32_t layer_chunks;
};
// What the planning launch says about request i.
struct Plan {
    int32_t need;                        // fresh pages it takes (0 if it is left out)
    int32_t ok;                          // carried out (if its pages are there)
    int32_t src, slots;                  // page whose first slots go to its first fresh page, or -1
};
struct Free {                            // free pages by stretches of SEG counts
    const int32_t* count;                // [n_seg]
    const int32_t* list;                 // [n_seg * SEG]
    int32_t n_seg;
};

__device__ __forceinline__ void flag(int32_t* status, int bit) {
    if (status) atomicOr(status, bit);
}
__device__ __forceinline__ int block_sum(int v, int32_t* sh) {           // sh: 33 words; every thread gets the sum
    const int warp = threadIdx.x >> 5, nw = (int)(blockDim.x >> 5);
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int t = ((int)threadIdx.x < nw) ? sh[threadIdx.x] : 0;
        t = __reduce_add_sync(0xffffffffu, t);
        if (threadIdx.x == 0) sh[32] = t;
    }
    __syncthreads();
    return sh[32];
}
// exclusive prefix sum over the CTA; `total` is the sum
__device__ __forceinline__ int block_scan(int v, int32_t* sh, int& total) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nw = (int)(blockDim.x >> 5);
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) sh[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int t = lane < nw ? sh[lane] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, t, o);
            if (lane >= o) t += y;
        }
        sh[lane] = t;
    }
    __syncthreads();
    total = sh[nw - 1];
    return x - v + (warp ? sh[warp - 1] : 0);
}

// chunk `c` (0 .. chunks-1) of page src -> dst, first `slots` slots of every tile
__device__ __forceinline__ void copy_chunk(const Geometry& g, int src, int dst, int slots, int c) {
    const int layer = c / g.layer_chunks, part = c % g.layer_chunks;
    const uint4* s = g.pool + layer * g.layer_vecs + (int64_t)src * g.page_vecs;
    uint4* d = g.pool + layer * g.layer_vecs + (int64_t)dst * g.page_vecs;
    uint4 v[VPT];
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int i = part * CHUNK + k * NT + (int)threadIdx.x;
        if (i < g.page_vecs && ((i & g.tile_mask) >> g.slot_shift) < slots) v[k] = __ldcs(s + i);
    }
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int i = part * CHUNK + k * NT + (int)threadIdx.x;
        if (i < g.page_vecs && ((i & g.tile_mask) >> g.slot_shift) < slots) __stcs(d + i, v[k]);
    }
}

// ---- copy -----------------------------------------------------------------------------------------------------
// Each CTA takes one contiguous run of chunks, so that it judges few entries: whether one may be carried out depends on the whole
// list (read once per entry and CTA, 8 bytes an entry).
__global__ void __launch_bounds__(NT) pages_copy_kernel(const Geometry g, int n, const int32_t* __restrict__ count,
                                                        const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                        const int32_t* __restrict__ n_slots, int32_t* status) {
    if (count) n = min(n, max(*count, 0));
    const int64_t total = (int64_t)n * g.chunks;
    const int64_t hi = total * (blockIdx.x + 1) / gridDim.x;
    int at = -1, s = -1, d = -1, slots = 0;
    for (int64_t c = total * blockIdx.x / gridDim.x; c < hi; ++c) {
        const int i = (int)(c / g.chunks);
        if (i != at) {
            at = i;
            s = src[i];
            d = dst[i];
            if (s >= 0) {
                int bad = s >= g.n_pages || d < 0 || d >= g.n_pages;
                for (int k = threadIdx.x; k < n; k += NT) {
                    const int sk = src[k];
                    bad |= sk >= 0 && (sk == d || (k < i && dst[k] == d));
                }
                if (__syncthreads_or(bad)) {
                    if (threadIdx.x == 0) flag(status, DFLASH_DEV_BAD_PAGE);
                    s = -1;
                }
            }
            slots = n_slots ? min(max(n_slots[i], 0), g.page_size) : g.page_size;
        }
        if (s >= 0) copy_chunk(g, s, d, slots, (int)(c % g.chunks));
    }
}

// ---- free pages ---------------------------------------------------------------------------------------------------
// stretch `seg` of the counts: its free pages by rising index
__device__ void list_free(const int32_t* __restrict__ ref, int n_pages, int seg, int32_t* count, int32_t* list, int32_t* sh) {
    constexpr int PER = SEG / NT;                       // neighbouring counts of one thread
    const int p0 = seg * SEG + (int)threadIdx.x * PER;
    unsigned mask = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (p0 + k < n_pages && ref[p0 + k] <= 0) mask |= 1u << k;
    int total;
    int at = block_scan(__popc(mask), sh, total);
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (mask >> k & 1) list[(int64_t)seg * SEG + at++] = p0 + k;
    if (threadIdx.x == 0) count[seg] = total;
}
__device__ __forceinline__ int free_page(const Free& f, int k) {        // the k-th free page (k below their number)
    for (int s = 0; s < f.n_seg; ++s) {
        const int c = f.count[s];
        if (k < c) return f.list[(int64_t)s * SEG + k];
        k -= c;
    }
    return -1;
}
__device__ __forceinline__ int n_free(const Free& f, int32_t* sh) {
    int v = 0;
    for (int s = threadIdx.x; s < f.n_seg; s += (int)blockDim.x) v += f.count[s];
    return block_sum(v, sh);
}

// ---- fork -----------------------------------------------------------------------------------------------------
struct ForkArgs {
    Geometry g;
    int32_t n, n_rows, max_pages, n_seg;
    const int32_t *parent, *child, *len;
    int32_t *table, *ref;
    int32_t *copy_src, *copy_dst, *copy_slots;
    Plan* plan;
    int32_t *seg_count, *free_list;
    int32_t* status;
};

__global__ void __launch_bounds__(NT) pages_fork_plan_kernel(const ForkArgs a) {
    __shared__ int32_t sh[33];
    ptx::pdl_trigger();
    if ((int)blockIdx.x >= a.n) return list_free(a.ref, a.g.n_pages, blockIdx.x - a.n, a.seg_count, a.free_list, sh);
    const int i = blockIdx.x, p = a.parent[i], c = a.child[i], len = max(a.len[i], 0), ps = a.g.page_size;
    int bits = 0;
    const int pages = (int)(((int64_t)len + ps - 1) / ps);
    if (p < 0 || p >= a.n_rows || c < 0 || c >= a.n_rows || p == c) {
        bits = DFLASH_DEV_BAD_ROW;
    } else if (pages > a.max_pages) {
        bits = DFLASH_DEV_CTX_OVERFLOW;
    } else {
        for (int k = threadIdx.x; k < a.n; k += NT) {
            const int ck = a.child[k];
            if (ck == p || (ck == c && k < i)) bits |= DFLASH_DEV_BAD_ROW;
        }
        for (int j = threadIdx.x; j < a.max_pages; j += NT) {
            if (a.table[(int64_t)c * a.max_pages + j] >= 0) bits |= DFLASH_DEV_BAD_ROW;
            if (j < pages) {
                const int e = a.table[(int64_t)p * a.max_pages + j];
                if (e < 0 || e >= a.g.n_pages) bits |= DFLASH_DEV_BAD_PAGE;
            }
        }
    }
    if (bits) flag(a.status, bits);
    const int bad = __syncthreads_or(bits);
    if (threadIdx.x == 0) {
        const int rest = len % ps, need = !bad && rest > 0;
        a.plan[i] = Plan{need, !bad, need ? a.table[(int64_t)p * a.max_pages + len / ps] : -1, rest};
    }
}

// Pages that the requests before i take, for every thread of a CTA of NT. In 64 bits: 65535 requests may ask for 2^30 pages each, and a sum that
// wrapped to a negative number would pass for one that fits. The warps add up 24-bit words (below 2^29) and what lies above them.
__device__ __forceinline__ int64_t need_before(const Plan* plan, int i, int32_t* sh) {
    int64_t v = 0;
    for (int k = threadIdx.x; k < i; k += NT) v += plan[k].need;
    const int low = __reduce_add_sync(0xffffffffu, (int)(v & 0xffffff)), high = __reduce_add_sync(0xffffffffu, (int)(v >> 24));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) {
        sh[threadIdx.x >> 5] = low;
        sh[NT / 32 + (threadIdx.x >> 5)] = high;
    }
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) v += ((int64_t)sh[NT / 32 + w] << 24) + sh[w];
    return v;
}
static_assert(2 * NT / 32 <= 33, "words of need_before");
// Page copies of the planned requests: chunk c of all, CTA `cta` of `n_cta`.
__device__ void apply_copies(const Geometry& g, const Plan* plan, int n, const Free& f, int avail, int cta, int n_cta, int32_t* sh) {
    int at = -1, dst = -1;
    Plan p{};
    for (int64_t c = cta; c < (int64_t)n * g.chunks; c += n_cta) {
        const int i = (int)(c / g.chunks);
        if (i != at) {
            at = i;
            p = plan[i];
            if (p.src >= 0) {
                const int64_t base = need_before(plan, i, sh);
                dst = base + p.need <= avail ? free_page(f, (int)base) : -1;
            }
        }
        if (p.src >= 0 && dst >= 0) copy_chunk(g, p.src, dst, p.slots, (int)(c % g.chunks));
    }
}
__device__ __forceinline__ void report_copy(int32_t* copy_src, int32_t* copy_dst, int32_t* copy_slots, int i, int src, int dst, int slots) {
    if (copy_src && threadIdx.x == 0) {
        copy_src[i] = dst >= 0 ? src : -1;
        copy_dst[i] = dst;
        copy_slots[i] = dst >= 0 ? slots : 0;
    }
}

__global__ void __launch_bounds__(NT) pages_fork_apply_kernel(const ForkArgs a) {
    __shared__ int32_t sh[33];
    ptx::pdl_wait();
    const Free f{a.seg_count, a.free_list, a.n_seg};
    const int avail = n_free(f, sh);
    if ((int)blockIdx.x >= a.n)
        return apply_copies(a.g, a.plan, a.n, f, avail, blockIdx.x - a.n, gridDim.x - a.n, sh);
    const int i = blockIdx.x;
    const Plan p = a.plan[i];
    int fresh = -1;
    bool go = p.ok;
    if (p.need) {
        const int64_t base = need_before(a.plan, i, sh);
        go = base + p.need <= avail;
        if (go) fresh = free_page(f, (int)base);
        else if (threadIdx.x == 0) flag(a.status, DFLASH_DEV_POOL_FULL);
    }
    report_copy(a.copy_src, a.copy_dst, a.copy_slots, i, p.src, fresh, p.slots);
    if (!go) return;
    const int whole = max(a.len[i], 0) / a.g.page_size;
    const int32_t* from = a.table + (int64_t)a.parent[i] * a.max_pages;
    int32_t* to = a.table + (int64_t)a.child[i] * a.max_pages;
    for (int j = threadIdx.x; j < a.max_pages; j += NT) {
        int e = -1;
        if (j < whole) {
            e = from[j];
            atomicAdd(a.ref + e, 1);
        } else if (j == whole && fresh >= 0) {
            e = fresh;
            a.ref[e] = 1;
        }
        to[j] = e;
    }
}

// ---- resize -----------------------------------------------------------------------------------------------------
struct ResizeArgs {
    Geometry g;
    int32_t n, n_rows, max_pages, n_seg, words;
    const int32_t *rows, *len, *cap;
    int32_t *table, *ref;
    int32_t *copy_src, *copy_dst, *copy_slots;
    Plan* plan;
    uint32_t* fresh_bits;                // [n][words] entries that get a fresh page
    int32_t *seg_count, *free_list;
    int32_t* status;
};

__global__ void __launch_bounds__(NT) pages_resize_plan_kernel(const ResizeArgs a) {
    __shared__ int32_t sh[33];
    ptx::pdl_trigger();
    if ((int)blockIdx.x >= a.n) return list_free(a.ref, a.g.n_pages, blockIdx.x - a.n, a.seg_count, a.free_list, sh);
    const int i = blockIdx.x, row = a.rows[i], cap = max(a.cap[i], 0), len = min(max(a.len[i], 0), cap), ps = a.g.page_size;
    const int want = (int)(((int64_t)cap + ps - 1) / ps), first = len / ps;        // page of the next position
    int bits = 0, need = 0;
    if (row < 0 || row >= a.n_rows) {
        bits = DFLASH_DEV_BAD_ROW;
    } else if (want > a.max_pages) {
        bits = DFLASH_DEV_CTX_OVERFLOW;
    } else {
        for (int k = threadIdx.x; k < i; k += NT)
            if (a.rows[k] == row) bits |= DFLASH_DEV_BAD_ROW;
        for (int j0 = 0; j0 < a.words * 32; j0 += NT) {
            const int j = j0 + (int)threadIdx.x;
            bool fresh = false;
            if (j < a.max_pages) {
                const int e = a.table[(int64_t)row * a.max_pages + j];
                if (e >= a.g.n_pages || (e < 0 && (int64_t)j * ps < len)) bits |= DFLASH_DEV_BAD_PAGE;
                else if (j < want) fresh = e < 0 || (j >= first && len < cap && a.ref[e] > 1);
            }
            const uint32_t w = __ballot_sync(0xffffffffu, fresh);
            if ((threadIdx.x & 31) == 0 && j / 32 < a.words) a.fresh_bits[(int64_t)i * a.words + j / 32] = w;
            need += fresh;
        }
    }
    if (bits) flag(a.status, bits);
    const int bad = __syncthreads_or(bits);
    need = block_sum(need, sh);
    if (threadIdx.x == 0) {
        // no entry below `first` gets a fresh page, so the copied page, if any, is the request's first one
        int src = -1;
        if (!bad && len % ps > 0 && len < cap) {
            const int e = a.table[(int64_t)row * a.max_pages + first];
            if (a.ref[e] > 1) src = e;
        }
        a.plan[i] = Plan{bad ? 0 : need, !bad, src, len % ps};
    }
}

__global__ void __launch_bounds__(NT) pages_resize_apply_kernel(const ResizeArgs a) {
    __shared__ int32_t sh[33];
    ptx::pdl_wait();
    const Free f{a.seg_count, a.free_list, a.n_seg};
    const int avail = n_free(f, sh);
    if ((int)blockIdx.x >= a.n)
        return apply_copies(a.g, a.plan, a.n, f, avail, blockIdx.x - a.n, gridDim.x - a.n, sh);
    const int i = blockIdx.x;
    const Plan p = a.plan[i];
    int base = 0;
    bool go = p.ok;
    if (p.need) {
        const int64_t before = need_before(a.plan, i, sh);
        go = before + p.need <= avail;
        if (go) base = (int)before;
        else if (threadIdx.x == 0) flag(a.status, DFLASH_DEV_POOL_FULL);
    }
    report_copy(a.copy_src, a.copy_dst, a.copy_slots, i, p.src, go && p.src >= 0 ? free_page(f, base) : -1, p.slots);
    if (!go) return;
    const int want = (int)(((int64_t)max(a.cap[i], 0) + a.g.page_size - 1) / a.g.page_size);
    int32_t* row = a.table + (int64_t)a.rows[i] * a.max_pages;
    const uint32_t* words = a.fresh_bits + (int64_t)i * a.words;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int run = base;                                    // fresh pages handed to the entries before j0
    for (int j0 = 0; j0 < a.max_pages; j0 += NT) {
        const int j = j0 + (int)threadIdx.x;
        uint32_t mine = 0;
        int rank = run;
#pragma unroll
        for (int w = 0; w < NT / 32; ++w) {
            const uint32_t x = j0 / 32 + w < a.words ? words[j0 / 32 + w] : 0u;
            if (w < warp) rank += __popc(x);
            if (w == warp) mine = x;
            run += __popc(x);
        }
        if (j >= a.max_pages) continue;
        const int e = row[j];
        const bool fresh = mine >> lane & 1;
        if (e >= 0 && (fresh || j >= want)) atomicSub(a.ref + e, 1);
        if (fresh) {
            const int page = free_page(f, rank + __popc(mine & ((1u << lane) - 1u)));
            a.ref[page] = 1;
            row[j] = page;
        } else if (j >= want && e != -1) {
            row[j] = -1;
        }
    }
}

// ---- compact ------------------------------------------------------------------------------------------------------
struct CompactArgs {
    Geometry g;
    int32_t n_rows, max_pages;
    int32_t *table, *ref;
    int32_t *n_live, *copy_src, *copy_dst, *n_copies;
    int32_t *hole, *mover;               // [n_pages / 2] pairs: page mover[k] goes to page hole[k]
    int32_t* rank;                       // [n_pages] of a page behind the border: its k; of one that is not in use: NOT_LIVE
    int32_t* pairs;                      // [1]
    int32_t move_ctas;
    int32_t* status;
};

// Every CTA counts the whole pool itself (the counts come out of L2) and lists the holes and movers of its own stretch.
constexpr int NT_COMPACT = 1024, NOT_LIVE = (int)0x80000000;
__global__ void __launch_bounds__(NT_COMPACT) pages_compact_plan_kernel(const CompactArgs a) {
    __shared__ int32_t sh[33];
    ptx::pdl_trigger();
    const int n = a.g.n_pages, lo = blockIdx.x * SEG;
    int all = 0, before = 0;
    for (int p = threadIdx.x; p < n; p += NT_COMPACT) {
        const int live = a.ref[p] > 0;
        all += live;
        if (p < lo) before += live;
    }
    const int border = block_sum(all, sh);
    before = block_sum(before, sh);
    int front = 0;                                     // live pages below the border
    for (int p = threadIdx.x; p < border; p += NT_COMPACT) front += a.ref[p] > 0;
    front = block_sum(front, sh);
    constexpr int PER = SEG / NT_COMPACT;
    const int p0 = lo + (int)threadIdx.x * PER;
    unsigned mask = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (p0 + k < n && a.ref[p0 + k] > 0) mask |= 1u << k;
    int total;
    int live_before = before + block_scan(__popc(mask), sh, total);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int p = p0 + k;
        if (p < n) {
            const bool live = mask >> k & 1;
            a.rank[p] = live ? live_before - front : NOT_LIVE;
            if (p < border && !live) a.hole[p - live_before] = p;
            if (p >= border && live) a.mover[live_before - front] = p;
            live_before += live;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.pairs[0] = border - front;
        a.pairs[1] = border;
        if (a.n_live) *a.n_live = border;
        if (a.n_copies) *a.n_copies = border - front;
    }
}

__global__ void __launch_bounds__(NT) pages_compact_apply_kernel(const CompactArgs a) {
    ptx::pdl_wait();
    const int pairs = a.pairs[0], border = a.pairs[1];
    if ((int)blockIdx.x < a.move_ctas) {
        const int64_t total = (int64_t)pairs * a.g.chunks, hi = total * (blockIdx.x + 1) / a.move_ctas;
        for (int64_t c = total * blockIdx.x / a.move_ctas; c < hi; ++c) {
            const int k = (int)(c / a.g.chunks);
            copy_chunk(a.g, a.mover[k], a.hole[k], a.g.page_size, (int)(c % a.g.chunks));
        }
        return;
    }
    const int64_t at = (int64_t)(blockIdx.x - a.move_ctas) * NT + threadIdx.x, step = (int64_t)(gridDim.x - a.move_ctas) * NT;
    for (int64_t k = at; k < a.g.n_pages / 2; k += step) {
        const bool pair = k < pairs;
        if (pair) {
            a.ref[a.hole[k]] = a.ref[a.mover[k]];
            a.ref[a.mover[k]] = 0;
        }
        if (a.copy_src) {
            a.copy_src[k] = pair ? a.mover[k] : -1;
            a.copy_dst[k] = pair ? a.hole[k] : -1;
        }
    }
    for (int64_t j = at; j < (int64_t)a.n_rows * a.max_pages; j += step) {
        const int e = a.table[j];
        if (e < 0) continue;
        const int k = e < a.g.n_pages ? a.rank[e] : NOT_LIVE;
        if (k == NOT_LIVE) flag(a.status, DFLASH_DEV_BAD_PAGE);          // it would name another sequence's page, once a mover has come there
        else if (e >= border) a.table[j] = a.hole[k];
    }
}

int ilog2(int v) {
    int n = 0;
    while ((1 << n) < v) ++n;
    return n;
}
Geometry geometry(const dflash_config& c, void* pool, int n_pages) {
    Geometry g{};
    const int slot_vecs = c.head_dim * elem_size(c.dtype) / 16, tile = c.page_size * slot_vecs;      // powers of two
    g.pool = (uint4*)pool;
    g.n_pages = n_pages;
    g.n_layers = c.n_layers;
    g.page_size = c.page_size;
    g.page_vecs = 2 * c.n_kv_heads * tile;
    g.layer_vecs = (int64_t)n_pages * g.page_vecs;
    g.tile_mask = tile - 1;
    g.slot_shift = ilog2(slot_vecs);
    g.layer_chunks = (g.page_vecs + CHUNK - 1) / CHUNK;
    g.chunks = g.n_layers * g.layer_chunks;
    return g;
}
int n_segs(int n_pages) { return (n_pages + SEG - 1) / SEG; }
int copy_ctas(const dflash_handle* h, const Geometry& g, int64_t n) {
    return (int)std::max<int64_t>(1, std::min<int64_t>(n * g.chunks, (int64_t)h->sm_count * CTAS_PER_SM));
}
struct PagesWs {
    Plan* plan;
    uint32_t* fresh_bits;
    int32_t *seg_count, *free_list;
    int32_t *hole, *mover, *rank, *pairs;
    int64_t bytes;
};
PagesWs carve_pages(void* base, int n, int max_pages, int n_pages) {
    PagesWs w{};
    {
        Arena a(base);
        w.plan = (Plan*)a.take((int64_t)n * sizeof(Plan));
        w.fresh_bits = (uint32_t*)a.take((int64_t)n * ((max_pages + 31) / 32) * 4);
        w.seg_count = (int32_t*)a.take((int64_t)n_segs(n_pages) * 4);
        w.free_list = (int32_t*)a.take((int64_t)n_segs(n_pages) * SEG * 4);
        w.bytes = a.off;
    }
    Arena a(base);                       // the compaction's lists take the place of the others
    w.hole = (int32_t*)a.take((int64_t)(n_pages / 2 + 1) * 4);
    w.mover = (int32_t*)a.take((int64_t)(n_pages / 2 + 1) * 4);
    w.rank = (int32_t*)a.take((int64_t)n_pages * 4);
    w.pairs = (int32_t*)a.take(8);
    w.bytes = std::max(w.bytes, a.off);
    return w;
}
int launched(cudaError_t e, int n) {
    if (e != cudaSuccess) return DFLASH_ERR_CUDA;
    g_launches += n;
    return DFLASH_OK;
}

}  // namespace

int64_t pages_workspace_bytes(int n, int max_pages, int n_pages) { return carve_pages(nullptr, n, max_pages, n_pages).bytes; }

int launch_pages_copy(const Launch& L, const dflash_pages_copy_args& a) {
    const Geometry g = geometry(L.h->cfg, a.kv_pool, a.n_pool_pages);
    return launched(launch_ordered(pages_copy_kernel, dim3(copy_ctas(L.h, g, a.n)), dim3(NT), 0, L.st, g, a.n, a.count, a.src, a.dst, a.n_slots, L.status), 1);
}

int launch_pages_fork(const Launch& L, const dflash_pages_fork_args& a) {
    const PagesWs w = carve_pages(a.workspace, a.n, a.max_pages, a.n_pool_pages);
    ForkArgs k{};
    k.g = geometry(L.h->cfg, a.kv_pool, a.n_pool_pages);
    k.n = a.n; k.n_rows = a.n_rows; k.max_pages = a.max_pages; k.n_seg = n_segs(a.n_pool_pages);
    k.parent = a.parent; k.child = a.child; k.len = a.fork_len; k.table = a.page_table; k.ref = a.ref_count;
    k.copy_src = a.copy_src; k.copy_dst = a.copy_dst; k.copy_slots = a.copy_slots;
    k.plan = w.plan; k.seg_count = w.seg_count; k.free_list = w.free_list; k.status = L.status;
    const int rc = launched(launch_ordered(pages_fork_plan_kernel, dim3(a.n + k.n_seg), dim3(NT), 0, L.st, k), 1);
    if (rc != DFLASH_OK) return rc;
    return launched(launch_pdl(pages_fork_apply_kernel, dim3(a.n + copy_ctas(L.h, k.g, a.n)), dim3(NT), 0, L.st, k), 1);
}

int launch_pages_resize(const Launch& L, const dflash_pages_resize_args& a) {
    const PagesWs w = carve_pages(a.workspace, a.n, a.max_pages, a.n_pool_pages);
    ResizeArgs k{};
    k.g = geometry(L.h->cfg, a.kv_pool, a.n_pool_pages);
    k.n = a.n; k.n_rows = a.n_rows; k.max_pages = a.max_pages; k.n_seg = n_segs(a.n_pool_pages); k.words = (a.max_pages + 31) / 32;
    k.rows = a.rows; k.len = a.keep_len; k.cap = a.capacity; k.table = a.page_table; k.ref = a.ref_count;
    k.copy_src = a.copy_src; k.copy_dst = a.copy_dst; k.copy_slots = a.copy_slots;
    k.plan = w.plan; k.fresh_bits = w.fresh_bits; k.seg_count = w.seg_count; k.free_list = w.free_list; k.status = L.status;
    const int rc = launched(launch_ordered(pages_resize_plan_kernel, dim3(a.n + k.n_seg), dim3(NT), 0, L.st, k), 1);
    if (rc != DFLASH_OK) return rc;
    return launched(launch_pdl(pages_resize_apply_kernel, dim3(a.n + copy_ctas(L.h, k.g, a.n)), dim3(NT), 0, L.st, k), 1);
}

int launch_pages_compact(const Launch& L, const dflash_pages_compact_args& a) {
    const PagesWs w = carve_pages(a.workspace, 0, a.max_pages, a.n_pool_pages);
    CompactArgs k{};
    k.g = geometry(L.h->cfg, a.kv_pool, a.n_pool_pages);
    k.n_rows = a.n_rows; k.max_pages = a.max_pages; k.table = a.page_table; k.ref = a.ref_count;
    k.n_live = a.n_live; k.copy_src = a.copy_src; k.copy_dst = a.copy_dst; k.n_copies = a.n_copies;
    k.hole = w.hole; k.mover = w.mover; k.rank = w.rank; k.pairs = w.pairs; k.status = L.status;
    k.move_ctas = copy_ctas(L.h, k.g, std::max(a.n_pool_pages / 2, 1));
    const int64_t entries = std::max<int64_t>((int64_t)a.n_rows * a.max_pages, a.n_pool_pages / 2);
    const int table_ctas = (int)std::max<int64_t>(1, std::min<int64_t>((entries + NT - 1) / NT, 2 * (int64_t)L.h->sm_count));
    const int rc = launched(launch_ordered(pages_compact_plan_kernel, dim3(n_segs(a.n_pool_pages)), dim3(NT_COMPACT), 0, L.st, k), 1);
    if (rc != DFLASH_OK) return rc;
    return launched(launch_pdl(pages_compact_apply_kernel, dim3(k.move_ctas + table_ctas), dim3(NT), 0, L.st, k), 1);
}

}  // namespace dflash
