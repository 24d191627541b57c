// How the work of the shared-prefix attention is cut up: one chain of key tiles over all (rows, kv head) items, of which
// every CTA takes an equal stretch by cost. Shared by the tensor-core kernel, the CUDA-core kernel and the merge.
//
// Entries: the groups (rows of all their sequences against the prefix), then the sequences (their rows against what is
// their own: cached keys behind the prefix, and the block). The query rows of an entry and kv head are "packed":
// row (b, r, j) of the Hq/Hkv heads j that share the kv head, in this order. An item is one kv head of an entry, up to two tiles
// of packed rows, and a range of key tiles. Lengths and groups are device data, so each CTA works the chain out itself
// (one pass of the CTA over groups and sequences).
#pragma once

#include "dflash_internal.h"

namespace dflash {
namespace {

constexpr int CHUNK_KEYS = 64;           // keys per chunk; a tile is one or two chunks

struct PlanParams {
    int32_t S, R, G, Hkv, n_groups, max_ctx_len;
    int32_t row_tile;                    // packed rows per query tile
    int32_t tiles_per_item;              // query tiles of an item that read each key tile together: 1 or 2
    int32_t chunks_per_tile;             // chunks of a key tile: 1 or 2
    int32_t cost_item, cost_one, cost_two;   // of an item's start, of a key tile with one query tile, with two
    const int32_t *group_start, *prefix_len, *ctx_len;
    int32_t* status;
};

struct Entry {
    int32_t seq, n_rows;                 // first sequence; packed rows per kv head
    int32_t lo, hi, block;               // cached keys [lo, hi); block rows are keys too
    int32_t chunk0, n_chunks, n_tiles;   // chunks of 64 keys from chunk0 * 64 on, the block's chunk last
    int32_t items, blocks;               // items of row tiles per kv head and key block; key blocks
    int32_t single;                      // 1: the last of these items has one row tile
    int64_t cost;                        // of all kv heads
};

// Clamped length; one that max_ctx_len does not cover is flagged (by `tell`).
__host__ __device__ __forceinline__ int plan_len(const PlanParams& p, int v, bool tell) {
    if (v > p.max_ctx_len) {
#ifdef __CUDA_ARCH__
        if (tell && p.status) atomicOr(p.status, DFLASH_DEV_CTX_OVERFLOW);
#endif
        return p.max_ctx_len;
    }
    return v > 0 ? v : 0;
}
// group of sequence b, or -1 (group_start does not fall)
__host__ __device__ __forceinline__ int plan_group(const PlanParams& p, int b) {
    int lo = 0, hi = p.n_groups + 1;     // first index with group_start > b
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (p.group_start[mid] > b) hi = mid;
        else lo = mid + 1;
    }
    const int g = lo - 1;
    return g < p.n_groups ? g : -1;      // -1 as well when b lies before the first group
}
// how many of sequence b's keys its group's prefix item deals with (0 or the whole prefix)
__host__ __device__ __forceinline__ int plan_shared(const PlanParams& p, int g, int len) {
    if (g < 0) return 0;
    const int P = plan_len(p, p.prefix_len[g], false);
    return len >= P ? P : 0;
}

// A call of few key tiles is cut into single ones: no cost for an item's start then, which would leave CTAs idle.
__host__ __device__ __forceinline__ int64_t plan_cost(PlanParams& p, int64_t tiles, int64_t cost, int n_cta) {
    if (tiles > 2 * (int64_t)n_cta) return cost;
    p.cost_item = 0;
    return 0;                            // to be summed up again
}
// How many CTAs share a chain of this cost: each stretch is at least as long as the largest distance between the starts of
// neighbouring key tiles, so that every CTA below this number has one (the merge reads the results of all CTAs from an
// item's first to its last).
__host__ __device__ __forceinline__ int plan_ctas(const PlanParams& p, int64_t total, int n_cta) {
    const int64_t most = total / (p.cost_item + (p.cost_one > p.cost_two ? p.cost_one : p.cost_two));
    return most < 1 ? 1 : most < n_cta ? (int)most : n_cta;
}

__host__ __device__ __forceinline__ int64_t plan_lo(int64_t total, int cta, int n_cta) {     // where a CTA's stretch begins
    return cta < n_cta ? (total * cta + n_cta - 1) / n_cta : total;
}

// `share`: costs a CTA takes (0: not known yet, key blocks are left at 1). Long prefixes are cut into blocks of about one CTA's
// share, ordered before the row tiles: CTAs that run side by side then read the same keys, which come out of L2.
__host__ __device__ __forceinline__ Entry plan_entry(const PlanParams& p, int e, bool groups_ok, int64_t share, bool tell) {
    Entry x{};
    x.blocks = 1;
    if (e < p.n_groups) {
        if (groups_ok) {
            x.seq = p.group_start[e];
            x.n_rows = (p.group_start[e + 1] - x.seq) * p.R * p.G;
            x.hi = plan_len(p, p.prefix_len[e], tell);
        }
    } else {
        x.seq = e - p.n_groups;
        x.n_rows = p.R * p.G;
        x.hi = plan_len(p, p.ctx_len[x.seq], tell);
        x.lo = groups_ok ? plan_shared(p, plan_group(p, x.seq), x.hi) : 0;
        x.block = 1;
    }
    x.chunk0 = x.lo / CHUNK_KEYS;
    x.n_chunks = (x.hi > x.lo ? (x.hi + CHUNK_KEYS - 1) / CHUNK_KEYS - x.chunk0 : 0) + x.block;
    if (x.n_rows == 0) x.n_chunks = 0;
    x.n_tiles = (x.n_chunks + p.chunks_per_tile - 1) / p.chunks_per_tile;
    if (x.n_tiles == 0) return x;
    const int row_tiles = (x.n_rows + p.row_tile - 1) / p.row_tile;
    x.items = (row_tiles + p.tiles_per_item - 1) / p.tiles_per_item;
    x.single = row_tiles % p.tiles_per_item != 0 || p.tiles_per_item == 1;
    const int64_t one = p.tiles_per_item == 1 ? (int64_t)x.items * p.cost_one : (int64_t)(x.items - x.single) * p.cost_two + x.single * p.cost_one;
    if (share > 0 && x.items > 1) {
        const int64_t per = (int64_t)x.n_tiles * p.cost_two;
        const int64_t blocks = (per + share / 2) / share;
        x.blocks = blocks < 1 ? 1 : blocks > x.n_tiles ? x.n_tiles : (int)blocks;
    }
    x.cost = (int64_t)p.Hkv * ((int64_t)x.items * x.blocks * p.cost_item + x.n_tiles * one);
    return x;
}
__host__ __device__ __forceinline__ int entry_items(const PlanParams& p, const Entry& x) { return x.n_tiles ? p.Hkv * x.items * x.blocks : 0; }

// One CTA's stretch of an item.
struct Segment {
    int32_t kvh, seq, n_rows, row0;      // packed rows [row0, row0 + row_tile * tiles) of the entry, those below n_rows count
    int32_t two;                         // two query tiles
    int32_t lo, hi, block;               // as in Entry
    int32_t chunk, n_chunks;             // first chunk (as 64-key index into the cache) and number; the block's chunk is
    int32_t ctx_chunks;                  //   the one behind ctx_chunks chunks of the segment (block = 1) or absent
    int32_t item;                        // number among the items of groups, or among those of sequences
    int32_t prefix;                      // an item of a group
    int32_t first, last;                 // holds the item's first / last key tile
};

// Walks the segments of one CTA. Every thread that walks holds the same state.
struct Walker {
    Entry x;
    int32_t e, kvh, kb, it;              // entry, kv head, key block, item of row tiles
    int32_t item;                        // number of that item
    int32_t n_group_items;
    int64_t start;                       // cost at which it starts
    int64_t lo, hi;                      // the CTA's stretch of costs
    int64_t share;
    bool groups_ok, done;                // done: the item has been looked at
};
__host__ __device__ __forceinline__ int block_lo(const Entry& x, int kb) { return (int)((int64_t)x.n_tiles * kb / x.blocks); }
__host__ __device__ __forceinline__ int item_cost_tile(const PlanParams& p, const Entry& x, int it) {
    return (p.tiles_per_item == 1 || (x.single && it == x.items - 1)) ? p.cost_one : p.cost_two;
}
// first key tile of an item of n tiles that starts at cost `at` or later; tile 0 starts with the item
__host__ __device__ __forceinline__ int tile_at(const PlanParams& p, int64_t start, int n, int cost, int64_t at) {
    if (at <= start) return 0;
    const int64_t j = (at - start - p.cost_item + cost - 1) / cost;
    return j < 1 ? 1 : j > n ? n : (int)j;
}

struct PlanShared {
    int64_t warp[16], warp2[16];
    int32_t warp_items[16];
    int32_t n_group_items;
    int32_t e, item;                     // entry with the CTA's first cost, and the number of its first item
    int64_t start;
};

// All threads of the CTA (n_threads of them) call this. `infos`: entry's first item and geometry for the merge, written by CTA 0.
struct GroupInfo { int32_t item0, items, blocks, single; };
// group whose prefix item covers this sequence or -1, its first packed row there; its own items, numbered from the first sequence's on
struct SeqInfo { int32_t group, row_off, item0, blocks; };

template <int N_THREADS>
__device__ __forceinline__ bool plan_cta(PlanParams& p, PlanShared& sh, Walker& w, GroupInfo* ginfo, SeqInfo* sinfo) {
    constexpr int NW = N_THREADS / 32;
    static_assert(NW <= 16, "scratch");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool teller = blockIdx.x == 0;
    int bad = 0;
    for (int g = tid; g <= p.n_groups && p.n_groups > 0; g += N_THREADS) {
        const int a = p.group_start[g];
        bad |= a < 0 || a > p.S || (g > 0 && p.group_start[g - 1] > a);
    }
    bad = __syncthreads_or(bad);
    const bool ok = !bad && p.n_groups > 0;
    if (bad && teller && tid == 0 && p.status) atomicOr(p.status, DFLASH_DEV_BAD_GROUP);
    const int n = p.n_groups + p.S, per = (n + N_THREADS - 1) / N_THREADS;
    const int e0 = min(n, tid * per), e1 = min(n, e0 + per);
    // total cost with whole prefixes gives the share of a CTA, which gives the key blocks
    int64_t c = 0, tiles = 0;
    for (int e = e0; e < e1; ++e) {
        const Entry x = plan_entry(p, e, ok, 0, teller);
        c += x.cost;
        tiles += (int64_t)p.Hkv * x.items * x.n_tiles;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        c += __shfl_xor_sync(0xffffffffu, c, o);
        tiles += __shfl_xor_sync(0xffffffffu, tiles, o);
    }
    if (lane == 0) { sh.warp[warp] = c; sh.warp2[warp] = tiles; }
    __syncthreads();
    int64_t raw = 0;
    tiles = 0;
    for (int k = 0; k < NW; ++k) { raw += sh.warp[k]; tiles += sh.warp2[k]; }
    if (plan_cost(p, tiles, raw, gridDim.x) == 0) raw = tiles * p.cost_two;      // both tile costs are close: only key blocks depend on it
    const int64_t share = (raw + gridDim.x - 1) / gridDim.x;
    // running costs and items
    int64_t mine = 0;
    int items = 0;
    for (int e = e0; e < e1; ++e) {
        const Entry x = plan_entry(p, e, ok, share, false);
        mine += x.cost;
        items += entry_items(p, x);
    }
    int64_t run = mine;
    int run_items = items;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, run, o);
        const int z = __shfl_up_sync(0xffffffffu, run_items, o);
        if (lane >= o) { run += y; run_items += z; }
    }
    __syncthreads();
    if (lane == 31) { sh.warp[warp] = run; sh.warp_items[warp] = run_items; }
    __syncthreads();
    run -= mine;
    run_items -= items;
    int64_t total = 0;
    for (int k = 0; k < NW; ++k) {
        if (k < warp) { run += sh.warp[k]; run_items += sh.warp_items[k]; }
        total += sh.warp[k];
    }
    const int n_cta = plan_ctas(p, total, gridDim.x);
    const int64_t lo = plan_lo(total, blockIdx.x, n_cta), hi = plan_lo(total, blockIdx.x + 1, n_cta);
    for (int e = e0; e < e1; ++e) {
        const Entry x = plan_entry(p, e, ok, share, false);
        if (x.cost > 0 && run <= lo && lo < run + x.cost) { sh.e = e; sh.item = run_items; sh.start = run; }
        if (e == p.n_groups) sh.n_group_items = run_items;
        if (teller) {
            if (e < p.n_groups) {
                ginfo[e] = GroupInfo{run_items, x.items, x.blocks, x.single};
            } else {
                const int b = e - p.n_groups, g = ok ? plan_group(p, b) : -1;
                const int shared = plan_shared(p, g, x.hi);
                sinfo[b] = SeqInfo{shared > 0 ? g : -1, shared > 0 ? (b - p.group_start[g]) * p.R * p.G : 0, run_items /* of all */, x.blocks};
            }
        }
        run += x.cost;
        run_items += entry_items(p, x);
    }
    __syncthreads();
    w.groups_ok = ok;
    w.share = share;
    w.lo = lo;
    w.hi = hi;
    return lo < hi;
}

// Positions the walker at the first item that has a key tile at cost w.lo or later.
__host__ __device__ __forceinline__ void walk_begin(const PlanParams& p, const PlanShared& sh, Walker& w) {
    w.e = sh.e;
    w.x = plan_entry(p, w.e, w.groups_ok, w.share, false);
    const Entry& x = w.x;
    int64_t off = w.lo - sh.start;
    const int64_t per_head = x.cost / p.Hkv;
    w.kvh = (int)(off / per_head);
    off -= w.kvh * per_head;
    w.start = sh.start + w.kvh * per_head;
    w.kb = 0;
    int64_t two = 0;
    int n = 0;
    const int full = x.items - x.single;           // items with cost_two (or, with one tile an item, none)
    for (;; ++w.kb) {
        n = block_lo(x, w.kb + 1) - block_lo(x, w.kb);
        const int64_t c2 = (int64_t)p.cost_item + (int64_t)n * p.cost_two, c1 = (int64_t)p.cost_item + (int64_t)n * p.cost_one;
        const int64_t cost = p.tiles_per_item == 1 ? x.items * c1 : full * c2 + x.single * c1;
        if (off < cost || w.kb == x.blocks - 1) { two = p.tiles_per_item == 1 ? c1 : c2; break; }
        off -= cost;
        w.start += cost;
    }
    w.it = off / two < x.items - 1 ? (int)(off / two) : x.items - 1;
    w.start += w.it * two;
    w.n_group_items = sh.n_group_items;
    w.done = false;
    w.item = sh.item + (w.kvh * x.blocks + w.kb) * x.items + w.it;
}
__host__ __device__ __forceinline__ void walk_on(const PlanParams& p, Walker& w) {       // to the next item
    const Entry& x = w.x;
    const int n = block_lo(x, w.kb + 1) - block_lo(x, w.kb);
    w.start += (int64_t)p.cost_item + (int64_t)n * item_cost_tile(p, x, w.it);
    ++w.item;
    w.done = false;
    if (++w.it < x.items) return;
    w.it = 0;
    if (++w.kb < x.blocks) return;
    w.kb = 0;
    if (++w.kvh < p.Hkv) return;
    w.kvh = 0;
    if (w.start >= w.hi) return;
    do {
        if (++w.e >= p.n_groups + p.S) return;
        w.x = plan_entry(p, w.e, w.groups_ok, w.share, false);
    } while (w.x.cost == 0);
}
// Next segment of this CTA, or false. The step past an item is left to the next call, so that what the segment loads can be
// requested before the lengths of another sequence are.
__host__ __device__ __forceinline__ bool walk_next(const PlanParams& p, Walker& w, Segment& s) {
    for (;;) {
        if (w.done) walk_on(p, w);
        if (w.e >= p.n_groups + p.S || w.start >= w.hi) return false;
        w.done = true;
        const Entry& x = w.x;
        const int t0 = block_lo(x, w.kb), n = block_lo(x, w.kb + 1) - t0;
        const int cost = item_cost_tile(p, x, w.it);
        const int a = tile_at(p, w.start, n, cost, w.lo), b = tile_at(p, w.start, n, cost, w.hi);
        if (a >= b) continue;
        s.kvh = w.kvh;
        s.seq = x.seq;
        s.n_rows = x.n_rows;
        s.row0 = w.it * p.tiles_per_item * p.row_tile;
        s.two = p.tiles_per_item == 2 && !(x.single && w.it == x.items - 1);
        s.lo = x.lo;
        s.hi = x.hi;
        const int c0 = (t0 + a) * p.chunks_per_tile, c1 = (t0 + b) * p.chunks_per_tile < x.n_chunks ? (t0 + b) * p.chunks_per_tile : x.n_chunks;
        s.chunk = x.chunk0 + c0;
        s.n_chunks = c1 - c0;
        s.block = x.block && c1 == x.n_chunks;
        s.ctx_chunks = s.n_chunks - s.block;
        s.prefix = w.e < p.n_groups;
        s.item = w.item - (s.prefix ? 0 : w.n_group_items);
        s.first = a == 0;
        s.last = b == n;
        return true;
    }
}

}  // namespace
}  // namespace dflash
