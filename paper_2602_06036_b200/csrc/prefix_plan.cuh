// How the work of the shared-prefix attention is cut up: one chain of key tiles over all (rows, kv head) items, of which
// every CTA takes an equal stretch by cost. A small kernel writes each CTA's segments down (the arithmetic inlined into the
// attention kernel itself made its code 231 KB long and its instruction cache miss all the time: 32 sequences x 17 rows behind 32768 positions took 567 us, now 276).
//
// Entries: the groups (rows of all their sequences against the prefix), then the sequences (their rows against what is
// their own: cached keys behind the prefix, and the block). The query rows of an entry and kv head are "packed":
// row (b, r, j) of the Hq/Hkv heads j that share the kv head, in this order. An item is one kv head of an entry, up to two tiles
// of packed rows, and a range of key tiles.
#pragma once

#include "dflash_internal.h"
#include "ptx_sm100.cuh"

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
    int32_t group;                       // of a sequence, or -1
    int32_t lo, hi, block;               // cached keys [lo, hi); block rows are keys too
    int32_t chunk0, n_chunks, n_tiles;   // chunks of 64 keys from chunk0 * 64 on, the block's chunk last
    int32_t items, blocks;               // items of row tiles per kv head and key block; key blocks
    int32_t single;                      // 1: the last of these items has one row tile
    int32_t cost;                        // of all kv heads
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

// Costs are 32-bit numbers: the host refuses a call whose bound of them is higher (plan_fits).
//
// A call of few key tiles is cut into single ones: no cost for an item's start then, which would leave CTAs idle. Measured on 148 CTAs, with and without
// this: 64 tiles of 4 sequences x 16 rows behind 512 positions 20.8 us and 26.7, 96 tiles behind 1024 22.8 and 27.5, 192 tiles of 8 x 16 rows 29.3 and 29.8; but 192
// tiles of 8 x 1 rows behind 2048 25.4 and 22.4, 256 of one sequence of 4096 28.1 and 25.2. Above the border, single tiles of one sequence of 6000 (376 of them) would take 30.4
// us instead of 28.1, of 8 x 16 rows behind 2048 (384) 32.9 instead of 34.8.
__host__ __device__ __forceinline__ bool plan_few(const PlanParams& p, int tiles, int n_cta) { return tiles <= 2 * n_cta; }
// Length of a CTA's stretch of costs: its share, and at least the largest distance between the starts of neighbouring key
// tiles, so that every CTA up to the last used one has a tile (the merge reads the results of all CTAs from an item's first to its last).
__host__ __device__ __forceinline__ int plan_stretch(const PlanParams& p, int total, int n_cta) {
    const int share = (total + n_cta - 1) / n_cta, gap = p.cost_item + (p.cost_one > p.cost_two ? p.cost_one : p.cost_two);
    return share > gap ? share : gap;
}

// Entry e with whole prefixes, its cost left open.
__host__ __device__ __forceinline__ Entry plan_entry(const PlanParams& p, int e, bool groups_ok, bool tell) {
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
        x.group = groups_ok ? plan_group(p, x.seq) : -1;
        x.lo = plan_shared(p, x.group, x.hi);
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
    return x;
}
// A prefix that none of its group's sequences reads is no work, and its pages need not exist. Which these are is known when all entries are: they
// count in the shares that key blocks are measured by, and not in what is handed out.
__host__ __device__ __forceinline__ void entry_unread(Entry& x) { x.n_rows = x.n_chunks = x.n_tiles = x.items = x.cost = 0; }
// `share`: cost that a CTA takes. Long prefixes are cut into key blocks of about that much, ordered before the row tiles: CTAs that run side by
// side then read the same keys, which come out of L2.
__host__ __device__ __forceinline__ void entry_blocks(const PlanParams& p, Entry& x, int32_t share) {
    if (x.n_tiles == 0 || x.items < 2) return;
    const int blocks = (x.n_tiles * p.cost_two + share / 2) / share;
    x.blocks = blocks < 1 ? 1 : blocks > x.n_tiles ? x.n_tiles : blocks;
}
__host__ __device__ __forceinline__ void entry_cost(const PlanParams& p, Entry& x) {
    if (x.n_tiles == 0) return;
    const int one = p.tiles_per_item == 1 ? x.items * p.cost_one : (x.items - x.single) * p.cost_two + x.single * p.cost_one;
    x.cost = p.Hkv * (x.items * x.blocks * p.cost_item + x.n_tiles * one);
}
__host__ __device__ __forceinline__ int entry_items(const PlanParams& p, const Entry& x) { return x.n_tiles ? p.Hkv * x.items * x.blocks : 0; }

// One CTA's stretch of an item.
struct Segment {
    int32_t kvh, seq, n_rows, row0;      // packed rows [row0, row0 + row_tile * tiles) of the entry, those below n_rows count
    int32_t two;                         // two query tiles
    int32_t lo, hi, block;               // as in Entry
    int32_t chunk, n_chunks;             // first chunk (as 64-key index into the cache) and number; the block's chunk is
    int32_t ctx_chunks;                  //   the one behind ctx_chunks chunks of the segment (block = 1) or absent
    int32_t prefix;                      // an item of a group
    int32_t slot;                        // where its partial result goes (group items and sequence items apart)
    int32_t pad[3];
};
static_assert(sizeof(Segment) == 64, "copied by 16 lanes");

__host__ __device__ __forceinline__ int block_lo(const Entry& x, int kb) {      // even blocks, the first ones a tile longer
    const int q = x.n_tiles / x.blocks, r = x.n_tiles % x.blocks;
    return kb * q + (kb < r ? kb : r);
}
__host__ __device__ __forceinline__ int item_cost_tile(const PlanParams& p, const Entry& x, int it) {
    return (p.tiles_per_item == 1 || (x.single && it == x.items - 1)) ? p.cost_one : p.cost_two;
}
// first key tile of an item of n tiles that starts at cost `at` or later; tile 0 starts with the item
__host__ __device__ __forceinline__ int tile_at(const PlanParams& p, int start, int n, int cost, int at) {
    if (at <= start) return 0;
    const int j = (at - start - p.cost_item + cost - 1) / cost;
    return j < 1 ? 1 : j > n ? n : j;
}
// Item number k of an entry: kv head, key block, item of row tiles; its key tiles, cost a tile and start (from the entry's).
struct Item {
    int32_t kvh, kb, it, t0, n, cost, start;
};
__host__ __device__ __forceinline__ Item plan_item(const PlanParams& p, const Entry& x, int k) {
    Item m;
    m.it = k % x.items;
    m.kb = k / x.items % x.blocks;
    m.kvh = k / x.items / x.blocks;
    m.t0 = block_lo(x, m.kb);
    m.n = block_lo(x, m.kb + 1) - m.t0;
    m.cost = item_cost_tile(p, x, m.it);
    const int full = p.tiles_per_item == 1 ? p.cost_one : p.cost_two;      // of every row tile item but a single last one
    const int row = (x.items - 1) * full + item_cost_tile(p, x, x.items - 1);
    m.start = m.kvh * (x.cost / p.Hkv) + m.kb * x.items * p.cost_item + m.t0 * row + m.it * (p.cost_item + m.n * full);
    return m;
}
__host__ __device__ __forceinline__ int item_last(const PlanParams& p, const Item& m) {      // cost at which the last key tile starts, from the item's
    return m.n > 1 ? p.cost_item + (m.n - 1) * m.cost : 0;
}
// The key tiles of the item that CTA `cta` takes (start: cost of the item in the chain); false if none
__host__ __device__ __forceinline__ bool plan_segment(const PlanParams& p, const Entry& x, const Item& m, int start, int stretch, int cta, Segment& s) {
    const int a = tile_at(p, start, m.n, m.cost, cta * stretch), b = tile_at(p, start, m.n, m.cost, (cta + 1) * stretch);
    if (a >= b) return false;
    s.kvh = m.kvh;
    s.seq = x.seq;
    s.n_rows = x.n_rows;
    s.row0 = m.it * p.tiles_per_item * p.row_tile;
    s.two = p.tiles_per_item == 2 && !(x.single && m.it == x.items - 1);
    s.lo = x.lo;
    s.hi = x.hi;
    const int c0 = (m.t0 + a) * p.chunks_per_tile, end = (m.t0 + b) * p.chunks_per_tile, c1 = end < x.n_chunks ? end : x.n_chunks;
    s.chunk = x.chunk0 + c0;
    s.n_chunks = c1 - c0;
    s.block = x.block && c1 == x.n_chunks;
    s.ctx_chunks = s.n_chunks - s.block;
    return true;
}

// What the plan says to the other kernels.
// Of a sequence, for the merge: the items of its group (none: blocks = 0), its first packed row there, and its own items.
struct SeqInfo {
    int32_t group_item0, group_items, group_blocks, group_single;
    int32_t row_off, item0, blocks, n_group_items;     // n_group_items: of the call
};
static_assert(sizeof(SeqInfo) == 32, "two 16-byte loads");
struct PlanOut {
    Segment* segs;                       // [items + CTAs]: segment of item i in CTA c has index i + c, so a CTA's segments are neighbours
    int2* list;                          // [CTAs] first segment and number of them
    int2* ctas;                          // [items] first and last CTA
    SeqInfo* sinfo;                      // [S]
    Entry* entries;                      // [n_groups + S] scratch, used where shared memory is too small: entries, and the cost and item at
    int32_t* start;                      // [n_groups + S]      which each starts
    int32_t* item0;                      // [n_groups + S + 1]
};

constexpr int PLAN_THREADS = 512, MAX_CTAS = 512, PLAN_CACHE = 512;

// One CTA. Passes of all threads over groups and sequences (entries and their total cost, and which prefixes are read at all; then key blocks,
// running costs and items), then one thread per item. What takes its time is latency: lengths and groups are fetched once, and everything in between stays in shared memory where it fits.
__global__ void __launch_bounds__(PLAN_THREADS) prefix_plan_kernel(PlanParams p, const PlanOut o, int grid) {
    constexpr int NW = PLAN_THREADS / 32;
    __shared__ int32_t s_cost[NW], s_tiles[NW], s_items[NW];
    __shared__ int32_t s_first[MAX_CTAS], s_n[MAX_CTAS];
    __shared__ int32_t s_len[PLAN_CACHE], s_prefix[PLAN_CACHE], s_start[PLAN_CACHE + 1];
    __shared__ Entry s_entry[PLAN_CACHE];
    __shared__ int32_t s_at[PLAN_CACHE], s_item0[PLAN_CACHE + 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    ptx::pdl_trigger();
    for (int c = tid; c < grid; c += PLAN_THREADS) {
        s_first[c] = 0x7fffffff;
        s_n[c] = 0;
    }
    if (p.S <= PLAN_CACHE) {
        for (int b = tid; b < p.S; b += PLAN_THREADS) s_len[b] = p.ctx_len[b];
        p.ctx_len = s_len;
    }
    if (p.n_groups <= PLAN_CACHE && p.n_groups > 0) {
        for (int g = tid; g <= p.n_groups; g += PLAN_THREADS) {
            s_start[g] = p.group_start[g];
            if (g < p.n_groups) s_prefix[g] = p.prefix_len[g];
        }
        p.group_start = s_start;
        p.prefix_len = s_prefix;
    }
    const int n = p.n_groups + p.S, per = (n + PLAN_THREADS - 1) / PLAN_THREADS;
    const bool small = n <= PLAN_CACHE;
    Entry* ent = small ? s_entry : o.entries;
    int32_t *at = small ? s_at : o.start, *item0 = small ? s_item0 : o.item0;
    for (int g = tid; g < p.n_groups; g += PLAN_THREADS) at[g] = 0;          // until the running costs are known: whether a group's prefix is read
    __syncthreads();
    int bad = 0;
    for (int g = tid; g <= p.n_groups && p.n_groups > 0; g += PLAN_THREADS) {
        const int a = p.group_start[g];
        bad |= a < 0 || a > p.S || (g > 0 && p.group_start[g - 1] > a);
    }
    bad = __syncthreads_or(bad);
    const bool ok = !bad && p.n_groups > 0;
    if (bad && tid == 0 && p.status) atomicOr(p.status, DFLASH_DEV_BAD_GROUP);
    const int e0 = min(n, tid * per), e1 = min(n, e0 + per);         // this thread's entries
    int cost = 0, tiles = 0, items = 0;
#pragma unroll 1
    for (int e = e0; e < e1; ++e) {
        Entry x = plan_entry(p, e, ok, true);
        if (x.lo > 0) at[x.group] = 1;
        entry_cost(p, x);
        cost += x.cost;
        tiles += p.Hkv * x.items * x.n_tiles;
        ent[e] = x;
    }
    cost = __reduce_add_sync(0xffffffffu, cost);
    tiles = __reduce_add_sync(0xffffffffu, tiles);
    if (lane == 0) { s_cost[warp] = cost; s_tiles[warp] = tiles; }
    __syncthreads();
    int total = __reduce_add_sync(0xffffffffu, lane < NW ? s_cost[lane] : 0);
    tiles = __reduce_add_sync(0xffffffffu, lane < NW ? s_tiles[lane] : 0);
    if (plan_few(p, tiles, grid)) {
        p.cost_item = 0;
        total = tiles * p.cost_two;
    }
    const int share = (total + grid - 1) / grid;
    cost = 0;
#pragma unroll 1
    for (int e = e0; e < e1; ++e) {
        Entry x = ent[e];
        if (e < p.n_groups && !at[e]) {
            entry_unread(x);
            ent[e] = x;
        }
        entry_blocks(p, x, share);
        entry_cost(p, x);
        ent[e].blocks = x.blocks;
        ent[e].cost = x.cost;
        cost += x.cost;
        items += entry_items(p, x);
    }
    int run = cost, run_items = items;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, run, d), z = __shfl_up_sync(0xffffffffu, run_items, d);
        if (lane >= d) { run += y; run_items += z; }
    }
    __syncthreads();
    if (lane == 31) { s_cost[warp] = run; s_items[warp] = run_items; }
    __syncthreads();
    const int wc = lane < NW ? s_cost[lane] : 0, wi = lane < NW ? s_items[lane] : 0;        // one warp's sums per lane
    run += __reduce_add_sync(0xffffffffu, lane < warp ? wc : 0) - cost;
    run_items += __reduce_add_sync(0xffffffffu, lane < warp ? wi : 0) - items;
    total = __reduce_add_sync(0xffffffffu, wc);
    const int n_items = __reduce_add_sync(0xffffffffu, wi);
#pragma unroll 1
    for (int e = e0; e < e1; ++e) {
        const Entry x = ent[e];
        at[e] = run;
        item0[e] = run_items;
        run += x.cost;
        run_items += entry_items(p, x);
    }
    if (tid == 0) item0[n] = n_items;
    const int stretch = plan_stretch(p, total, grid);
    __syncthreads();
    const int n_group_items = item0[p.n_groups];
#pragma unroll 1
    for (int b = tid; b < p.S; b += PLAN_THREADS) {
        const Entry& x = ent[p.n_groups + b];
        SeqInfo q{0, 0, 0, 0, 0, item0[p.n_groups + b], x.blocks, n_group_items};
        if (x.lo > 0) {                  // the keys below x.lo are the group's items
            const int g = x.group;
            q = SeqInfo{item0[g], ent[g].items, ent[g].blocks, ent[g].single, (b - p.group_start[g]) * p.R * p.G, q.item0, q.blocks, n_group_items};
        }
        o.sinfo[b] = q;
    }
#pragma unroll 1
    for (int i = tid; i < n_items; i += PLAN_THREADS) {
        int lo = 0, hi = n;              // last entry that starts at item i or before (entries without items share a start)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (item0[mid] <= i) lo = mid;
            else hi = mid;
        }
        const Entry& x = ent[lo];
        const Item m = plan_item(p, x, i - item0[lo]);
        const int start = at[lo] + m.start, c0 = start / stretch, c1 = (start + item_last(p, m)) / stretch;
        o.ctas[i] = make_int2(c0, c1);
#pragma unroll 1
        for (int c = c0; c <= c1; ++c) {
            Segment s{};
            if (!plan_segment(p, x, m, start, stretch, c, s)) continue;
            s.prefix = lo < p.n_groups;
            s.slot = i + c - (s.prefix ? 0 : n_group_items);
            o.segs[i + c] = s;
            atomicMin(&s_first[c], i + c);
            atomicAdd(&s_n[c], 1);
        }
    }
    __syncthreads();
    for (int c = tid; c < grid; c += PLAN_THREADS) o.list[c] = make_int2(s_first[c], s_n[c]);
}

}  // namespace
}  // namespace dflash
