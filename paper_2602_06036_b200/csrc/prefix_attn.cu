// Block attention of a batch whose sequences share long prefixes.
//   out[b, r, h] = sum_k p_k v_k / sum_k p_k,   p_k = exp(scale q[b, r, h] . k_k - m),   lse = m + ln sum_k p_k
// over k = the cached positions of sequence b and the block's own rows. A softmax over a union of key sets is put together
// from its parts: with (m_i, l_i, o_i) of part i, M = max m_i,  out = sum e^(m_i - M) o_i / sum e^(m_i - M) l_i. So the rows of
// all sequences of a group go against the prefix as ONE matrix product, each sequence's rows go against its own keys,
// and a last launch merges the parts of every row in a fixed order. A small first launch cuts up the work (prefix_plan.cuh).
// The tensor-core kernel for bf16 is in prefix_attn_tc.cuh; here are the CUDA-core kernel, the merge and the launches.
#include "prefix_attn.cuh"

#include "prefix_attn_tc.cuh"

#include <algorithm>
#include <cstdint>
#include <memory>
#include <new>
#include <type_traits>

namespace dflash {
namespace {

using namespace ptx;

// ---- CUDA-core kernel: fp32, and bf16 with pages of less than 8 tokens ----------------------------------------------
// 64 packed rows against chunks of 64 keys; 256 threads, each 4 x 4 scores and 4 x hd/16 outputs. One call of few rows is bound by the latency of
// its loads: with a chunk's K and V all under way at once, 16 bytes a load, 3 sequences x 5 rows behind 40 fp32 positions take 19 us in a graph (25 with 4-byte loads).
constexpr int SIMT_THREADS = 256, SIMT_ROWS = 64;
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
}
template <int HD>
constexpr int simt_smem() { return (SIMT_ROWS * (HD + 4) * 2 + CHUNK_KEYS * HD + SIMT_ROWS * (CHUNK_KEYS + 4) + 2 * SIMT_ROWS) * 4; }

template <typename T, int HD>
__global__ void __launch_bounds__(SIMT_THREADS) prefix_attn_simt_kernel(const __grid_constant__ Params p) {
    extern __shared__ float sm[];
    float* sQ = sm;                                  // [64][HD + 4]
    float* sK = sQ + SIMT_ROWS * (HD + 4);           // [64][HD + 4]
    float* sV = sK + CHUNK_KEYS * (HD + 4);          // [64][HD]
    float* sP = sV + CHUNK_KEYS * HD;                // [64][68]
    float* sAlpha = sP + SIMT_ROWS * (CHUNK_KEYS + 4);
    if (threadIdx.x == 0) trace_min(p.trace, 0);
    pdl_trigger();
    pdl_wait();
    const int2 list = __ldcg(p.po.list + blockIdx.x);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;      // scores: rows 4 ty + i, keys tx + 16 j; outputs: columns 4 tx + 64 j
    const T *Q = (const T*)p.q, *KB = (const T*)p.k_blk, *VB = (const T*)p.v_blk, *pool = (const T*)p.pool;
    const int G = p.plan.G, R = p.plan.R, Hkv = p.plan.Hkv;
    for (int k = 0; k < list.y; ++k) {
        const Segment s = p.po.segs[list.x + k];
        __syncthreads();
        const int rows = min(SIMT_ROWS, s.n_rows - s.row0);
        for (int i = threadIdx.x; i < SIMT_ROWS * HD / 4; i += SIMT_THREADS) {
            const int row = i / (HD / 4), d = i % (HD / 4) * 4, pr = s.row0 + row;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (row < rows) v = load4(Q + (((int64_t)s.seq * R + pr / G) * p.Hq + s.kvh * G + pr % G) * HD + d);
            *reinterpret_cast<float4*>(sQ + row * (HD + 4) + d) = v;
        }
        float o[4][HD / 16], m[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = -CUDART_INF_F;
            l[i] = 0.f;
#pragma unroll
            for (int j = 0; j < HD / 16; ++j) o[i][j] = 0.f;
        }
        for (int c = 0; c < s.n_chunks; ++c) {
            const bool block = c >= s.ctx_chunks;
            const int key0 = (s.chunk + c) * CHUNK_KEYS;
            __syncthreads();                         // the previous chunk is used up
            // a key that does not exist loads as zeros and is masked below; 16 threads a key, each of which looks four keys up and then has all their loads under way
            unsigned long long exist = 0;
            const T *kp[4], *vp[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int key = 16 * k + ty;
                kp[k] = vp[k] = nullptr;
                if (block) {
                    if (key < R) {
                        kp[k] = KB + (((int64_t)s.seq * R + key) * Hkv + s.kvh) * HD;
                        vp[k] = VB + (((int64_t)s.seq * R + key) * Hkv + s.kvh) * HD;
                    }
                } else if (key0 + key >= s.lo && key0 + key < s.hi) {
                    const int pos = key0 + key, j = pos / p.page_size;
                    const int page = j < p.max_pages ? __ldg(p.page_table + (int64_t)s.seq * p.max_pages + j) : -1;
                    if (page >= 0 && page < p.n_pages) {
                        kp[k] = pool + ((((int64_t)p.layer * p.n_pages + page) * 2 * Hkv + s.kvh) * p.page_size + pos % p.page_size) * HD;
                        vp[k] = kp[k] + (int64_t)Hkv * p.page_size * HD;
                    } else if (tx == 0 && p.status) {
                        atomicOr(p.status, DFLASH_DEV_BAD_PAGE);
                    }
                }
                if (kp[k]) exist |= 1ull << key;
            }
            float4 kv[4][2][HD / 64];
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int x = 0; x < HD / 64; ++x) {
                    const int d = 64 * x + 4 * tx;
                    kv[k][0][x] = kp[k] ? load4(kp[k] + d) : make_float4(0.f, 0.f, 0.f, 0.f);
                    kv[k][1][x] = kp[k] ? load4(vp[k] + d) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int x = 0; x < HD / 64; ++x) {
                    const int key = 16 * k + ty, d = 64 * x + 4 * tx;
                    *reinterpret_cast<float4*>(sK + key * (HD + 4) + d) = kv[k][0][x];
                    *reinterpret_cast<float4*>(sV + key * HD + d) = kv[k][1][x];
                }
            // which keys exist, for everybody: each thread knows 4 of them
            uint32_t lo = (uint32_t)exist, hi = (uint32_t)(exist >> 32);
            lo = __reduce_or_sync(0xffffffffu, lo);
            hi = __reduce_or_sync(0xffffffffu, hi);
            uint32_t* words = reinterpret_cast<uint32_t*>(sAlpha + SIMT_ROWS);      // [8 warps][2]
            if ((threadIdx.x & 31) == 0) {
                words[(threadIdx.x >> 5) * 2] = lo;
                words[(threadIdx.x >> 5) * 2 + 1] = hi;
            }
            __syncthreads();
            lo = hi = 0;
            for (int k = 0; k < SIMT_THREADS / 32; ++k) { lo |= words[2 * k]; hi |= words[2 * k + 1]; }
            exist = ((unsigned long long)hi << 32) | lo;
            float z[4][4] = {};
            for (int d = 0; d < HD; d += 4) {
                float4 a[4], b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(sQ + (4 * ty + i) * (HD + 4) + d);
#pragma unroll
                for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const float4*>(sK + (tx + 16 * j) * (HD + 4) + d);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        z[i][j] = fmaf(a[i].x, b[j].x, fmaf(a[i].y, b[j].y, fmaf(a[i].z, b[j].z, fmaf(a[i].w, b[j].w, z[i][j]))));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = (s.row0 + 4 * ty + i) / G;
                const unsigned long long seen = block && p.causal ? exist & (r >= 63 ? ~0ull : (2ull << r) - 1) : exist;
                float mx = -CUDART_INF_F;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    z[i][j] = (seen >> (tx + 16 * j) & 1) ? z[i][j] * p.scale_log2 : -CUDART_INF_F;
                    mx = fmaxf(mx, z[i][j]);
                }
#pragma unroll
                for (int x = 8; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
                const float m_new = fmaxf(m[i], mx), m_use = m_new > -CUDART_INF_F ? m_new : 0.f;
                const float alpha = m[i] > -CUDART_INF_F ? exp2f(m[i] - m_use) : 0.f;
                m[i] = m_new;
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = exp2f(z[i][j] - m_use);
                    sum += e;
                    sP[(4 * ty + i) * (CHUNK_KEYS + 4) + tx + 16 * j] = e;
                }
#pragma unroll
                for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
                l[i] = l[i] * alpha + sum;
#pragma unroll
                for (int j = 0; j < HD / 16; ++j) o[i][j] *= alpha;
            }
            __syncwarp();                            // a row's 16 threads sit in one warp
            // hidden: a row of V that a row does not see has no say in it, whatever it holds (0 x infinity is NaN)
            auto values = [&](auto hidden) {
                for (int key = 0; key < CHUNK_KEYS; ++key) {
                    float pr[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) pr[i] = sP[(4 * ty + i) * (CHUNK_KEYS + 4) + key];
#pragma unroll
                    for (int j = 0; j < HD / 64; ++j) {
                        const float4 v = *reinterpret_cast<const float4*>(sV + key * HD + 64 * j + 4 * tx);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (hidden && key > (s.row0 + 4 * ty + i) / G) continue;
                            o[i][4 * j + 0] = fmaf(pr[i], v.x, o[i][4 * j + 0]);
                            o[i][4 * j + 1] = fmaf(pr[i], v.y, o[i][4 * j + 1]);
                            o[i][4 * j + 2] = fmaf(pr[i], v.z, o[i][4 * j + 2]);
                            o[i][4 * j + 3] = fmaf(pr[i], v.w, o[i][4 * j + 3]);
                        }
                    }
                }
            };
            if (block && p.causal) values(std::true_type{});
            else values(std::false_type{});
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 4 * ty + i;
            if (row >= rows) continue;
            const int64_t at = slot_row(p, s.prefix != 0, s.slot, 0, row);
            if (tx == 0) p.ml[at] = make_float2(m[i], l[i]);
#pragma unroll
            for (int j = 0; j < HD / 64; ++j)
                *reinterpret_cast<float4*>(p.part + part_offset(at, HD, 16 * j + tx)) = make_float4(o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]);
        }
    }
    if (threadIdx.x == 0) trace_max(p.trace, 3);
}

// ---- merge ----------------------------------------------------------------------------------------------------------
// Four neighbouring packed rows of a (sequence, kv head) by W warps (eight lanes a row), each of which takes every W-th part of these rows; their sums are
// added up at the end, so that the order is fixed. A warp requests PB parts together, results and statistics alike: the kernel waits for L2, not
// for bytes. W = 4 where there are few rows (decoding: 8.3 -> 5.4 us), W = 1 where there are enough for all SMs, which is said of 8 units (of four rows) an SM.
// Whole calls behind 4096 positions, W = 4 and W = 1: 1024 units 39.6 us and 42.8, 1280 (on W = 1's side) 46.6 and 50.3, 1536 47.4 and 46.5, 2048 54.8 and 50.7, 4096 85.7 and 75.4.
template <typename T, int HD, int W>
__global__ void __launch_bounds__(128) prefix_merge_kernel(const __grid_constant__ Params p) {
    constexpr int PB = 4;
    __shared__ float4 s_acc[W == 1 ? 1 : 4][4][HD / 4];
    __shared__ float2 s_ml[4][4];
    unsigned long long* trace = p.trace ? p.trace + 4 : nullptr;
    if (threadIdx.x == 0) trace_min(trace, 0);
    const int RG = p.plan.R * p.plan.G, per_head = (RG + 3) / 4;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub8 = lane >> 2;          // columns 4 sub8 + 32 k
    const int unit = W == 1 ? blockIdx.x * 4 + warp : blockIdx.x, row0 = unit % per_head * 4;
    const int bh = min(unit / per_head, p.plan.S * p.plan.Hkv - 1), b = bh / p.plan.Hkv, kvh = bh % p.plan.Hkv;
    const int pr = min(row0 + (lane & 3), RG - 1);                                        // rows behind the last one repeat it
    const int tpi = p.plan.tiles_per_item, tr = p.plan.row_tile;
    pdl_wait();
    if (threadIdx.x == 0) trace_min(trace, 1);
    const int4* sp = reinterpret_cast<const int4*>(p.po.sinfo + b);
    const int4 s0 = __ldcg(sp), s1 = __ldcg(sp + 1);
    const SeqInfo si{s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
    const int gat = si.row_off + pr, gtile = gat / tr, otile = pr / tr, own_tiles = (RG + tr - 1) / tr, own_items = (own_tiles + tpi - 1) / tpi;
    const bool g_one = si.group_single && gtile / tpi == si.group_items - 1, o_one = own_tiles % tpi != 0 && otile / tpi == own_items - 1;   // one query tile

    float M = -CUDART_INF_F, L = 0.f;
    float4 acc[HD / 32];
#pragma unroll
    for (int k = 0; k < HD / 32; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    // The row's items: key blocks of the group, then its own. Its eight lanes look eight of them up at a time, and then go through
    // all the parts of these.
    const int n_items = si.group_blocks + si.blocks;
    int skip = W == 1 ? 0 : warp;                    // parts until this warp's next one
    const int most = __reduce_max_sync(0xffffffffu, n_items);
    for (int e0 = 0; e0 < most; e0 += 8) {
        const int e = e0 + sub8, kb = e - si.group_blocks;
        int slot = 0, n = 0;                         // of item e: slot of its first part, parts
        if (e < n_items) {
            const bool own = kb >= 0;
            const int item = own ? si.item0 + (kvh * si.blocks + kb) * own_items + otile / tpi
                                 : si.group_item0 + (kvh * si.group_blocks + e) * si.group_items + gtile / tpi;
            const int2 ctas = __ldcg(p.po.ctas + item);
            slot = item + ctas.x - (own ? si.n_group_items : 0);
            n = (ctas.y - ctas.x + 1) * (tpi == 2 && (own ? o_one : g_one) ? 2 : 1);
        }
        int end = n;                                 // parts up to this item's end
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, end, d);
            if (lane >= d) end += y;
        }
        const int total = __shfl_sync(0xffffffffu, end, 28 + (lane & 3));
        const int rounds = __reduce_max_sync(0xffffffffu, total);
        for (int k0 = 0; k0 < rounds; k0 += W * PB) {      // the same for all lanes, which exchange values in it; rows differ in `skip` and `total`
            float2 ml[PB];
            float4 o[PB][HD / 32];
#pragma unroll
            for (int k = 0; k < PB; ++k) {
                const int part = skip + k0 + W * k;
                // the item that holds it: as many of the row's items end before it; and that item's first part
                const int x = min(__popc(__ballot_sync(0xffffffffu, part >= end) & 0x11111111u << (lane & 3)), 7);
                const int before = __shfl_sync(0xffffffffu, end, 4 * max(x - 1, 0) + (lane & 3)), first = x > 0 ? before : 0;
                const int sl = __shfl_sync(0xffffffffu, slot, 4 * x + (lane & 3));
                const bool own = e0 + x >= si.group_blocks, two_subs = tpi == 2 && (own ? o_one : g_one);
                ml[k] = make_float2(-CUDART_INF_F, 0.f);
                if (part < total) {
                    const int q = part - first, tile = own ? otile : gtile;
                    const int64_t r = slot_row(p, !own, sl + (two_subs ? q >> 1 : q), two_subs ? q & 1 : tile % tpi, (own ? pr : gat) - tile * tr);
                    ml[k] = __ldcg(p.ml + r);
#pragma unroll
                    for (int c = 0; c < HD / 32; ++c) o[k][c] = __ldcg(reinterpret_cast<const float4*>(p.part + part_offset(r, HD, c * 8 + sub8)));
                }
            }
            float top = M;
#pragma unroll
            for (int k = 0; k < PB; ++k)
                if (ml[k].y != 0.f) top = fmaxf(top, ml[k].x);
            const float ref = top > -CUDART_INF_F ? top : 0.f;
            const float keep = M > -CUDART_INF_F ? exp2f(M - ref) : 0.f;
            M = top;
            L *= keep;
#pragma unroll
            for (int x = 0; x < HD / 32; ++x) { acc[x].x *= keep; acc[x].y *= keep; acc[x].z *= keep; acc[x].w *= keep; }
#pragma unroll
            for (int k = 0; k < PB; ++k) {
                if (ml[k].y == 0.f) continue;        // no key in that part: what lies there was never written
                const float wgt = exp2f(ml[k].x - ref);
                L = fmaf(ml[k].y, wgt, L);
#pragma unroll
                for (int x = 0; x < HD / 32; ++x) {
                    acc[x].x = fmaf(o[k][x].x, wgt, acc[x].x);
                    acc[x].y = fmaf(o[k][x].y, wgt, acc[x].y);
                    acc[x].z = fmaf(o[k][x].z, wgt, acc[x].z);
                    acc[x].w = fmaf(o[k][x].w, wgt, acc[x].w);
                }
            }
        }
        // parts of this warp among the next eight items: those at `skip`, `skip` + W, ... of them
        const int passed = total - skip;
        skip = passed <= 0 ? -passed : (W - passed % W) % W;
    }
    auto store = [&](int r4, int c, float4 v, float m, float sum) {      // four columns of row row0 + r4
        const int prow = row0 + r4;
        if (prow >= RG || unit / per_head >= p.plan.S * p.plan.Hkv) return;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;                  // a row that saw no key gives zeros
        const int64_t r = (int64_t)b * p.plan.R + prow / p.plan.G;
        const int head = kvh * p.plan.G + prow % p.plan.G;
        if (p.lse && c == 0) p.lse[r * p.Hq + head] = sum == 0.f ? -CUDART_INF_F : (m + log2f(sum)) * 0.6931471805599453f;
        T* dst = (T*)p.out + (r * p.Hq + head) * HD + c;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(dst) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
        else *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
    };
    if constexpr (W == 1) {
#pragma unroll
        for (int x = 0; x < HD / 32; ++x) store(lane & 3, x * 32 + sub8 * 4, acc[x], M > -CUDART_INF_F ? M : 0.f, L);
    } else {                                         // the four warps' sums, by warp; then a warp a row
#pragma unroll
        for (int x = 0; x < HD / 32; ++x) s_acc[warp][lane & 3][x * 8 + sub8] = acc[x];
        if (sub8 == 0) s_ml[warp][lane & 3] = make_float2(M, L);
        __syncthreads();
        float top = -CUDART_INF_F, sum = 0.f, w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) top = fmaxf(top, s_ml[k][warp].x);
        const float ref = top > -CUDART_INF_F ? top : 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[k] = exp2f(s_ml[k][warp].x - ref);
            sum = fmaf(s_ml[k][warp].y, w[k], sum);
        }
        if (lane < HD / 4) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float4 x = s_acc[k][warp][lane];
                v.x = fmaf(x.x, w[k], v.x); v.y = fmaf(x.y, w[k], v.y); v.z = fmaf(x.z, w[k], v.z); v.w = fmaf(x.w, w[k], v.w);
            }
            store(warp, lane * 4, v, ref, sum);
        }
    }
    if (threadIdx.x == 0) trace_max(trace, 3);
}

// ---- host ---------------------------------------------------------------------------------------------------------
bool use_tc(const dflash_config& c) { return c.dtype == DFLASH_BF16 && c.page_size >= 8; }

struct Sizes {
    int n_cta, row_tile, tiles_per_item, chunks_per_tile, own_rows;
    int64_t group_items, own_items, group_slots, own_slots;
};
Sizes sizes(const dflash_config& c, int64_t S, int64_t R, int64_t n_groups, int sm_count) {
    Sizes z{};
    const int G = c.n_q_heads / c.n_kv_heads;
    const bool tc = use_tc(c);
    z.n_cta = tc ? sm_count : 2 * sm_count;
    z.row_tile = tc ? 128 / G * G : SIMT_ROWS;
    z.tiles_per_item = z.chunks_per_tile = tc ? 2 : 1;
    z.own_rows = (int)align_up(std::min<int64_t>(R * G, z.row_tile), 8);
    // an upper bound of what plan_cta counts: a key block more than one costs at least half a CTA's share
    const int64_t per_item = (int64_t)z.row_tile * z.tiles_per_item;
    z.group_items = c.n_kv_heads * (S * R * G / per_item + std::min(n_groups, S)) + 2 * z.n_cta;
    z.own_items = c.n_kv_heads * S * ((R * G + per_item - 1) / per_item) + 2 * z.n_cta;
    z.group_slots = n_groups > 0 ? z.group_items + z.n_cta : 0;
    if (n_groups == 0) z.group_items = 0;
    z.own_slots = z.own_items + z.n_cta;
    return z;
}
struct PrefixWs {
    float* part;
    float2* ml;
    PlanOut po;
    int64_t bytes;
};
PrefixWs carve_prefix(void* base, const Sizes& z, const dflash_config& c, int64_t S, int64_t n_groups) {
    Arena a(base);
    PrefixWs w{};
    const int64_t rows = z.group_slots * 256 + z.own_slots * 2 * z.own_rows;
    w.part = (float*)a.take(rows * c.head_dim * 4);
    w.ml = (float2*)a.take(rows * 8);
    const int64_t items = z.group_items + z.own_items, n = n_groups + S;
    w.po.segs = (Segment*)a.take((items + z.n_cta) * sizeof(Segment));
    w.po.list = (int2*)a.take(z.n_cta * sizeof(int2));
    w.po.ctas = (int2*)a.take(items * sizeof(int2));
    w.po.sinfo = (SeqInfo*)a.take(S * sizeof(SeqInfo));
    w.po.entries = (Entry*)a.take(n > PLAN_CACHE ? n * sizeof(Entry) : 0);
    w.po.start = (int32_t*)a.take(n * 4);
    w.po.item0 = (int32_t*)a.take((n + 1) * 4);
    w.bytes = a.off;
    return w;
}
PlanParams plan_params(const dflash_config& c, const Sizes& z, int S, int R, int n_groups, int max_ctx_len) {
    PlanParams q{};
    q.S = S; q.R = R; q.G = c.n_q_heads / c.n_kv_heads; q.Hkv = c.n_kv_heads; q.n_groups = n_groups; q.max_ctx_len = max_ctx_len;
    q.row_tile = z.row_tile; q.tiles_per_item = z.tiles_per_item; q.chunks_per_tile = z.chunks_per_tile;
    // Tensor-core kernel, in units of 500 clocks: a key tile takes 2650 with one query tile (its bytes at the HBM rate) and 3560 with two (its products),
    // the change to another item about 4500. (One query tile for as much as two, 8 : 5 : 9, left CTAs waiting: 32 sequences x 17 rows behind
    // 32768 positions 311 us, then 282; an item for 12 is better for many whole contexts, 112 us against 116, and no better or worse elsewhere.)
    // CUDA cores: a chunk takes about as long as it takes to begin an item.
    const bool tc = use_tc(c);
    q.cost_item = tc ? 10 : 3; q.cost_one = tc ? 5 : 4; q.cost_two = tc ? 7 : 4;
    return q;
}
// whether the costs of any lengths up to max_ctx_len stay below 2^31 with room for the sums that plan_kernel forms
bool plan_fits(const dflash_config& c, const Sizes& z, int64_t S, int64_t R, int64_t n_groups, int64_t max_ctx_len) {
    const int64_t G = c.n_q_heads / c.n_kv_heads, per_item = (int64_t)z.row_tile * z.tiles_per_item;
    const int64_t tiles = max_ctx_len / (CHUNK_KEYS * z.chunks_per_tile) + 3;
    const int64_t items = S * ((R * G + per_item - 1) / per_item) + (S * R * G / per_item + std::min(n_groups, S));
    return items <= (1 << 24) && c.n_kv_heads * items * tiles * 17 < (1ll << 30);
}

template <int HD>
int launch_tc(const Launch& L, const dflash_prefix_attn_args& a, const Params& p, int n_cta) {
    const dflash_config& c = L.h->cfg;
    const int G = p.plan.G, Hkv = p.plan.Hkv;
    CUtensorMap tq, tpool, tkb, tvb;
    {   // q as [S*R][Hkv][G][hd]: a box of whole (sequence, row)s holds packed rows
        const uint64_t dims[4] = {(uint64_t)HD, (uint64_t)G, (uint64_t)Hkv, (uint64_t)a.batch * a.rows};
        const uint64_t str[3] = {(uint64_t)HD * 2, (uint64_t)G * HD * 2, (uint64_t)p.Hq * HD * 2};
        const uint32_t box[4] = {64, (uint32_t)G, 1, (uint32_t)p.rows_per_tile};
        if (!tmap_encode_bf16(&tq, a.q, 4, dims, str, box)) return DFLASH_ERR_CUDA;
    }
    {
        const uint64_t dims[2] = {(uint64_t)HD, (uint64_t)c.n_layers * a.n_pool_pages * 2 * Hkv * c.page_size};
        const uint64_t str[1] = {(uint64_t)HD * 2};
        const uint32_t box[2] = {64, (uint32_t)p.box};
        if (!tmap_encode_bf16(&tpool, a.kv_pool, 2, dims, str, box)) return DFLASH_ERR_CUDA;
    }
    {
        const uint64_t dims[2] = {(uint64_t)Hkv * HD, (uint64_t)a.batch * a.rows};
        const uint64_t str[1] = {(uint64_t)Hkv * HD * 2};
        const uint32_t box[2] = {64, 32};
        if (!tmap_encode_bf16(&tkb, a.k_blk, 2, dims, str, box) || !tmap_encode_bf16(&tvb, a.v_blk, 2, dims, str, box)) return DFLASH_ERR_CUDA;
    }
    static bool set[MAX_DEVICES] = {};
    const int dev = current_device_slot();
    if (dev < 0 || !set[dev]) {
        if (cudaFuncSetAttribute(prefix_attn_tc_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<HD>::SMEM) != cudaSuccess) return DFLASH_ERR_CUDA;
        if (dev >= 0) set[dev] = true;
    }
    return launch_pdl(prefix_attn_tc_kernel<HD>, dim3(n_cta), dim3(N_THREADS), (size_t)Shape<HD>::SMEM, L.st, tq, tpool, tkb, tvb, p) == cudaSuccess
               ? DFLASH_OK : DFLASH_ERR_CUDA;
}
template <typename T, int HD>
int launch_simt(const Launch& L, const Params& p, int n_cta) {
    constexpr int smem = simt_smem<HD>();
    static bool set[MAX_DEVICES] = {};
    const int dev = current_device_slot();
    if (dev < 0 || !set[dev]) {
        if (cudaFuncSetAttribute(prefix_attn_simt_kernel<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return DFLASH_ERR_CUDA;
        if (dev >= 0) set[dev] = true;
    }
    return launch_pdl(prefix_attn_simt_kernel<T, HD>, dim3(n_cta), dim3(SIMT_THREADS), (size_t)smem, L.st, p) == cudaSuccess ? DFLASH_OK : DFLASH_ERR_CUDA;
}

template <typename T, int HD>
int launch_merge(const Launch& L, const Params& p) {
    const int64_t units = (int64_t)p.plan.S * p.plan.Hkv * ((p.plan.R * p.plan.G + 3) / 4);
    const cudaError_t e = units >= 8 * (int64_t)L.h->sm_count
        ? launch_pdl(prefix_merge_kernel<T, HD, 1>, dim3((unsigned)((units + 3) / 4)), dim3(128), 0, L.st, p)
        : launch_pdl(prefix_merge_kernel<T, HD, 4>, dim3((unsigned)units), dim3(128), 0, L.st, p);
    return e == cudaSuccess ? DFLASH_OK : DFLASH_ERR_CUDA;
}

}  // namespace

bool prefix_attn_supported(const dflash_config& c) { return c.n_q_heads / c.n_kv_heads <= 128; }

int64_t prefix_attn_workspace_bytes(const dflash_handle* h, int64_t batch, int64_t rows, int64_t groups) {
    const Sizes z = sizes(h->cfg, batch, rows, groups, h->sm_count);
    return carve_prefix(nullptr, z, h->cfg, batch, groups).bytes;
}

int prefix_plan_check(const dflash_config& c, int sm_count, int S, int R, int n_groups, const int32_t* group_start, const int32_t* prefix_len,
                      const int32_t* ctx_len, int max_ctx_len, int64_t* info) {
    const Sizes z = sizes(c, S, R, n_groups, sm_count);
    if (!plan_fits(c, z, S, R, n_groups, max_ctx_len)) return -2;
    PlanParams p = plan_params(c, z, S, R, n_groups, max_ctx_len);
    p.group_start = group_start; p.prefix_len = prefix_len; p.ctx_len = ctx_len;
    const int n = n_groups + S;
    int total = 0, all_tiles = 0;
    const std::unique_ptr<char[]> read(new (std::nothrow) char[n]());       // of a group: any of its sequences reads the prefix
    if (!read) return DFLASH_ERR_CUDA;
    for (int e = 0; e < n; ++e) {
        Entry x = plan_entry(p, e, n_groups > 0, false);
        if (x.lo > 0) read[x.group] = 1;
        entry_cost(p, x);
        total += x.cost;
        all_tiles += p.Hkv * x.items * x.n_tiles;
    }
    if (plan_few(p, all_tiles, z.n_cta)) {
        p.cost_item = 0;
        total = all_tiles * p.cost_two;
    }
    const int share = (total + z.n_cta - 1) / z.n_cta;
    auto entry = [&](int e) {
        Entry x = plan_entry(p, e, n_groups > 0, false);
        if (e < n_groups && !read[e]) entry_unread(x);
        entry_blocks(p, x, share);
        entry_cost(p, x);
        return x;
    };
    int64_t items = 0, group_items = 0, tiles = 0, segments = 0;
    total = all_tiles = 0;
    for (int e = 0; e < n; ++e) {
        const Entry x = entry(e);
        all_tiles += p.Hkv * x.items * x.n_tiles;
        if (e == n_groups) group_items = items;
        total += x.cost;
        items += entry_items(p, x);
    }
    int rc = group_items > z.group_items || items - group_items > z.own_items ? 1 : 0;
    const int stretch = plan_stretch(p, total, z.n_cta);
    int at = 0, cta = 0, spent = 0, most = 0, least = INT32_MAX;      // the chain is followed item by item: CTAs take turns without a gap
    int64_t i = 0;
    for (int e = 0; rc == 0 && e < n; ++e) {
        const Entry x = entry(e);
        const int entry_at = at, count = entry_items(p, x);
        for (int k = 0; rc == 0 && k < count; ++k, ++i) {
            const Item m = plan_item(p, x, k);
            if (m.kvh < 0 || m.kvh >= p.Hkv || m.n < 1 || entry_at + m.start != at) { rc = 2; break; }      // an item starts where the one before it ends
            const int c0 = at / stretch, c1 = (at + item_last(p, m)) / stretch;
            if (c0 < cta || c0 > cta + 1 || c1 >= z.n_cta) { rc = 3; break; }
            int chunk = x.chunk0 + m.t0 * p.chunks_per_tile;
            for (int c = c0; c <= c1; ++c) {
                Segment s{};
                if (!plan_segment(p, x, m, at, stretch, c, s)) { rc = 4; break; }       // a CTA without work between two that have some
                if (c != cta) {
                    most = std::max(most, spent);
                    least = std::min(least, spent);
                    spent = 0;
                }
                cta = c;
                const int t = (s.n_chunks + p.chunks_per_tile - 1) / p.chunks_per_tile;
                if (s.chunk != chunk || s.n_chunks < 1 || (c < c1 && s.n_chunks % p.chunks_per_tile)) rc = 5;
                chunk += s.n_chunks;
                if (s.row0 >= s.n_rows || (s.two && s.row0 + p.row_tile >= s.n_rows)) rc = 6;
                if (s.ctx_chunks > 0 && (s.chunk + s.ctx_chunks - 1) * (int64_t)CHUNK_KEYS >= s.hi) rc = 6;
                const bool group = e < n_groups;
                if (i + c - (group ? 0 : group_items) >= (group ? z.group_slots : z.own_slots)) rc = 7;
                tiles += t;
                spent += (c == c0 ? p.cost_item : 0) + t * m.cost;
                ++segments;
            }
            if (rc == 0 && chunk - x.chunk0 != std::min((m.t0 + m.n) * p.chunks_per_tile, x.n_chunks)) rc = 5;
            at += p.cost_item + m.n * m.cost;
        }
    }
    if (rc == 0 && (tiles != all_tiles || at != total || i != items)) rc = 8;
    if (info) { info[0] = items; info[1] = group_items; info[2] = tiles; info[3] = segments; info[4] = least; info[5] = most; }
    return rc;
}

int launch_prefix_attention(const Launch& L, const dflash_prefix_attn_args& a) {
    const dflash_config& c = L.h->cfg;
    const Sizes z = sizes(c, a.batch, a.rows, a.n_groups, L.h->sm_count);
    const PrefixWs w = carve_prefix(a.workspace, z, c, a.batch, a.n_groups);
    Params p{};
    p.plan = plan_params(c, z, a.batch, a.rows, a.n_groups, a.max_ctx_len);
    p.plan.group_start = a.group_start; p.plan.prefix_len = a.prefix_len; p.plan.ctx_len = a.ctx_len; p.plan.status = L.status;
    p.Hq = c.n_q_heads; p.page_size = c.page_size; p.max_pages = a.max_pages; p.n_pages = a.n_pool_pages; p.layer = a.layer;
    p.causal = a.mode == DFLASH_ATTN_CAUSAL;
    p.box = std::min(c.page_size, 64);
    p.rows_per_tile = z.row_tile / p.plan.G;
    p.group_slots = (int)z.group_slots; p.own_rows = z.own_rows;
    p.scale_log2 = c.softmax_scale * 1.4426950408889634f;
    p.page_table = a.page_table; p.q = a.q; p.k_blk = a.k_blk; p.v_blk = a.v_blk; p.pool = a.kv_pool; p.out = a.out; p.lse = a.lse_out;
    p.part = w.part; p.ml = w.ml; p.po = w.po;
    p.status = L.status; p.trace = L.trace;
    if (z.n_cta > MAX_CTAS || !plan_fits(c, z, a.batch, a.rows, a.n_groups, a.max_ctx_len)) return DFLASH_ERR_UNSUPPORTED;
    // plain stream order: the plan reads lengths that the caller's previous call may have written
    const cudaError_t e = launch_ordered(prefix_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, L.st, p.plan, w.po, z.n_cta);
    if (e != cudaSuccess) return DFLASH_ERR_CUDA;
    ++g_launches;
    const bool wide = c.head_dim == 128;
    int rc;
    if (use_tc(c)) rc = wide ? launch_tc<128>(L, a, p, z.n_cta) : launch_tc<64>(L, a, p, z.n_cta);
    else if (c.dtype == DFLASH_F32) rc = wide ? launch_simt<float, 128>(L, p, z.n_cta) : launch_simt<float, 64>(L, p, z.n_cta);
    else rc = wide ? launch_simt<__nv_bfloat16, 128>(L, p, z.n_cta) : launch_simt<__nv_bfloat16, 64>(L, p, z.n_cta);
    if (rc != DFLASH_OK) return rc;
    ++g_launches;
    if (c.dtype == DFLASH_F32) rc = wide ? launch_merge<float, 128>(L, p) : launch_merge<float, 64>(L, p);
    else rc = wide ? launch_merge<__nv_bfloat16, 128>(L, p) : launch_merge<__nv_bfloat16, 64>(L, p);
    if (rc != DFLASH_OK) return rc;
    ++g_launches;
    return DFLASH_OK;
}

}  // namespace dflash
