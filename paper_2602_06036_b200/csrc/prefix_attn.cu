// Block attention of a batch whose sequences share long prefixes.
//   out[b, r, h] = sum_k p_k v_k / sum_k p_k,   p_k = exp(scale q[b, r, h] . k_k - m),   lse = m + ln sum_k p_k
// over k = the cached positions of sequence b and the block's own rows. A softmax over a union of key sets is put together
// from its parts: with (m_i, l_i, o_i) of part i, M = max m_i,  out = sum e^(m_i - M) o_i / sum e^(m_i - M) l_i. So the rows of
// all sequences of a group go against the prefix as ONE matrix product, each sequence's rows go against its own keys,
// and a second launch merges the parts of every row in a fixed order (prefix_plan.cuh cuts up the work).
//
// Tensor-core kernel (bf16): one persistent CTA per SM with a TMA warp, an MMA warp and two softmax warpgroups. An item with two
// query tiles (128 rows each) gives one to each warpgroup, which read every K/V tile of 128 keys together; an item
// with one tile has the warpgroups take alternate key tiles. So while one warpgroup is at its exponentials the tensor core works for the other.
//   S_t = Q_t K^T   tcgen05.mma, operands in shared memory, 128 x 128 fp32 in TMEM
//   softmax         one thread per row; the running maximum is only raised when a tile tops it by more than 2^8 (the row of O_t in
//                   TMEM is then rescaled in place); P goes back into the TMEM columns of S as bf16
//   O_t += P_t V    tcgen05.mma with P from TMEM, V as an MN-major operand straight from the page layout
// K and V tiles go through one ring of 32 KB stages that runs on across items. Every wait is bounded.
#include "prefix_attn.cuh"

#include "prefix_plan.cuh"
#include "ptx_sm100.cuh"

#include <math_constants.h>

#include <algorithm>
#include <cstdint>
#include <new>

namespace dflash {
namespace {

using namespace ptx;

constexpr float GAP = 8.f;               // log2 units by which a tile has to top the running maximum to raise it

struct Params {
    PlanParams plan;
    int32_t Hq, page_size, max_pages, n_pages, layer, causal;
    int32_t box;                         // keys per copy: min(page_size, 64)
    int32_t rows_per_tile;               // (sequence, row) pairs per query tile
    int32_t group_slots;                 // partial results of group items come first
    int32_t own_rows;                    // packed rows of a partial result of a sequence item (a multiple of 8)
    float scale_log2;
    const int32_t* page_table;
    const void *q, *k_blk, *v_blk, *pool;
    void* out;
    float* lse;
    float* part;                         // [group_slots][2][128] rows, then [own slots][2][own_rows]
    float2* ml;                          // (running maximum in log2 units, sum) of the same rows
    int32_t *cta0, *cta1;                // first and last CTA of an item: group items, then those of sequences
    int32_t group_items;                 // entries of cta0 / cta1 kept for group items
    GroupInfo* ginfo;
    SeqInfo* sinfo;
    int32_t* meta;                       // [0] number of group items
    int32_t* status;
    unsigned long long* trace;
};
// Partial results are kept in groups of 8 rows x hd: [row / 8][hd / 4][row % 8][4], so that neighbouring threads (rows) write,
// and the merge's lanes read, whole 128-byte lines.
__device__ __forceinline__ int64_t slot_row(const Params& p, bool group, int slot, int sub, int row) {
    return group ? ((int64_t)slot * 2 + sub) * 128 + row : (int64_t)p.group_slots * 256 + ((int64_t)slot * 2 + sub) * p.own_rows + row;
}
__device__ __forceinline__ int64_t part_offset(int64_t row, int hd, int c4) { return (row >> 3) * 8 * hd + c4 * 32 + (row & 7) * 4; }

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&t);
}

// ---- tensor-core kernel -----------------------------------------------------------------------------------------
constexpr int N_THREADS = 320;           // warps 0-3, 4-7: softmax; 8: copies; 9: MMA
constexpr int KT = 128;                  // keys per tile
constexpr uint32_t TMEM_COLS = 512;      // S0 | S1 | O0 | O1, 128 columns each
constexpr int NI = 16;                   // ring of tile masks: more tiles than the K/V ring can hold (checked below)

struct TileInfo {
    unsigned long long mask[2];          // keys of each chunk that exist
    int32_t causal_chunk;                // chunk (0 or 1) that holds the block in causal mode, else 2
    int32_t full;                        // all 128 keys exist and nothing is causal
};
template <int HD>
struct Shape {
    static constexpr int HALVES = HD / 64;                    // 64-element (128-byte) column halves of an operand
    static constexpr int Q_BYTES = 128 * HD * 2;
    static constexpr int STAGE = KT * HD * 2;
    static constexpr int NS = HD == 128 ? 5 : 10;
    static constexpr int SMEM = 1024 + 2 * Q_BYTES + NS * STAGE + 1536;
    static_assert(SMEM <= 227 * 1024, "shared memory of one CTA");
    static_assert(NI > NS, "a tile's mask outlives its K and V stages");
};

__device__ __forceinline__ void tmem_ld32_nowait(uint32_t taddr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// V tile as MN-major operand: [key][64 elements] halves, `half_bytes` apart, 8-key groups 1 KiB apart
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr, uint32_t half_bytes) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(half_bytes >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// D += A B with A (bf16, M rows in the TMEM lanes, two K elements a column) in TMEM
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Positions of a segment's loads in the ring (load n of the CTA uses stage n % NS, its (n / NS)-th use). Two query tiles: K0 V0 K1 V1 ...;
// one tile: K0 K1 V0 K2 V1 ..., the order in which the MMA warp needs them.
__device__ __forceinline__ int load_k(int two, int n, int j) { return two ? 2 * j : (j == 0 ? 0 : 2 * j - 1); }
__device__ __forceinline__ int load_v(int two, int n, int j) { return two ? 2 * j + 1 : (j + 1 < n ? 2 * j + 2 : 2 * n - 1); }

template <int HD>
__global__ void __launch_bounds__(N_THREADS, 1)
prefix_attn_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmPool, const __grid_constant__ CUtensorMap tmKb,
                      const __grid_constant__ CUtensorMap tmVb, const __grid_constant__ Params p) {
    using Sh = Shape<HD>;
    constexpr int NS = Sh::NS;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sQ = smem;
    uint8_t* ring = sQ + 2 * Sh::Q_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(ring + NS * Sh::STAGE);
    uint64_t* q_full = bars;
    uint64_t* q_empty = bars + 1;
    uint64_t* full = bars + 2;             // [NS]
    uint64_t* empty = full + NS;           // [NS]
    uint64_t* s_full = empty + NS;         // [2] S_t written (and all earlier products done)
    uint64_t* p_full = s_full + 2;         // [2] P_t written, O_t rescaled, missing V rows zeroed
    uint64_t* o_full = p_full + 2;         // [2] the segment's last product into O_t done
    TileInfo* infos = reinterpret_cast<TileInfo*>(o_full + 2);          // [NI]
    Segment* seg_sh = reinterpret_cast<Segment*>(infos + NI);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(seg_sh + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    PlanShared* plan_sh = reinterpret_cast<PlanShared*>(ring);          // before the ring is in use
    static_assert(sizeof(uint64_t) * (8 + 2 * NS) + sizeof(TileInfo) * NI + sizeof(Segment) + 8 <= 1536, "barriers and masks");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        trace_min(p.trace, 0);
        mbar_init(q_full, 1);
        mbar_init(q_empty, 9);             // the MMA warp's commit and one arrival of each softmax warp
        for (int s = 0; s < NS; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int t = 0; t < 2; ++t) { mbar_init(&s_full[t], 1); mbar_init(&p_full[t], 4); mbar_init(&o_full[t], 1); }
        *abort_flag = 0;
        fence_barrier_init();
        fence_proxy_async();
    }
    if (warp == 9) tmem_alloc(tmem_slot, TMEM_COLS);
    pdl_trigger();
    Walker w;
    PlanParams plan = p.plan;
    const bool work = plan_cta<N_THREADS>(plan, *plan_sh, w, p.ginfo, p.sinfo);
    if (blockIdx.x == 0 && threadIdx.x == 0) p.meta[0] = plan_sh->n_group_items;
    if (work && warp == 8) walk_begin(plan, *plan_sh, w);
    fence_proxy_async();                   // the plan's scratch lies where copies will land
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (!work) {
        // nothing to do: on to the end
    } else if (warp == 8) {
        // ---------------- copies ----------------
        const uint64_t keep = policy_evict_last(), once = policy_evict_first();
        int load = 0, tile = 0, n_seg = 0, issued_q = 0;
        int win_row = -1, win_base = 0, win = -1;        // page numbers of 32 boxes, one per lane
        bool ok = true;
        Segment s;
        while (ok && walk_next(plan, w, s)) {
            const int n = (s.n_chunks + 1) >> 1, n_loads = 2 * n;
            const int shift = 31 - __clz(p.box), per_chunk = CHUNK_KEYS >> shift;
            const uint64_t pol = s.prefix ? keep : once;
            auto page_of = [&](int box) {                // page of the 64-key or smaller box (every lane calls)
                if (s.seq != win_row || box < win_base || box >= win_base + 32) {
                    win_row = s.seq;
                    win_base = box;
                    const int64_t j = (((int64_t)box + lane) << shift) / p.page_size;
                    win = j < p.max_pages ? __ldg(p.page_table + (int64_t)s.seq * p.max_pages + j) : -1;
                }
                const int page = __shfl_sync(0xffffffffu, win, box - win_base);
                return page >= 0 && page < p.n_pages ? page : -1;
            };
            auto issue = [&](int l) {                    // the segment's l-th load
                // which tile, K or V
                int j = 0, v = 0;
                if (s.two) { j = l >> 1; v = l & 1; }
                else if (l == 0) { j = 0; v = 0; }
                else if (l == n_loads - 1) { j = n - 1; v = 1; }
                else { v = (l & 1) ^ 1; j = v ? l / 2 - 1 : (l + 1) / 2; }
                const int st = load % NS;
                if (!__shfl_sync(0xffffffffu, lane == 0 ? (int)mbar_wait(&empty[st], ((load / NS) & 1) ^ 1, abort_flag) : 0, 0)) return false;
                uint8_t* dst = ring + (size_t)st * Sh::STAGE;
                // the copies of this tile: boxes of the cached chunks, then the block's rows
                uint32_t bytes = 0;
                unsigned long long mask[2] = {0, 0};
                int causal_chunk = 2;
                for (int pass = 0; pass < 2; ++pass) {   // first count the bytes and work out the masks, then copy
                    if (pass == 1) {
                        if (lane == 0) {
                            if (!v) {
                                TileInfo* ti = &infos[(tile + j) % NI];
                                ti->mask[0] = mask[0];
                                ti->mask[1] = mask[1];
                                ti->causal_chunk = causal_chunk;
                                ti->full = mask[0] == ~0ull && mask[1] == ~0ull;
                            }
                            mbar_expect_tx(&full[st], bytes);
                        }
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int ch = 2 * j + c;
                        if (ch >= s.n_chunks) continue;
                        if (ch >= s.ctx_chunks) {        // the block: a box of 32 rows
                            if (pass == 0) {
                                bytes += 32 * HD * 2;
                                mask[c] = (1ull << p.plan.R) - 1;
                                if (p.causal) causal_chunk = c;
                            } else if (lane == 0) {
#pragma unroll
                                for (int h = 0; h < Sh::HALVES; ++h)
                                    tma_load_2d(dst + h * (KT * 128) + c * 8192, v ? &tmVb : &tmKb, s.kvh * HD + h * 64, s.seq * p.plan.R, &full[st], once);
                            }
                            continue;
                        }
                        const int key0 = (s.chunk + ch) * CHUNK_KEYS;
                        unsigned long long m = 0;
                        for (int x = 0; x < per_chunk; ++x) {
                            const int key = key0 + x * p.box;
                            if (key >= s.hi || key + p.box <= s.lo) continue;
                            const int page = page_of(key >> shift);
                            if (page < 0) {
                                if (pass == 0 && !v && lane == 0 && p.status) atomicOr(p.status, DFLASH_DEV_BAD_PAGE);
                                continue;
                            }
                            if (pass == 0) {
                                bytes += p.box * HD * 2;
                                m |= (p.box == 64 ? ~0ull : ((1ull << p.box) - 1)) << (x * p.box);
                            } else if (lane == 0) {
                                const int row = (int)((((int64_t)p.layer * p.n_pages + page) * 2 + v) * p.plan.Hkv + s.kvh) * p.page_size + (key & (p.page_size - 1));
#pragma unroll
                                for (int h = 0; h < Sh::HALVES; ++h)
                                    tma_load_2d(dst + h * (KT * 128) + c * 8192 + x * p.box * 128, &tmPool, h * 64, row, &full[st], pol);
                            }
                        }
                        if (pass == 0) {
                            if (s.hi - key0 < 64) m &= (1ull << (s.hi - key0)) - 1;
                            if (s.lo > key0) m &= ~0ull << (s.lo - key0);
                            mask[c] = m;
                        }
                    }
                }
                ++load;
                return true;
            };
            // the first loads do not wait for the previous segment's last product, so that the ring stays full while it ends
            const int pre = min(NS - 1, n_loads);
            int l = 0;
            for (; l < pre && ok; ++l) ok = issue(l);
            if (!ok) break;
            if (n_seg > 0 && !__shfl_sync(0xffffffffu, lane == 0 ? (int)mbar_wait(q_empty, (n_seg - 1) & 1, abort_flag) : 0, 0)) { ok = false; break; }
            if (lane == 0) {
                *seg_sh = s;
                const int q_row = s.seq * p.plan.R + s.row0 / p.plan.G;      // a tile begins with a whole (sequence, row)
                const uint32_t bytes = (uint32_t)p.plan.row_tile * HD * 2;
                mbar_expect_tx(q_full, s.two ? 2 * bytes : bytes);
                for (int t = 0; t <= s.two; ++t)
#pragma unroll
                    for (int h = 0; h < Sh::HALVES; ++h)
                        tma_load_4d(sQ + t * Sh::Q_BYTES + h * (128 * 128), &tmQ, h * 64, 0, s.kvh, q_row + t * p.rows_per_tile, q_full, keep);
                if (s.first) p.cta0[(s.prefix ? 0 : p.group_items) + s.item] = blockIdx.x;
                if (s.last) p.cta1[(s.prefix ? 0 : p.group_items) + s.item] = blockIdx.x;
            }
            __syncwarp();
            issued_q = ++n_seg;
            for (; l < n_loads && ok; ++l) ok = issue(l);
            tile += n;
        }
        if (ok && lane == 0) {             // an empty segment ends the other roles
            if (n_seg > 0 && !mbar_wait(q_empty, (n_seg - 1) & 1, abort_flag)) ok = false;
            if (ok) {
                seg_sh->n_chunks = 0;
                mbar_arrive(q_full);
            }
        }
        if (lane == 0 && !ok) {
            *abort_flag = 1;
            if (p.status) atomicOr(p.status, DFLASH_DEV_TIMEOUT);
            // copies in flight have to land before the CTA's shared memory is given up
            int dummy = 0;
            for (int k = max(0, load - NS); k < load; ++k) mbar_wait(&full[k % NS], (k / NS) & 1, &dummy, DRAIN_LIMIT);
            if (issued_q > 0) mbar_wait(q_full, (issued_q - 1) & 1, &dummy, DRAIN_LIMIT);
        }
        __syncwarp();
    } else if (warp == 9) {
        // ---------------- products ----------------
        if (lane == 0) {
            const uint32_t q_addr = smem_u32(sQ), ring_addr = smem_u32(ring);
            int base = 0, n_p[2] = {0, 0};
            bool ok = true;
            for (int k = 0;; ++k) {
                if (!mbar_wait(q_full, k & 1, abort_flag)) { ok = false; break; }
                const int two = seg_sh->two, n_chunks = seg_sh->n_chunks, n = (n_chunks + 1) >> 1;
                if (n == 0) break;
                auto wait_load = [&](int l) {
                    const int g = base + l;
                    const bool r = mbar_wait(&full[g % NS], (g / NS) & 1, abort_flag);
                    tc_fence_after();
                    return r;
                };
                auto chunks = [&](int j) { return min(2, n_chunks - 2 * j); };
                auto scores = [&](int t, int j) {        // S_t = Q K_j^T
                    const uint32_t k_addr = ring_addr + (uint32_t)((base + load_k(two, n, j)) % NS) * Sh::STAGE;
                    const uint32_t qa = q_addr + (two ? t * Sh::Q_BYTES : 0);
                    const uint32_t idesc = instr_desc_bf16(128, 64 * chunks(j));
#pragma unroll
                    for (int kk = 0; kk < HD / 16; ++kk)
                        mma_bf16(tmem + t * 128, smem_desc_sw128(qa + (kk >> 2) * (128 * 128) + (kk & 3) * 32),
                                 smem_desc_sw128(k_addr + (kk >> 2) * (KT * 128) + (kk & 3) * 32), idesc, kk > 0 ? 1u : 0u);
                    mma_commit(&s_full[t]);
                };
                auto values = [&](int t, int j, bool fresh) {   // O_t (+)= P_t V_j
                    const uint32_t v_addr = ring_addr + (uint32_t)((base + load_v(two, n, j)) % NS) * Sh::STAGE;
                    constexpr uint32_t idesc = instr_desc_bf16(128, HD) | (1u << 16);     // B is MN-major
                    const int steps = 4 * chunks(j);
                    for (int kk = 0; kk < steps; ++kk)
                        mma_bf16_ts(tmem + 256 + t * 128, tmem + t * 128 + kk * 8, smem_desc_mn(v_addr + kk * 2048, KT * 128), idesc,
                                    (!fresh || kk > 0) ? 1u : 0u);
                };
                auto release = [&](int l) { mma_commit(&empty[(base + l) % NS]); };
                auto wait_p = [&](int t) {
                    const bool r = mbar_wait(&p_full[t], n_p[t] & 1, abort_flag);
                    ++n_p[t];
                    tc_fence_after();
                    return r;
                };
                if (two) {
                    if (!(ok = wait_load(load_k(two, n, 0)))) break;
                    scores(0, 0);
                    scores(1, 0);
                    release(load_k(two, n, 0));
                    if (n == 1) mma_commit(q_empty);
                    for (int j = 0; j < n && ok; ++j) {
                        for (int t = 0; t < 2 && ok; ++t) {
                            if (t == 0 && !(ok = wait_load(load_v(two, n, j)))) break;
                            if (!(ok = wait_p(t))) break;
                            values(t, j, j == 0);
                            if (t == 1) release(load_v(two, n, j));
                            if (j + 1 == n) { mma_commit(&o_full[t]); continue; }
                            if (t == 0 && !(ok = wait_load(load_k(two, n, j + 1)))) break;
                            scores(t, j + 1);
                            if (t == 1) {
                                release(load_k(two, n, j + 1));
                                if (j + 2 == n) mma_commit(q_empty);
                            }
                        }
                    }
                } else {
                    for (int j = 0; j < min(n, 2) && ok; ++j) {
                        if (!(ok = wait_load(load_k(two, n, j)))) break;
                        scores(j, j);
                        release(load_k(two, n, j));
                    }
                    if (ok && n <= 2) mma_commit(q_empty);
                    for (int j = 0; j < n && ok; ++j) {
                        const int t = j & 1;
                        if (!(ok = wait_load(load_v(two, n, j)) && wait_p(t))) break;
                        values(t, j, j < 2);
                        release(load_v(two, n, j));
                        if (j + 2 >= n) { mma_commit(&o_full[t]); continue; }
                        if (!(ok = wait_load(load_k(two, n, j + 2)))) break;
                        scores(t, j + 2);
                        release(load_k(two, n, j + 2));
                        if (j + 3 == n) mma_commit(q_empty);
                    }
                }
                if (!ok) break;
                base += 2 * n;
            }
            if (!ok) {
                *abort_flag = 1;
                if (p.status) atomicOr(p.status, DFLASH_DEV_TIMEOUT);
            }
        }
        __syncwarp();
    } else {
        // ---------------- softmax: thread = query row ----------------
        const int t = warp >> 2, ew = warp & 3, row = ew * 32 + lane;
        const uint32_t lanes = (uint32_t)(ew * 32) << 16;
        const uint32_t tS = tmem + t * 128 + lanes, tO = tmem + 256 + t * 128 + lanes;
        int base = 0, tile0 = 0, n_s = 0, n_o = 0;
        bool ok = true;
        for (int k = 0;; ++k) {
            if (!mbar_wait(q_full, k & 1, abort_flag)) { ok = false; break; }
            const int two = seg_sh->two, n_chunks = seg_sh->n_chunks, n = (n_chunks + 1) >> 1;
            if (n == 0) break;
            const int row0 = seg_sh->row0 + (two ? t * p.plan.row_tile : 0);
            const int rows_here = min(p.plan.row_tile, seg_sh->n_rows - row0);      // rows of this tile that exist
            const bool prefix = seg_sh->prefix != 0;
            const int item = seg_sh->item, r = (row0 + row) / p.plan.G;             // r: block row, in a sequence's item
            __syncwarp();
            if (lane == 0) mbar_arrive(q_empty);
            const bool busy = ew * 32 < rows_here;       // this warp has rows
            float m_run = -CUDART_INF_F, l_run = 0.f;
            const int step = two ? 1 : 2, first = two ? 0 : t;
            for (int j = first; j < n; j += step) {
                if (!mbar_wait(&s_full[t], n_s & 1, abort_flag)) { ok = false; break; }
                ++n_s;
                tc_fence_after();
                const TileInfo* ti = &infos[(tile0 + j) % NI];
                const int groups = 2 * min(2, n_chunks - 2 * j);                    // 32-key groups of the tile
                const unsigned long long mask0 = ti->mask[0], mask1 = ti->mask[1];
                const bool all = ti->full;
                if (busy) {
                    float s[128];
                    tmem_ld32_nowait(tS, s);
                    tmem_ld32_nowait(tS + 32, s + 32);
                    if (groups == 4) {
                        tmem_ld32_nowait(tS + 64, s + 64);
                        tmem_ld32_nowait(tS + 96, s + 96);
                    }
                    tmem_ld_wait();
                    if (!all) {
                        const int cc = ti->causal_chunk;
                        const unsigned long long seen = r >= 63 ? ~0ull : (2ull << r) - 1;
                        const unsigned long long m0 = cc == 0 ? mask0 & seen : mask0, m1 = cc == 1 ? mask1 & seen : mask1;
                        const uint32_t w4[4] = {(uint32_t)m0, (uint32_t)(m0 >> 32), (uint32_t)m1, (uint32_t)(m1 >> 32)};
#pragma unroll
                        for (int g = 0; g < 4; ++g)
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                if (!(w4[g] >> c & 1)) s[g * 32 + c] = -CUDART_INF_F;
                    }
                    float mx4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                    for (int c = 0; c < 128; ++c) mx4[c & 3] = fmaxf(mx4[c & 3], s[c]);
                    const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * p.scale_log2;      // scale > 0
                    const bool raise = mx > m_run + GAP || (m_run == -CUDART_INF_F && mx > -CUDART_INF_F);
                    const float m_new = raise ? mx : m_run;
                    const float alpha = (raise && m_run > -CUDART_INF_F) ? fast_exp2(m_run - m_new) : 1.f;
                    const float m_use = m_new > -CUDART_INF_F ? m_new : 0.f;
                    m_run = m_new;
                    // every earlier product into O_t is done (S_t was issued behind it)
                    if (j > first && __any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll
                        for (int c4 = 0; c4 < HD / 32; ++c4) {
                            float o[32];
                            tmem_ld32_nowait(tO + c4 * 32, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int d = 0; d < 32; ++d) o[d] *= alpha;
                            tmem_st32(tO + c4 * 32, reinterpret_cast<const uint32_t*>(o));
                        }
                    }
                    float sum4[4] = {0.f, 0.f, 0.f, 0.f};
                    uint32_t pk[64];
#pragma unroll
                    for (int c = 0; c < 128; c += 2) {
                        const float a = fast_exp2(fmaf(s[c], p.scale_log2, -m_use)), b = fast_exp2(fmaf(s[c + 1], p.scale_log2, -m_use));
                        sum4[(c >> 1) & 3] += a + b;
                        pk[c >> 1] = pack_bf16(a, b);       // P in bf16: relative error 2^-9 a term against the 2^-9 of the operands V and K
                    }
                    tmem_st32(tS, pk);
                    tmem_st32(tS + 32, pk + 32);
                    tmem_st_wait();
                    l_run = l_run * alpha + ((sum4[0] + sum4[1]) + (sum4[2] + sum4[3]));
                }
                if (!all) {
                    // V rows that do not exist must not poison P V: 0 x whatever the page holds there
                    const int g = base + load_v(two, n, j);
                    if (!mbar_wait(&full[g % NS], (g / NS) & 1, abort_flag)) { ok = false; break; }
                    uint8_t* dV = ring + (size_t)(g % NS) * Sh::STAGE;
                    const bool here = row < 64 ? (mask0 >> row & 1) : (mask1 >> (row - 64) & 1);
                    if (!here && row < groups * 32) {
#pragma unroll
                        for (int h = 0; h < Sh::HALVES; ++h)
#pragma unroll
                            for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4*>(dV + h * (KT * 128) + row * 128 + c * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[t]);
            }
            if (!ok) break;
            // ---- the segment's partial result ----
            const bool any = n > first;
            if (any) {
                if (!mbar_wait(&o_full[t], n_o & 1, abort_flag)) { ok = false; break; }
                ++n_o;
                tc_fence_after();
            }
            if (busy) {
                const int64_t at = slot_row(p, prefix, item + (int)blockIdx.x, t, row);
                if (row < rows_here) p.ml[at] = make_float2(m_run, l_run);
                if (any) {
#pragma unroll
                    for (int c4 = 0; c4 < HD / 32; ++c4) {
                        float o[32];
                        tmem_ld32_nowait(tO + c4 * 32, o);
                        tmem_ld_wait();
                        if (row < rows_here) {
#pragma unroll
                            for (int d = 0; d < 32; d += 4)
                                *reinterpret_cast<float4*>(p.part + part_offset(at, HD, c4 * 8 + d / 4)) = make_float4(o[d], o[d + 1], o[d + 2], o[d + 3]);
                        }
                    }
                }
            }
            tc_fence_before();             // O_t is read: the next segment's first p_full lets it be overwritten
            base += 2 * n;
            tile0 += n;
        }
        if (!ok) {
            *abort_flag = 1;
            if (lane == 0 && p.status) atomicOr(p.status, DFLASH_DEV_TIMEOUT);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, TMEM_COLS);
    }
    if (threadIdx.x == 0) trace_max(p.trace, 3);
}

// ---- CUDA-core kernel: fp32, and bf16 with pages of less than 8 tokens ----------------------------------------------
// 64 packed rows against chunks of 64 keys; 256 threads, each 4 x 4 scores and 4 x hd/16 outputs.
constexpr int SIMT_THREADS = 256, SIMT_ROWS = 64;
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <int HD>
constexpr int simt_smem() { return (SIMT_ROWS * (HD + 4) * 2 + CHUNK_KEYS * HD + SIMT_ROWS * (CHUNK_KEYS + 4) + 2 * SIMT_ROWS) * 4; }

template <typename T, int HD>
__global__ void __launch_bounds__(SIMT_THREADS) prefix_attn_simt_kernel(const __grid_constant__ Params p) {
    __shared__ PlanShared plan_sh;
    extern __shared__ float sm[];
    float* sQ = sm;                                  // [64][HD + 4]
    float* sK = sQ + SIMT_ROWS * (HD + 4);           // [64][HD + 4]
    float* sV = sK + CHUNK_KEYS * (HD + 4);          // [64][HD]
    float* sP = sV + CHUNK_KEYS * HD;                // [64][68]
    float* sAlpha = sP + SIMT_ROWS * (CHUNK_KEYS + 4);
    if (threadIdx.x == 0) trace_min(p.trace, 0);
    pdl_trigger();
    Walker w;
    PlanParams plan = p.plan;
    const bool work = plan_cta<SIMT_THREADS>(plan, plan_sh, w, p.ginfo, p.sinfo);
    if (blockIdx.x == 0 && threadIdx.x == 0) p.meta[0] = plan_sh.n_group_items;
    if (!work) return;
    walk_begin(plan, plan_sh, w);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;      // scores: rows 4 ty + i, keys tx + 16 j; outputs: columns 4 tx + 64 j
    const T *Q = (const T*)p.q, *KB = (const T*)p.k_blk, *VB = (const T*)p.v_blk, *pool = (const T*)p.pool;
    const int G = p.plan.G, R = p.plan.R, Hkv = p.plan.Hkv;
    Segment s;
    while (walk_next(plan, w, s)) {
        __syncthreads();
        const int rows = min(SIMT_ROWS, s.n_rows - s.row0);
        for (int i = threadIdx.x; i < SIMT_ROWS * HD; i += SIMT_THREADS) {
            const int row = i / HD, d = i % HD, pr = s.row0 + row;
            float v = 0.f;
            if (row < rows) v = to_f(Q[(((int64_t)s.seq * R + pr / G) * p.Hq + s.kvh * G + pr % G) * HD + d]);
            sQ[row * (HD + 4) + d] = v;
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
            // a key that does not exist loads as zeros and is masked below
            unsigned long long exist = 0;
            for (int k = 0; k < CHUNK_KEYS; k += 16) {   // 16 threads a key: each row of 16 threads looks its keys up
                const int key = k + ty;
                const T *kp = nullptr, *vp = nullptr;
                if (block) {
                    if (key < R) {
                        kp = KB + (((int64_t)s.seq * R + key) * Hkv + s.kvh) * HD;
                        vp = VB + (((int64_t)s.seq * R + key) * Hkv + s.kvh) * HD;
                    }
                } else if (key0 + key >= s.lo && key0 + key < s.hi) {
                    const int pos = key0 + key, j = pos / p.page_size;
                    const int page = j < p.max_pages ? __ldg(p.page_table + (int64_t)s.seq * p.max_pages + j) : -1;
                    if (page >= 0 && page < p.n_pages) {
                        kp = pool + ((((int64_t)p.layer * p.n_pages + page) * 2 * Hkv + s.kvh) * p.page_size + pos % p.page_size) * HD;
                        vp = kp + (int64_t)Hkv * p.page_size * HD;
                    } else if (tx == 0 && p.status) {
                        atomicOr(p.status, DFLASH_DEV_BAD_PAGE);
                    }
                }
                for (int d = tx; d < HD; d += 16) {
                    sK[key * (HD + 4) + d] = kp ? to_f(kp[d]) : 0.f;
                    sV[key * HD + d] = vp ? to_f(vp[d]) : 0.f;
                }
                if (kp) exist |= 1ull << key;
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
            for (int k = 0; k < CHUNK_KEYS; ++k) {
                float pr[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) pr[i] = sP[(4 * ty + i) * (CHUNK_KEYS + 4) + k];
#pragma unroll
                for (int j = 0; j < HD / 64; ++j) {
                    const float4 v = *reinterpret_cast<const float4*>(sV + k * HD + 64 * j + 4 * tx);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        o[i][4 * j + 0] = fmaf(pr[i], v.x, o[i][4 * j + 0]);
                        o[i][4 * j + 1] = fmaf(pr[i], v.y, o[i][4 * j + 1]);
                        o[i][4 * j + 2] = fmaf(pr[i], v.z, o[i][4 * j + 2]);
                        o[i][4 * j + 3] = fmaf(pr[i], v.w, o[i][4 * j + 3]);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 4 * ty + i;
            if (row >= rows) continue;
            const int64_t at = slot_row(p, s.prefix != 0, s.item + (int)blockIdx.x, 0, row);
            if (tx == 0) p.ml[at] = make_float2(m[i], l[i]);
#pragma unroll
            for (int j = 0; j < HD / 64; ++j)
                *reinterpret_cast<float4*>(p.part + part_offset(at, HD, 16 * j + tx)) = make_float4(o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]);
        }
        if (threadIdx.x == 0) {
            if (s.first) p.cta0[(s.prefix ? 0 : p.group_items) + s.item] = blockIdx.x;
            if (s.last) p.cta1[(s.prefix ? 0 : p.group_items) + s.item] = blockIdx.x;
        }
    }
    if (threadIdx.x == 0) trace_max(p.trace, 3);
}

// ---- merge ----------------------------------------------------------------------------------------------------------
// One warp per 8 packed rows of a (sequence, kv head), four lanes a row. Parts are added in a fixed order: the prefix's key blocks, then the
// sequence's own keys, each by rising CTA.
template <typename F>
__device__ __forceinline__ void for_parts(const Params& p, const SeqInfo& si, const GroupInfo& gi, int kvh, int pr, F f) {
    const int tpi = p.plan.tiles_per_item, tr = p.plan.row_tile;
    auto item_parts = [&](bool group, int item, bool one, int tile, int row) {
        const int* c0 = p.cta0 + (group ? 0 : p.group_items) + item;
        const int* c1 = p.cta1 + (group ? 0 : p.group_items) + item;
        const int lo = __ldcg(c0), hi = __ldcg(c1);
        for (int c = lo; c <= hi; ++c) {
            if (!one) {
                f(slot_row(p, group, item + c, tile % tpi, row));
            } else {
                f(slot_row(p, group, item + c, 0, row));
                if (tpi == 2) f(slot_row(p, group, item + c, 1, row));
            }
        }
    };
    if (si.group >= 0) {
        const int gr = si.row_off + pr, tile = gr / tr, it = tile / tpi;
        for (int kb = 0; kb < gi.blocks; ++kb)
            item_parts(true, gi.item0 + (kvh * gi.blocks + kb) * gi.items + it, gi.single && it == gi.items - 1, tile, gr % tr);
    }
    const int row_tiles = (p.plan.R * p.plan.G + tr - 1) / tr, items = (row_tiles + tpi - 1) / tpi;
    const int single = row_tiles % tpi != 0 || tpi == 1, tile = pr / tr, it = tile / tpi;
    const int item0 = si.item0 - __ldcg(p.meta);
    for (int kb = 0; kb < si.blocks; ++kb) item_parts(false, item0 + (kvh * si.blocks + kb) * items + it, single && it == items - 1, tile, pr % tr);
}

template <typename T, int HD>
__global__ void __launch_bounds__(128) prefix_merge_kernel(const __grid_constant__ Params p) {
    unsigned long long* trace = p.trace ? p.trace + 4 : nullptr;
    if (threadIdx.x == 0) trace_min(trace, 0);
    const int RG = p.plan.R * p.plan.G, per_head = (RG + 7) / 8;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, quarter = lane >> 3;
    const int64_t bh = unit / per_head;
    const int pr = (int)(unit % per_head) * 8 + (lane & 7);
    pdl_wait();
    if (threadIdx.x == 0) trace_min(trace, 1);
    if (bh >= (int64_t)p.plan.S * p.plan.Hkv || pr >= RG) return;
    const int b = (int)(bh / p.plan.Hkv), kvh = (int)(bh % p.plan.Hkv);
    const SeqInfo si = p.sinfo[b];
    GroupInfo gi{};
    if (si.group >= 0) gi = p.ginfo[si.group];
    float M = -CUDART_INF_F;
    for_parts(p, si, gi, kvh, pr, [&](int64_t at) {
        const float2 ml = __ldcg(p.ml + at);
        if (ml.y != 0.f) M = fmaxf(M, ml.x);
    });
    const float M_use = M > -CUDART_INF_F ? M : 0.f;
    float L = 0.f;
    float4 acc[HD / 16];
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    for_parts(p, si, gi, kvh, pr, [&](int64_t at) {
        const float2 ml = __ldcg(p.ml + at);
        if (ml.y == 0.f) return;                  // no key in that part: its output was never written
        const float wgt = exp2f(ml.x - M_use);
        L += ml.y * wgt;
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
            const float4 o = __ldcg(reinterpret_cast<const float4*>(p.part + part_offset(at, HD, k * 4 + quarter)));
            acc[k].x += o.x * wgt;
            acc[k].y += o.y * wgt;
            acc[k].z += o.z * wgt;
            acc[k].w += o.w * wgt;
        }
    });
    const float inv = L == 0.f ? 0.f : 1.f / L;   // a row that saw no key (bad pages only) gives zeros
    const int64_t row = (int64_t)b * p.plan.R + pr / p.plan.G;
    const int head = kvh * p.plan.G + pr % p.plan.G;
    if (p.lse && quarter == 0) p.lse[row * p.Hq + head] = L == 0.f ? -CUDART_INF_F : (M_use + log2f(L)) * 0.6931471805599453f;
    T* dst = (T*)p.out + (row * p.Hq + head) * HD;
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
        const float4 v = make_float4(acc[k].x * inv, acc[k].y * inv, acc[k].z * inv, acc[k].w * inv);
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(dst + k * 16 + quarter * 4) = v;
        } else {
            *reinterpret_cast<uint2*>(dst + k * 16 + quarter * 4) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
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
    int32_t *cta0, *cta1, *meta;
    GroupInfo* ginfo;
    SeqInfo* sinfo;
    int64_t bytes;
};
PrefixWs carve_prefix(void* base, const Sizes& z, const dflash_config& c, int64_t S, int64_t n_groups) {
    Arena a(base);
    PrefixWs w{};
    const int64_t rows = z.group_slots * 256 + z.own_slots * 2 * z.own_rows;
    w.part = (float*)a.take(rows * c.head_dim * 4);
    w.ml = (float2*)a.take(rows * 8);
    w.cta0 = (int32_t*)a.take((z.group_items + z.own_items) * 4);
    w.cta1 = (int32_t*)a.take((z.group_items + z.own_items) * 4);
    w.meta = (int32_t*)a.take(4);
    w.ginfo = (GroupInfo*)a.take(std::max<int64_t>(n_groups, 1) * sizeof(GroupInfo));
    w.sinfo = (SeqInfo*)a.take(S * sizeof(SeqInfo));
    w.bytes = a.off;
    return w;
}
PlanParams plan_params(const dflash_config& c, const Sizes& z, int S, int R, int n_groups, int max_ctx_len) {
    PlanParams q{};
    q.S = S; q.R = R; q.G = c.n_q_heads / c.n_kv_heads; q.Hkv = c.n_kv_heads; q.n_groups = n_groups; q.max_ctx_len = max_ctx_len;
    q.row_tile = z.row_tile; q.tiles_per_item = z.tiles_per_item; q.chunks_per_tile = z.chunks_per_tile;
    q.cost_item = 3; q.cost_one = 4; q.cost_two = 4;
    return q;
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
    return launch_ordered(prefix_attn_tc_kernel<HD>, dim3(n_cta), dim3(N_THREADS), (size_t)Shape<HD>::SMEM, L.st, tq, tpool, tkb, tvb, p) == cudaSuccess
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
    return launch_ordered(prefix_attn_simt_kernel<T, HD>, dim3(n_cta), dim3(SIMT_THREADS), (size_t)smem, L.st, p) == cudaSuccess ? DFLASH_OK : DFLASH_ERR_CUDA;
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
    PlanParams p = plan_params(c, z, S, R, n_groups, max_ctx_len);
    p.group_start = group_start; p.prefix_len = prefix_len; p.ctx_len = ctx_len;
    const int n = n_groups + S;
    int64_t raw = 0, total = 0, all_tiles = 0;
    for (int e = 0; e < n; ++e) {
        const Entry x = plan_entry(p, e, n_groups > 0, 0, false);
        raw += x.cost;
        all_tiles += (int64_t)p.Hkv * x.items * x.n_tiles;
    }
    if (plan_cost(p, all_tiles, raw, z.n_cta) == 0) raw = all_tiles * p.cost_two;
    const int64_t share = (raw + z.n_cta - 1) / z.n_cta;
    int64_t *start = new (std::nothrow) int64_t[n + 1], *item0 = new (std::nothrow) int64_t[n + 1];
    int rc = start && item0 ? 0 : -1;
    int64_t items = 0, tiles = 0, group_items = 0, most = 0, least = INT64_MAX, segments = 0;
    for (int e = 0; rc == 0 && e <= n; ++e) {
        start[e] = total;
        item0[e] = items;
        if (e == n_groups) group_items = items;
        if (e == n) break;
        const Entry x = plan_entry(p, e, n_groups > 0, share, false);
        total += x.cost;
        items += entry_items(p, x);
        tiles += (int64_t)p.Hkv * x.items * x.n_tiles;
    }
    if (rc == 0 && (group_items > z.group_items || items - group_items > z.own_items)) rc = 1;
    int64_t seen = 0, item = -1, chunk_end = -1;      // tiles so far; the item that is under way and where it has got to
    const int n_cta = plan_ctas(p, total, z.n_cta);
    for (int cta = 0; rc == 0 && cta < n_cta; ++cta) {
        PlanShared sh{};
        Walker w{};
        w.groups_ok = n_groups > 0;
        w.share = share;
        w.lo = plan_lo(total, cta, n_cta);
        w.hi = plan_lo(total, cta + 1, n_cta);
        for (int e = 0; e < n; ++e)
            if (start[e] <= w.lo && w.lo < start[e + 1]) { sh.e = e; sh.item = (int32_t)item0[e]; sh.start = start[e]; }
        sh.n_group_items = (int32_t)group_items;
        walk_begin(p, sh, w);
        Segment s;
        int64_t cost = 0;
        while (rc == 0 && walk_next(p, w, s)) {
            const int64_t g = s.item + (s.prefix ? 0 : group_items);
            // the chain has no gap: an item begins with its first tile right behind the last tile of the one before
            if (s.first ? g != item + 1 || chunk_end != -1 : g != item || s.chunk != chunk_end) { rc = 2; break; }
            if (s.item + cta >= (s.prefix ? z.group_slots : z.own_slots)) rc = 3;
            if (s.row0 >= s.n_rows || s.n_chunks < 1 || (s.two && s.row0 + p.row_tile >= s.n_rows)) rc = 4;
            if ((s.chunk + s.ctx_chunks) * (int64_t)CHUNK_KEYS >= s.hi + CHUNK_KEYS && s.ctx_chunks > 0) rc = 5;      // no chunk behind the keys
            item = g;
            const int t = (s.n_chunks + p.chunks_per_tile - 1) / p.chunks_per_tile;
            chunk_end = s.last ? -1 : s.chunk + s.n_chunks;
            if (!s.last && s.n_chunks % p.chunks_per_tile) rc = 6;
            seen += t;
            cost += (s.first ? p.cost_item : 0) + (int64_t)t * (s.two ? p.cost_two : p.cost_one);
            ++segments;
        }
        if (rc == 0 && cost == 0) rc = 8;             // a CTA without work among those that have some
        most = std::max(most, cost);
        least = std::min(least, cost);
    }
    if (rc == 0 && (seen != tiles || item != items - 1 || chunk_end != -1)) rc = 7;
    if (info) { info[0] = items; info[1] = group_items; info[2] = tiles; info[3] = segments; info[4] = least; info[5] = most; }
    delete[] start;
    delete[] item0;
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
    p.group_slots = (int)z.group_slots; p.own_rows = z.own_rows; p.group_items = (int)z.group_items;
    p.scale_log2 = c.softmax_scale * 1.4426950408889634f;
    p.page_table = a.page_table; p.q = a.q; p.k_blk = a.k_blk; p.v_blk = a.v_blk; p.pool = a.kv_pool; p.out = a.out; p.lse = a.lse_out;
    p.part = w.part; p.ml = w.ml; p.cta0 = w.cta0; p.cta1 = w.cta1; p.ginfo = w.ginfo; p.sinfo = w.sinfo; p.meta = w.meta;
    p.status = L.status; p.trace = L.trace;
    const bool wide = c.head_dim == 128;
    int rc;
    if (use_tc(c)) rc = wide ? launch_tc<128>(L, a, p, z.n_cta) : launch_tc<64>(L, a, p, z.n_cta);
    else if (c.dtype == DFLASH_F32) rc = wide ? launch_simt<float, 128>(L, p, z.n_cta) : launch_simt<float, 64>(L, p, z.n_cta);
    else rc = wide ? launch_simt<__nv_bfloat16, 128>(L, p, z.n_cta) : launch_simt<__nv_bfloat16, 64>(L, p, z.n_cta);
    if (rc != DFLASH_OK) return rc;
    ++g_launches;
    const int64_t units = (int64_t)a.batch * p.plan.Hkv * ((a.rows * p.plan.G + 7) / 8);
    const dim3 grid((unsigned)((units + 3) / 4)), block(128);
    cudaError_t e;
    if (c.dtype == DFLASH_F32) e = wide ? launch_pdl(prefix_merge_kernel<float, 128>, grid, block, 0, L.st, p) : launch_pdl(prefix_merge_kernel<float, 64>, grid, block, 0, L.st, p);
    else e = wide ? launch_pdl(prefix_merge_kernel<__nv_bfloat16, 128>, grid, block, 0, L.st, p) : launch_pdl(prefix_merge_kernel<__nv_bfloat16, 64>, grid, block, 0, L.st, p);
    if (e != cudaSuccess) return DFLASH_ERR_CUDA;
    ++g_launches;
    return DFLASH_OK;
}

}  // namespace dflash
