// Tensor-core kernel of the shared-prefix attention (see prefix_attn.cu), and what it shares with the other kernels there.
#pragma once

#include "prefix_plan.cuh"
#include "ptx_sm100.cuh"

#include <math_constants.h>

namespace dflash {
namespace {

using namespace ptx;

// log2 units by which a tile has to top the running maximum to raise it: P and the sums may grow to 2^16 times what they would be otherwise, which
// costs no precision, and leaves fp32 2^96 for the values. The maximum is an fp32 number: rounded to bf16 it is off by 128 from scores of 2^15
// on, and the largest exponential is infinite or 0.
constexpr float GAP = 16.f;

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
    PlanOut po;
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
constexpr int N_THREADS = 640;           // warps 0-15: softmax; 16, 19: copies; 17, 18: products of one query tile each
// The block is launched with 96 registers a thread; the last four warps give up 32 of theirs: 512 * 104 + 128 * 64 = 640 * 96.
constexpr int REGS_SOFTMAX = 104, REGS_OTHER = 64;
constexpr int KT = 128;                  // keys per tile
constexpr uint32_t TMEM_COLS = 512;      // S0 | S1 | O0 | O1, 128 columns each
constexpr int NI = 12;                   // ring of tile masks: more tiles than the K and V rings can hold (checked below)

struct TileInfo {
    unsigned long long mask[2];          // keys of each chunk that exist
    int32_t causal_chunk;                // chunk (0 or 1) that holds the block in causal mode, else 2 (as for a block of one row)
    int32_t full;                        // all 128 keys exist and nothing is causal
};
// Shared memory as offsets from a 1024-byte boundary. The roles work with 32-bit addresses that each of them forms anew
// (role_base): anything they share is spilled for the sake of the softmax threads' registers, and a reload from local memory, which has next to
// no L1 beside 227 KB of shared memory, cost the MMA warp 0.3 us at every step.
template <int HD>
struct Shape {
    static constexpr int HALVES = HD / 64;                    // 64-element (128-byte) column halves of an operand
    static constexpr int Q_BYTES = 128 * HD * 2;
    static constexpr int STAGE = KT * HD * 2;
    // K and V tiles have a ring each, filled by a warp each: with one ring for both, a warp could come to a stage whose last two uses were
    // the other warp's and still open, and the wait for a phase's parity would let it pass. A K tile is used up a softmax earlier than its V tile.
    static constexpr int NK = HD == 128 ? 2 : 5, NV = HD == 128 ? 3 : 5;
    static constexpr uint32_t RING_K = 2 * Q_BYTES, RING_V = RING_K + NK * STAGE;
    // Queries are loaded a segment ahead: one query tile goes to the half of the queries' 2 tiles that the segment before does not use. (Loaded only
    // when the segment before had done its products, they held the change of item up: 148 sequences x 384 keys 90 us, then 83.)
    static constexpr uint32_t Q_FULL = RING_V + NV * STAGE;   // [2] by the segment's parity: its queries and its words in CUR are there
    static constexpr uint32_t Q_EMPTY = Q_FULL + 16;          // [2] queries used up, all earlier segments done with by every softmax warp
    // A wait for a phase's parity cannot tell a phase from the one before the last. Key tiles that are shared out between the MMA threads leave each
    // of them without news of the other's: it may wait for tile x while tile x - NV, the other's, has not landed. So the barriers of landed tiles are a longer ring:
    // tile x - NF has always landed by then. (For K: the thread's tile before x is at least x - 3, that one's stage was free once tile x - 3 - NK was
    // used. For V: with the scores of x, those of all tiles up to x - NK are there; the other thread, at most two segments behind, has used all its tiles
    // but the last of these, which is at least x - NK - 2.)
    static constexpr int NF = 8;
    static constexpr uint32_t FULL_K = Q_EMPTY + 16, FULL_V = FULL_K + 8 * NF;          // [NF] by tile
    static constexpr uint32_t EMPTY_K = FULL_V + 8 * NF, EMPTY_V = EMPTY_K + 8 * NK;   // [NK], [NV] by stage
    static constexpr uint32_t DRAIN = EMPTY_V + 8 * NV;       // [2] all products of an MMA thread that gives up
    static constexpr uint32_t TURN = DRAIN + 16;              // [2] the other MMA thread has issued its products
    static constexpr uint32_t S_FULL = TURN + 16;             // [2] S_t written (and all earlier products done)
    static constexpr uint32_t P_FULL = S_FULL + 16;           // [2] P_t written, O_t rescaled, missing V rows zeroed
    static constexpr uint32_t O_FULL = P_FULL + 16;           // [2] the segment's last product into O_t done
    static constexpr uint32_t INFO = O_FULL + 16;             // [NI] TileInfo
    static constexpr uint32_t CUR = INFO + NI * sizeof(TileInfo);       // [4] the segments whose queries are in shared memory, and the one before
    static constexpr uint32_t XCH = CUR + 4 * sizeof(Segment);          // [2][128] sums that one thread of a row hands to the other
    static constexpr uint32_t ODD_V = XCH + 1024;             // [4] by segment: its number + 1, if a block's V is not finite everywhere (CAUSAL)
    static constexpr uint32_t TMEM_SLOT = ODD_V + 16;
    static constexpr uint32_t ABORT = TMEM_SLOT + 4;
    static constexpr int SMEM = 1024 + ABORT + 4;
    static_assert(SMEM <= 227 * 1024, "shared memory of one CTA");
    static_assert(NI >= NK + NV + 2, "a tile's mask outlives its K and V stages");
    static_assert(NF >= NK + 3 && NF >= NV && (NF & (NF - 1)) == 0, "tile x - NF has landed when tile x is waited for");
};

// ---- 32-bit shared-memory addresses ----
extern __shared__ uint8_t prefix_smem[];
__device__ __forceinline__ uint32_t role_base() {
    uint32_t a;
    asm volatile("mov.u32 %0, %1;" : "=r"(a) : "r"(smem_u32(prefix_smem)));
    return (a + 1023) & ~1023u;
}
__device__ __forceinline__ int lds(uint32_t a) {
    int v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ unsigned long long lds64(uint32_t a) {
    unsigned long long v;
    asm volatile("ld.shared.b64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void sts(uint32_t a, int v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
__device__ __forceinline__ void sts64(uint32_t a, unsigned long long v) { asm volatile("st.shared.b64 [%0], %1;" ::"r"(a), "l"(v) : "memory"); }
__device__ __forceinline__ void zero16(uint32_t a) { asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(a), "r"(0) : "memory"); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity), "n"(1000000) : "memory");
    return ok != 0;
}
// Bounded wait; false if the limit ran out or another role gave up. The hint lets the hardware hold the thread for up to 1 ms a try: warps that
// poll take issue slots and memory-pipe slots from those that work. The loop stays a loop: unrolled at some thirty places it
// was most of the kernel's code, which then missed the instruction cache.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, uint32_t abort_at, long long limit = SPIN_LIMIT) {
    if (bar_try(bar, parity)) return true;
    const long long t0 = clock64();
#pragma unroll 1
    while (!bar_try(bar, parity)) {
        if ((abort_at && lds(abort_at)) || clock64() - t0 > limit) return false;
    }
    return true;
}
// lane 0 waits, the warp learns the outcome
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, uint32_t abort_at) {
    int ok = 0;
    if ((threadIdx.x & 31) == 0) ok = bar_wait(bar, parity, abort_at);
    ok = __shfl_sync(0xffffffffu, ok, 0);
    __syncwarp();
    return ok != 0;
}
// One lane of a converged warp, chosen such that the compiler knows it to be one; and a value that it shall know to be the same in all
// lanes. Products issued so (whole warp in step, operands in uniform registers) keep their rate beside sixteen busy warps, at 64 clocks
// each; issued by `lane == 0` they took 71.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xffffffff;\n\tselp.b32 %0, 1, 0, P;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar, uint64_t policy) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ void load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar, uint64_t policy) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4, %5}], [%6], %7;" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar), "l"(policy)
                 : "memory");
}

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
__device__ __forceinline__ float tmem_ld1(uint32_t taddr) {
    uint32_t v;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;" : "=r"(v) : "r"(taddr) : "memory");
    return __uint_as_float(v);
}
__device__ __forceinline__ void tmem_st1(uint32_t taddr, float v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};\n\ttcgen05.wait::st.sync.aligned;" ::"r"(taddr), "r"(__float_as_uint(v)) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
template <int N> __device__ __forceinline__ void reg_alloc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void reg_dealloc() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// the bf16 numbers of a pair that are infinite or NaN, all bits of each set
__device__ __forceinline__ uint32_t odd_bf16(uint32_t w) {
    return (((w & 0x7f807f80u) + 0x00800080u) >> 15 & 0x00010001u) * 0xffffu;      // an exponent of ones, and one more, carries into the sign's place
}
// two fp32 operations an instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Low words: K-major operand (leading offset unused); V tile as MN-major operand, [key][64 elements] halves `half_bytes` apart.
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr) { return ((addr & 0x3FFFFu) >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_lo_mn(uint32_t addr, uint32_t half_bytes) { return ((addr & 0x3FFFFu) >> 4) | ((half_bytes >> 4) << 16); }
// D (+)= A B with A in shared memory, or (bf16, M rows in the TMEM lanes, two K elements a column) in TMEM. The high words of the descriptors are the same for every tile here:
// stride 1024 bytes, version 1, 128-byte swizzle.
constexpr uint32_t DESC_HI = (1024 >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(DESC_HI)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(DESC_HI)
        : "memory");
}

// ---- copies: warp 16 K tiles, queries and tile masks; warp 19 V tiles ----
// A copy instruction costs its warp about 0.1 us and a tile of two 64-token pages takes four, hence two warps. The lanes
// look 32 boxes (64 keys, or a page if that is less) up at a time, so that a tile costs two shuffles besides its copies.
template <int HD>
__device__ __forceinline__ void copy_role(const CUtensorMap& tmQ, const CUtensorMap& tmPool, const CUtensorMap& tmKb, const CUtensorMap& tmVb, const Params& p) {
    using Sh = Shape<HD>;
    const uint32_t sb = role_base();
    const int lane = threadIdx.x & 31;
    const int vs = threadIdx.x >> 5 == 19;               // V tiles (one copy of the code for both warps: it stays in the instruction cache)
    const CUtensorMap* tmBlock = vs ? &tmVb : &tmKb;
    const uint32_t ring = sb + (vs ? Sh::RING_V : Sh::RING_K), full_at = sb + (vs ? Sh::FULL_V : Sh::FULL_K), empty_at = sb + (vs ? Sh::EMPTY_V : Sh::EMPTY_K);
    const int n_stages = vs ? Sh::NV : Sh::NK;
    int st = 0;                                          // next stage, and parity of the wait for it
    uint32_t phase = 1;
    const uint64_t keep = policy_evict_last(), once = policy_evict_first();
    const int shift = 31 - __clz(p.box), per_tile = KT >> shift, page_shift = 31 - __clz(p.page_size);
    const int2 list = __ldcg(p.po.list + blockIdx.x);
    auto fetch = [&](int k) { return k < list.y && lane < (int)sizeof(Segment) / 4 ? __ldcg(reinterpret_cast<const int*>(p.po.segs + list.x + k) + lane) : 0; };
    // physical page of box `box` of a segment (of its cached keys, boxes that hold none aside), or -1
    auto page_of = [&](int seq, int key0, int lo, int hi, int n_boxes, int box) {
        const int key = key0 + (box << shift), pg = key >> page_shift;
        return box < n_boxes && key < hi && key + p.box > lo && pg < p.max_pages ? __ldg(p.page_table + (int64_t)seq * p.max_pages + pg) : -1;
    };
#define WORD(words, field) __shfl_sync(0xffffffffu, words, offsetof(Segment, field) / 4)
    auto first_pages = [&](int words) {                  // of a segment's first 32 boxes
        return page_of(WORD(words, seq), WORD(words, chunk) * CHUNK_KEYS, WORD(words, lo), WORD(words, hi), WORD(words, ctx_chunks) * CHUNK_KEYS >> shift, lane);
    };
    // A word per lane of the next segment and of the one behind it; the next one's first pages: looked up a segment ahead
    int next = fetch(0), after = fetch(1), next_page = first_pages(next), two_before = 0;
    int issued = 0, n_seg = 0;                           // key tiles and segments so far
    bool ok = true;
#pragma unroll 1
    while (n_seg < list.y) {
        const int cur = next, first_page = next_page;
        next = after;
        after = fetch(n_seg + 2);
        next_page = first_pages(next);
#define SEG(field) WORD(cur, field)
        const int n_chunks = SEG(n_chunks), n = (n_chunks + 1) >> 1;
        const int ctx_chunks = SEG(ctx_chunks), two = SEG(two), seq = SEG(seq), kvh = SEG(kvh), key0 = SEG(chunk) * CHUNK_KEYS, key_lo = SEG(lo), key_hi = SEG(hi), row0 = SEG(row0);
        const uint64_t pol = SEG(prefix) ? keep : once;
        int win = -32, row = -1;                         // boxes win .. win + 31 of the segment: each lane's first pool row, or -1
        uint32_t there = 0, whole = 0;                   // of these: copied at all, all keys exist
        auto issue = [&](int j) {                        // this warp's copies of the segment's j-th tile
            const int box0 = j * per_tile, n_box = min(per_tile, (ctx_chunks * CHUNK_KEYS >> shift) - box0);     // boxes of cached keys
            if (n_box > 0 && box0 >= win + 32) {
                win = box0;
                const int key = key0 + ((box0 + lane) << shift), boxes = ctx_chunks * CHUNK_KEYS >> shift;
                const bool in = key < key_hi && key + p.box > key_lo && box0 + lane < boxes;
                const int page = j == 0 ? first_page : page_of(seq, key0, key_lo, key_hi, boxes, box0 + lane);
                const bool good = page >= 0 && page < p.n_pages;
                if (in && !good && !vs && p.status) atomicOr(p.status, DFLASH_DEV_BAD_PAGE);
                row = good ? (int)(((((int64_t)p.layer * p.n_pages + page) * 2 + vs) * p.plan.Hkv + kvh) * p.page_size) + (key & (p.page_size - 1)) : -1;
                there = __ballot_sync(0xffffffffu, good);
                whole = __ballot_sync(0xffffffffu, good && key >= key_lo && key + p.box <= key_hi);
            }
            const bool block = ctx_chunks < n_chunks && 2 * j + 2 >= n_chunks;      // the block's chunk is in this tile
            const int bc = ctx_chunks - 2 * j;           // and which of its two that is
            const uint32_t sel = n_box > 0 ? (uint32_t)((1ull << n_box) - 1) << (box0 - win) : 0u;
            if (!vs && lane == 0) {
                const uint32_t ti = sb + Sh::INFO + (issued % NI) * (uint32_t)sizeof(TileInfo);
                const bool full = n_box == per_tile && (whole & sel) == sel;
                if (!full) {
                    unsigned long long m0 = 0, m1 = 0;
#pragma unroll 1
                    for (int x = 0; x < n_box; ++x) {
                        if (!(there >> (box0 - win + x) & 1)) continue;
                        const int at = x << shift, key = key0 + j * KT + at;        // column of the tile, key
                        const int c0 = max(0, key_lo - key), c1 = min(p.box, key_hi - key);
                        const unsigned long long bits = (c1 >= 64 ? ~0ull : (1ull << c1) - 1) & ~((1ull << c0) - 1);
                        if (at < 64) m0 |= bits << at;
                        else m1 |= bits << (at - 64);
                    }
                    const unsigned long long rows = (1ull << p.plan.R) - 1;
                    if (block && bc == 0) m0 = rows;
                    if (block && bc == 1) m1 = rows;
                    sts64(ti, m0);
                    sts64(ti + 8, m1);
                    sts(ti + offsetof(TileInfo, causal_chunk), block && p.causal && p.plan.R > 1 ? bc : 2);
                }
                sts(ti + offsetof(TileInfo, full), full);
            }
            if (!warp_wait(empty_at + 8 * st, phase, sb + Sh::ABORT)) return false;
            const uint32_t dst = ring + st * Sh::STAGE, bar = full_at + 8 * (issued & (Sh::NF - 1));
            ++issued;
            if (lane == 0) bar_expect(bar, (uint32_t)(__popc(there & sel) * p.box + (block ? 32 : 0)) * (HD * 2));
#pragma unroll 1
            for (int x = 0; x < n_box; ++x) {
                const int y = __shfl_sync(0xffffffffu, row, box0 - win + x);
                if (lane == 0 && y >= 0) {
#pragma unroll
                    for (int h = 0; h < Sh::HALVES; ++h) load_2d(dst + h * (KT * 128) + (x << shift) * 128, &tmPool, h * 64, y, bar, pol);
                }
            }
            if (block && lane == 0) {                    // a box of 32 rows: the block, and others that the masks hide
#pragma unroll
                for (int h = 0; h < Sh::HALVES; ++h) load_2d(dst + h * (KT * 128) + bc * 8192, tmBlock, kvh * HD + h * 64, seq * p.plan.R, bar, once);
            }
            if (++st == n_stages) { st = 0; phase ^= 1; }
            return true;
        };
        // K tiles that do not need a stage the previous segment's last product still reads go ahead of the queries, if those have to wait for the
        // end of the previous segment
        int j = 0;
        if (!vs) {
            const int wait_for = two | two_before ? n_seg - 1 : n_seg - 2;       // the segment that uses the same half or halves
            two_before = two;
            if (wait_for == n_seg - 1) {
#pragma unroll 1
                for (; j < min(n, 2) && ok; ++j) ok = issue(j);
                if (!ok) break;
            }
            if (wait_for >= 0 && !warp_wait(sb + Sh::Q_EMPTY + 8 * (wait_for & 1), (wait_for >> 1) & 1, sb + Sh::ABORT)) { ok = false; break; }
            if (lane < (int)sizeof(Segment) / 4) sts(sb + Sh::CUR + (n_seg & 3) * (uint32_t)sizeof(Segment) + 4 * lane, cur);
            __syncwarp();
            if (lane == 0) {
                const int q_row = seq * p.plan.R + row0 / p.plan.G;        // a tile begins with a whole (sequence, row)
                const uint32_t bytes = (uint32_t)p.plan.row_tile * HD * 2, bar = sb + Sh::Q_FULL + 8 * (n_seg & 1), to = sb + (two ? 0 : (n_seg & 1) * Sh::Q_BYTES);
                bar_expect(bar, two ? 2 * bytes : bytes);
#pragma unroll 1
                for (int t = 0; t <= two; ++t)
#pragma unroll
                    for (int h = 0; h < Sh::HALVES; ++h)
                        load_4d(to + t * Sh::Q_BYTES + h * (128 * 128), &tmQ, h * 64, 0, kvh, q_row + t * p.rows_per_tile, bar, keep);
            }
            __syncwarp();
        }
#undef SEG
#undef WORD
        ++n_seg;
#pragma unroll 1
        for (; j < n && ok; ++j) ok = issue(j);
    }
    if (ok && !vs && lane == 0) {                        // an empty segment ends the other roles
        if (n_seg > 1 && !bar_wait(sb + Sh::Q_EMPTY + 8 * (n_seg & 1), (n_seg >> 1) - 1 & 1, sb + Sh::ABORT)) ok = false;
        if (ok) {
            sts(sb + Sh::CUR + (n_seg & 3) * (uint32_t)sizeof(Segment) + offsetof(Segment, n_chunks), 0);
            bar_arrive(sb + Sh::Q_FULL + 8 * (n_seg & 1));
        }
    }
    if (lane == 0) {
        if (!ok) {
            sts(sb + Sh::ABORT, 1);
            if (p.status) atomicOr(p.status, DFLASH_DEV_TIMEOUT);
        }
        // Copies in flight have to land before the CTA's shared memory is given up: also when all are issued, since the roles that use them may
        // give up later on. (Where none does, they land while these are at work, which this warp has nothing to do with any more.)
#pragma unroll 1
        for (int x = max(0, issued - n_stages); x < issued; ++x) bar_wait(full_at + 8 * (x & (Sh::NF - 1)), x / Sh::NF & 1, 0, DRAIN_LIMIT);      // the last copies into each stage
#pragma unroll 1
        for (int k = max(0, n_seg - (ok ? 1 : 2)); k < n_seg && !vs; ++k)      // the empty segment came by the barrier of the one before the last
            bar_wait(sb + Sh::Q_FULL + 8 * (k & 1), (k >> 1) & 1, 0, DRAIN_LIMIT);
    }
}

// ---- products: a thread for each query tile ----
// Products queue up only a few deep behind the issuing thread, and a wait on a barrier takes it 0.1 us even if there is nothing to wait for: one
// thread for both tiles left the tensor core idle between its groups of products (3370 clocks a key tile with hardly any to do). Two
// query tiles take turns, so that the products of one run while the other is at its softmax, and not both tiles' at once.
template <int HD>
__device__ __forceinline__ void mma_role(const Params& p, int t) {
    using Sh = Shape<HD>;
    const uint32_t sb = role_base(), tmem = uniform(lds(sb + Sh::TMEM_SLOT));
    const bool lead = elect_one();
    const uint32_t q_desc = desc_lo(sb), k_desc = desc_lo(sb + Sh::RING_K), v_desc = desc_lo_mn(sb + Sh::RING_V, KT * 128);
    uint32_t tile0 = 0;                                  // key tiles of the segments before
    uint32_t p_phase = 0, turn = t ^ 1;                  // parities of the next waits; thread 0 begins
    // The lanes look at the barriers one by one, so that one may give up where another finds the phase complete: they vote before any of them acts on it.
    // (Lanes that went separate ways would stand at different barriers of the warp for good.)
    bool ok = true;
#pragma unroll 1
    for (int k = 0;; ++k) {
        ok = __all_sync(0xffffffffu, bar_wait(sb + Sh::Q_FULL + 8 * (k & 1), (k >> 1) & 1, sb + Sh::ABORT));
        if (!ok) break;
        const uint32_t cur = sb + Sh::CUR + (k & 3) * (uint32_t)sizeof(Segment), q_empty = sb + Sh::Q_EMPTY + 8 * (k & 1);
        const int two = uniform(lds(cur + offsetof(Segment, two))), n_chunks = uniform(lds(cur + offsetof(Segment, n_chunks))), n = (n_chunks + 1) >> 1;
        if (n == 0) break;
        // Both threads say when they are done with a stage; with one query tile its only user does so twice.
        auto release = [&](uint32_t bar) {
            commit(bar);
            if (!two) commit(bar);
        };
        const int first = two ? 0 : t, step = two ? 1 : 2;       // this thread's key tiles; scores run one ahead of values
        const int last = two ? n : n + 1;
        if (first >= n && lead) commit(q_empty);
#pragma unroll 1
        for (int j = first; j <= last; j += step) {
            const int v = j - step;
            const bool do_v = v >= first && v < n, do_s = j < n;
            const uint32_t sv = (tile0 + v) % Sh::NV, sk = (tile0 + j) % Sh::NK;
            // the wait for P last: what comes after it adds to every tile's time
            if (do_v) ok = bar_wait(sb + Sh::FULL_V + 8 * ((tile0 + v) % Sh::NF), (tile0 + v) / Sh::NF & 1, sb + Sh::ABORT);
            if (do_s && ok) ok = bar_wait(sb + Sh::FULL_K + 8 * ((tile0 + j) % Sh::NF), (tile0 + j) / Sh::NF & 1, sb + Sh::ABORT);
            if (two && ok) {
                ok = bar_wait(sb + Sh::TURN + 8 * t, turn, sb + Sh::ABORT);
                turn ^= 1;
            }
            if (do_v && ok) {
                ok = bar_wait(sb + Sh::P_FULL + 8 * t, p_phase, sb + Sh::ABORT);
                p_phase ^= 1;
            }
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            if (lead) {
                if (do_v) {                              // O_t (+)= P_t V_v; the first product of a segment starts its accumulator
                    constexpr uint32_t idesc = instr_desc_bf16(128, HD) | (1u << 16);     // B is MN-major
                    const uint32_t vd = v_desc + sv * (Sh::STAGE >> 4), d = tmem + 256 + t * 128, a = tmem + t * 128, more = v > first;
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) mma_ts(d, a + kk * 8, vd + kk * (2048 >> 4), idesc, kk > 0 ? 1u : more);
                    if (n_chunks - 2 * v > 1) {
#pragma unroll
                        for (int kk = 4; kk < 8; ++kk) mma_ts(d, a + kk * 8, vd + kk * (2048 >> 4), idesc, 1u);
                    }
                    release(sb + Sh::EMPTY_V + 8 * sv);
                    if (v + step >= n) commit(sb + Sh::O_FULL + 8 * t);
                }
                // the other thread needs about 200 clocks to see its turn, and finds these products still running
                if (two) bar_arrive(sb + Sh::TURN + 8 * (t ^ 1));
                if (do_s) {                              // S_t = Q K_j^T; descriptors differ in their address field alone
                    const uint32_t kd = k_desc + sk * (Sh::STAGE >> 4), qd = q_desc + (two ? t : k & 1) * (Sh::Q_BYTES >> 4), d = tmem + t * 128;
                    const uint32_t idesc = instr_desc_bf16(128, 64 * min(2, n_chunks - 2 * j));
#pragma unroll
                    for (int kk = 0; kk < HD / 16; ++kk) {       // 16 elements of the row are 32 bytes; 64 elements on, the other column half begins
                        const uint32_t o = (kk >> 2) * (KT * 128 >> 4) + (kk & 3) * 2;
                        mma_ss(d, qd + o, kd + o, idesc, kk > 0);
                    }
                    commit(sb + Sh::S_FULL + 8 * t);
                    release(sb + Sh::EMPTY_K + 8 * sk);
                    if (j + step >= n) commit(q_empty);
                }
            }
            __syncwarp();
        }
        if (!ok) break;
        tile0 += n;
    }
    if (!ok) {
        sts(sb + Sh::ABORT, 1);
        if (p.status && lead) atomicOr(p.status, DFLASH_DEV_TIMEOUT);
        if (lead) commit(sb + Sh::DRAIN + 8 * t);        // TMEM is given back below: no product may still be running
        bar_wait(sb + Sh::DRAIN + 8 * t, 0, 0, DRAIN_LIMIT);
    }
}

// ---- softmax: two threads a query row, of 64 keys each ----
// Four warps a scheduler hide one another's latencies; with one thread a row (208 registers, two warps a scheduler) a tile's softmax took 2000 to 2900
// clocks against the 1024 of its products.
// P of 32 keys (16 columns), its part of the row sum, and (LOOK) the largest score. (A polynomial on the FMA pipes for a quarter of the exponentials, to
// relieve the special-function unit, made no difference to 17 rows of 32 sequences and cost 10 % for half of them.)
template <bool LOOK>
__device__ __forceinline__ void softmax_32(const float* s, float scale, float m, float2* sum, float& top, uint32_t* pk) {
    const float2 scale2 = make_float2(scale, scale), neg2 = make_float2(-m, -m);
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        if (LOOK) top = max3(top, s[2 * c], s[2 * c + 1]);
        float2 x = fma2(make_float2(s[2 * c], s[2 * c + 1]), scale2, neg2);
        x.x = fast_exp2(x.x);
        x.y = fast_exp2(x.y);
        sum[c & 1] = add2(sum[c & 1], x);
        pk[c] = pack_bf16(x.x, x.y);                     // P in bf16: as coarse as the operands V and K
    }
}
// Barriers over the 256 threads of one query tile. They are not bounded waits, so all eight warps have to come by: a bounded wait that ran out in
// one of them ends the others too at the next tile_any.
__device__ __forceinline__ void tile_bar(int t) { asm volatile("bar.sync %0, 256;" ::"r"(t + 1) : "memory"); }
__device__ __forceinline__ bool tile_any(int t, bool v) {
    uint32_t r;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %2, 0;\n\tbar.red.or.pred p, %1, 256, q;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r) : "r"(t + 1), "r"((uint32_t)v) : "memory");
    return r != 0;
}

// Numbers of a block's V that are not finite, added to a row's numerators (this thread's half of the columns) for block rows 0 .. last. Rare, and so done
// to the stored numbers: done before, in registers, it cost all calls up to 2 % (how the compiler then laid out the registers of the usual tiles).
template <int HD>
__device__ __forceinline__ void add_odd(const Params& p, float* part, int seq, int kvh, int h, int last) {
    const uint16_t* v = static_cast<const uint16_t*>(p.v_blk) + ((int64_t)seq * p.plan.R * p.plan.Hkv + kvh) * HD + h * (HD / 2);
#pragma unroll 1
    for (int key = 0; key <= last; ++key, v += p.plan.Hkv * HD) {
#pragma unroll 1
        for (int d = 0; d < HD / 2; ++d)
            if ((v[d] & 0x7f80) == 0x7f80) part[(d >> 2) * 32 + (d & 3)] += __uint_as_float((uint32_t)v[d] << 16);
    }
}
template <int HD>
__device__ __forceinline__ void softmax_role(const Params& p) {
    using Sh = Shape<HD>;
    const uint32_t sb = role_base();
    const int t = threadIdx.x >> 8, h = (threadIdx.x >> 7) & 1, ew = (threadIdx.x >> 5) & 3, row = threadIdx.x & 127, lane = threadIdx.x & 31;
    const uint32_t tS = lds(sb + Sh::TMEM_SLOT) + t * 128 + ((uint32_t)(ew * 32) << 16), tO = tS + 256 + h * (HD / 2);
    const uint32_t xch = sb + Sh::XCH + t * 512;
    uint32_t tile0 = 0;                                  // key tiles of the segments before
    uint32_t s_phase = 0, o_phase = 0;
    bool ok = true;
#pragma unroll 1
    for (int k = 0;; ++k) {
        ok = bar_wait(sb + Sh::Q_FULL + 8 * (k & 1), (k >> 1) & 1, sb + Sh::ABORT);
        if (tile_any(t, !ok)) { ok = false; break; }
        const uint32_t cur = sb + Sh::CUR + (k & 3) * (uint32_t)sizeof(Segment);     // stays until this warp, one segment on, arrives on Q_EMPTY
        const int two = lds(cur + offsetof(Segment, two)), n_chunks = lds(cur + offsetof(Segment, n_chunks)), n = (n_chunks + 1) >> 1;
        if (n == 0) break;
        __syncwarp();
        if (lane == 0) bar_arrive(sb + Sh::Q_EMPTY + 8 * (k & 1));
        auto first_row = [&] { return lds(cur + offsetof(Segment, row0)) + (two ? t * p.plan.row_tile : 0); };
        const bool mine = row < min(p.plan.row_tile, lds(cur + offsetof(Segment, n_rows)) - first_row());       // the row exists
        float m_run = -CUDART_INF_F, l_run = 0.f;        // l_run: of this thread's keys
        const int step = two ? 1 : 2, first = two ? 0 : t;
        // What a tile of V holds in places where P is 0 must not reach the rows: 0 x infinity or NaN is NaN. Threads h = 0 zero the rows that do not exist;
        // threads h = 1, in mode CAUSAL, see to the block's rows, each of which is hidden from some: numbers that are not finite (the padding of a block,
        // say) are taken out of the tile, and added at the end to the rows that see them. Four threads look at a row of V. (No time that shows: 32 whole
        // contexts of 8000 positions and 17 rows take 114 us in either mode.)
        auto mend_v = [&](int j, uint32_t ti) {
            const int chunk = lds(ti + offsetof(TileInfo, causal_chunk));
            if (h == 1 && chunk > 1) return true;
            const uint32_t x = tile0 + j, v = sb + Sh::RING_V + x % Sh::NV * Sh::STAGE;
            const bool landed = bar_wait(sb + Sh::FULL_V + 8 * (x % Sh::NF), x / Sh::NF & 1, sb + Sh::ABORT);
            if (h == 0) {
                if (!(lds64(ti + 8 * (row >> 6)) >> (row & 63) & 1)) {
#pragma unroll
                    for (int i = 0; i < Sh::HALVES; ++i)
#pragma unroll
                        for (int c = 0; c < 8; ++c) zero16(v + row * 128 + i * (KT * 128) + ((c ^ row) & 7) * 16);       // neighbouring rows in different banks (148 sequences x 128 keys: 61 us in one order, 52)
                }
            } else if ((row & 31) < p.plan.R) {
                constexpr int VECS = HD / 32;            // 16-byte vectors a thread
                const int key = row & 31;
#pragma unroll 2
                for (int c = (row >> 5) * VECS; c < ((row >> 5) + 1) * VECS; ++c) {
                    const uint32_t at = v + (chunk * 64 + key) * 128 + (c >> 3) * (KT * 128) + ((c ^ key) & 7) * 16;
                    uint4 w = lds128(at);
                    const uint4 odd = make_uint4(odd_bf16(w.x), odd_bf16(w.y), odd_bf16(w.z), odd_bf16(w.w));
                    if ((odd.x | odd.y | odd.z | odd.w) == 0) continue;
                    sts(sb + Sh::ODD_V + 4 * (k & 3), k + 1);
                    __threadfence_block();               // threads of the other query tile that find it taken out know of it
                    w = make_uint4(w.x & ~odd.x, w.y & ~odd.y, w.z & ~odd.z, w.w & ~odd.w);
                    sts128(at, w);
                }
            }
            fence_proxy_async();
            return landed;
        };
        // A warp without rows that exist has no P to work out (no row of O depends on another row's P, and these rows are not stored): it only comes by
        // the barriers and sees to its V rows. Decoding has 4 rows of 128; 32 sequences x 17 rows behind
        // 32768 positions, each with 68 rows of its own, took 279 us with all warps at work, then 273.
        const bool work = __any_sync(0xffffffffu, mine);
#pragma unroll 1
        for (int j = first; j < n && !work; j += step) {
            ok = bar_wait(sb + Sh::S_FULL + 8 * t, s_phase, sb + Sh::ABORT);
            s_phase ^= 1;
            const uint32_t ti = sb + Sh::INFO + ((tile0 + j) % NI) * (uint32_t)sizeof(TileInfo);
            const bool all = lds(ti + offsetof(TileInfo, full));
            if (!(all && j > first) || tile_any(t, !ok)) {
                if (!all) ok = mend_v(j, ti) && ok;
                if (tile_any(t, !ok)) { ok = false; break; }
            }
            __syncwarp();
            if (lane == 0) bar_arrive(sb + Sh::P_FULL + 8 * t);
        }
#pragma unroll 1
        for (int j = first; j < n && work; j += step) {
            ok = bar_wait(sb + Sh::S_FULL + 8 * t, s_phase, sb + Sh::ABORT);
            __syncwarp();                                // the lanes wait one by one, and loads and stores of TMEM are made by the whole warp in step
            s_phase ^= 1;
            tc_fence_after();
            const uint32_t ti = sb + Sh::INFO + ((tile0 + j) % NI) * (uint32_t)sizeof(TileInfo);
            const bool all = lds(ti + offsetof(TileInfo, full));
            float s[64];
            if (all && j > first) {
                // The usual case: all keys exist, and the running maximum still serves as the reference. P is worked out with it while the tile's own
                // maximum is, and nothing is exchanged but whether some row would have its maximum raised (then the tile is done over below).
                tmem_ld32_nowait(tS + h * 64, s);
                tmem_ld32_nowait(tS + h * 64 + 32, s + 32);
                tmem_ld_wait();
                float top = -CUDART_INF_F;
                float2 sum[2] = {};
                uint32_t pk[32];
                const float m_ref = m_run > -CUDART_INF_F ? m_run : 0.f;
#pragma unroll
                for (int g = 0; g < 2; ++g) softmax_32<true>(s + 32 * g, p.scale_log2, m_ref, sum, top, pk + 16 * g);
                top *= p.scale_log2;                     // scale > 0
                // The barrier also says that all of S_t is in registers: P_t takes the place of its first half. Rows that do not exist have no
                // say: they hold whatever was in shared memory, and the two ways round differently.
                const bool raise = mine && (top > m_run + GAP || (m_run == -CUDART_INF_F && top > -CUDART_INF_F));
                if (!tile_any(t, !ok || raise)) {
                    tmem_st16(tS + h * 32, pk);
                    tmem_st16(tS + h * 32 + 16, pk + 16);
                    sum[0] = add2(sum[0], sum[1]);
                    l_run += sum[0].x + sum[0].y;
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(sb + Sh::P_FULL + 8 * t);
                    continue;
                }
            }
            tmem_ld32_nowait(tS + h * 64, s);
            tmem_ld32_nowait(tS + h * 64 + 32, s + 32);
            if (!all) ok = mend_v(j, ti) && ok;
            __syncwarp();
            tmem_ld_wait();
            if (!all) {
                unsigned long long m = lds64(ti + 8 * h);
                const int r = (first_row() + row) / p.plan.G;       // block row, in a sequence's item
                if (lds(ti + offsetof(TileInfo, causal_chunk)) == h) m &= r >= 63 ? ~0ull : (2ull << r) - 1;
                const uint32_t w[2] = {(uint32_t)m, (uint32_t)(m >> 32)};
#pragma unroll
                for (int c = 0; c < 64; ++c)
                    if (!(w[c >> 5] >> (c & 31) & 1)) s[c] = -CUDART_INF_F;
            }
            float mx4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
            for (int c = 0; c < 64; c += 2) mx4[(c >> 1) & 3] = max3(mx4[(c >> 1) & 3], s[c], s[c + 1]);
            // The row's maximum. Its two threads tell each other by way of S_t itself, which both have in registers when they have come by the barrier
            // (shared memory has no room for 512 words more): columns 63 and 64, each thread's own until then. P_t takes the place of columns
            // 0 to 63; the one that holds column 63 is written by the thread that has read it.
            const float top_here = max3(fmaxf(mx4[0], mx4[1]), mx4[2], mx4[3]) * p.scale_log2;      // scale > 0
            tmem_st1(tS + 63 + h, top_here);
            tc_fence_before();
            if (tile_any(t, !ok)) { ok = false; break; }
            tc_fence_after();
            const float mx = fmaxf(top_here, tmem_ld1(tS + 64 - h));
            const bool raise = mx > m_run + GAP || (m_run == -CUDART_INF_F && mx > -CUDART_INF_F);
            const float m_new = raise ? mx : m_run;
            const float alpha = (raise && m_run > -CUDART_INF_F) ? fast_exp2(m_run - m_new) : 1.f;
            const float m_use = m_new > -CUDART_INF_F ? m_new : 0.f;
            m_run = m_new;
            // every earlier product into O_t is done (S_t was issued behind it)
            if (j > first && __any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll 1
                for (int c = 0; c < HD / 2; c += 16) {
                    float o[16];
                    tmem_ld16(tO + c, o);
#pragma unroll
                    for (int d = 0; d < 16; ++d) o[d] *= alpha;
                    tmem_st16(tO + c, reinterpret_cast<const uint32_t*>(o));
                }
            }
            float2 sum[2] = {};
            float unused = 0.f;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                uint32_t pk[16];
                softmax_32<false>(s + 32 * g, p.scale_log2, m_use, sum, unused, pk);
                tmem_st16(tS + h * 32 + g * 16, pk);
            }
            sum[0] = add2(sum[0], sum[1]);
            l_run = l_run * alpha + (sum[0].x + sum[0].y);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(sb + Sh::P_FULL + 8 * t);
        }
        if (!ok) break;
        // ---- the segment's partial result ----
        const bool any = n > first;
        if (any) {
            ok = bar_wait(sb + Sh::O_FULL + 8 * t, o_phase, sb + Sh::ABORT);
            __syncwarp();
            o_phase ^= 1;
            tc_fence_after();
        }
        const int64_t at = slot_row(p, lds(cur + offsetof(Segment, prefix)) != 0, lds(cur + offsetof(Segment, slot)), t, row);
        if (h == 1) sts(xch + 4 * row, __float_as_int(l_run));
        if (tile_any(t, !ok)) { ok = false; break; }
        if (h == 0 && mine) p.ml[at] = make_float2(m_run, l_run + __int_as_float(lds(xch + 4 * row)));
        tile_bar(t);
        if (any && __any_sync(0xffffffffu, mine)) {
#pragma unroll
            for (int c = 0; c < HD / 2; c += 32) {
                float o[32];
                __syncwarp();
                tmem_ld32_nowait(tO + c, o);
                tmem_ld_wait();
                if (mine) {
#pragma unroll
                    for (int d = 0; d < 32; d += 4)
                        *reinterpret_cast<float4*>(p.part + part_offset(at, HD, h * (HD / 8) + (c + d) / 4)) = make_float4(o[d], o[d + 1], o[d + 2], o[d + 3]);
                }
            }
            if (lds(sb + Sh::ODD_V + 4 * (k & 3)) == k + 1 && (two || (n - 1 & 1) == t) && mine)      // the block is in the last key tile
                add_odd<HD>(p, p.part + part_offset(at, HD, h * (HD / 8)), lds(cur + offsetof(Segment, seq)), lds(cur + offsetof(Segment, kvh)), h,
                            min((first_row() + row) / p.plan.G, p.plan.R - 1));
        }
        tc_fence_before();                               // O_t is read: the next segment's first P_FULL lets it be overwritten
        tile0 += n;
    }
    if (threadIdx.x == 0) trace_max(p.trace, 2);
    if (!ok) {
        sts(sb + Sh::ABORT, 1);
        if (lane == 0 && p.status) atomicOr(p.status, DFLASH_DEV_TIMEOUT);
    }
}

template <int HD>
__global__ void __launch_bounds__(N_THREADS, 1)
prefix_attn_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmPool, const __grid_constant__ CUtensorMap tmKb,
                      const __grid_constant__ CUtensorMap tmVb, const __grid_constant__ Params p) {
    using Sh = Shape<HD>;
    const uint32_t sb = role_base();
    const int warp = uniform(threadIdx.x >> 5);
    if (threadIdx.x == 0) {
        trace_min(p.trace, 0);
        for (int k = 0; k < 2; ++k) {
            bar_init(sb + Sh::Q_FULL + 8 * k, 1);
            bar_init(sb + Sh::Q_EMPTY + 8 * k, 18);      // a commit of each MMA thread and one arrival of each softmax warp
        }
#pragma unroll 1
        for (int s = 0; s < 2 * Sh::NF; ++s) bar_init(sb + Sh::FULL_K + 8 * s, 1);
#pragma unroll 1
        for (int s = 0; s < Sh::NK + Sh::NV; ++s) bar_init(sb + Sh::EMPTY_K + 8 * s, 2);
        for (int t = 0; t < 2; ++t) {
            bar_init(sb + Sh::DRAIN + 8 * t, 1);
            bar_init(sb + Sh::TURN + 8 * t, 1);
        }
        for (int t = 0; t < 2; ++t) {
            bar_init(sb + Sh::S_FULL + 8 * t, 1);
            bar_init(sb + Sh::P_FULL + 8 * t, 8);
            bar_init(sb + Sh::O_FULL + 8 * t, 1);
        }
        sts(sb + Sh::ABORT, 0);
        for (int k = 0; k < 4; ++k) sts(sb + Sh::ODD_V + 4 * k, 0);
        fence_barrier_init();
        fence_proxy_async();
    }
    if (warp == 17) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sb + Sh::TMEM_SLOT), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x >= 18 * 32 && threadIdx.x < 18 * 32 + 4) {           // the descriptors of the copies, while the plan is being made
        const CUtensorMap* m = threadIdx.x == 18 * 32 ? &tmQ : threadIdx.x == 18 * 32 + 1 ? &tmPool : threadIdx.x == 18 * 32 + 2 ? &tmKb : &tmVb;
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
    }
    pdl_trigger();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();
    if (threadIdx.x == 0) trace_min(p.trace, 1);
    if (__ldcg(&p.po.list[blockIdx.x].y) == 0) {
        // nothing to do: on to the end
    } else if (warp >= 16) {
        reg_dealloc<REGS_OTHER>();
        if (warp == 16 || warp == 19) copy_role<HD>(tmQ, tmPool, tmKb, tmVb, p);
        else mma_role<HD>(p, uniform(warp - 17));
        __syncwarp();
    } else {
        reg_alloc<REGS_SOFTMAX>();
        softmax_role<HD>(p);
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x >> 5 == 17) {
        tc_fence_after();
        tmem_dealloc(lds(role_base() + Sh::TMEM_SLOT), TMEM_COLS);
    }
    if (threadIdx.x == 0) trace_max(p.trace, 3);
}

}  // namespace
}  // namespace dflash
