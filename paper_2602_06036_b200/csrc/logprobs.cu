// Log probabilities of given tokens with the entropy and the top alternatives of a row of logits, and their gradient.
// With y = (z - M) / T, M the row's maximum and S = sum exp(y):
//   logprob(v) = y_v - ln S,   entropy = ln S - (sum y exp(y)) / S,
//   dz_v = (1/T) [ sum of g_i over the given tokens i that are v  -  p_v (G + gH (ln p_v + entropy)) ],  G = sum of all g_i, p = exp(logprob).
// Forward: one pass over the logits. Every thread keeps sums of e = exp(y) and of e y with a reference m in the place of M (see `Running`), and the largest entry
// of each of a few parts of what it has seen, from which the row's n_top largest are found afterwards (see `Candidates`). Tiles come by asynchronous
// copies into shared memory, two of them under way a CTA. Copies that go around L1 (.cg), bulk copies of 2 KB and a third tile were all slower (2048 x
// 151936 fp32 222, 199 and 225 us against 186 at the time: L1 holds what is under way, and shared memory is taken from it).
// Bound: fp32 by HBM (2048 x 151936: 187 us, 181 being the measured copy rate). bf16 (108 us) by no single unit: 95 us of bytes, 67 of exponentials (16 a clock and SM at the
// 1965 MHz of short runs), 70 of issue (8 slots an entry); a long run's power limit lowers the clock to some 1640 to 1720 MHz and all but the first with it (120 to 125 us). With alternatives the
// search adds 14 (20 of them) to 31 us (64), when its CTAs' rows end together. Rows of equal values cost it most (no bound keeps entries out, and they are cut down turn by turn):
// 2048 x 151936 bf16 172 us with 20 alternatives (122 otherwise) and 358 with 64 (138), 4096 x 32000 183 with 20 (71), 32 x 151936 18 (11).
#include "logprobs.cuh"
#include "logit_math.cuh"

#include <atomic>
#include <cmath>
#include <type_traits>

namespace dflash {
namespace {

constexpr int UNROLL = 4;
// A CTA of 256 threads, or of fewer where rows are short and many (see `launch_forward`)
template <int N>
struct Cta {
    static constexpr int THREADS = N, WARPS = N / 32, PER_SM = 1024 / N;
    static constexpr int TILE = N * UNROLL, TILE_BYTES = TILE * 16;      // 16-byte vectors of a tile: UNROLL a thread
};
constexpr int STAGES = 2;                                      // tiles under way
constexpr int MAX_CLUSTER = 8;
constexpr float LN2 = 0.6931471805599453f;
constexpr float FAR = -1.0e4f;                                 // below this many powers of two a term is 0, and its exponent only has to stay finite

// ---- a row as 16-byte vectors -----------------------------------------------------------------------------------
// Vector j holds entries j * VE - shift + (0 .. VE-1): the vectors lie on 16-byte borders whatever the row's start. The first and the last one may
// reach beyond the row; what they hold outside of it stands for -inf.
template <typename T>
struct Row {
    static constexpr int VE = 16 / (int)sizeof(T);
    const char* base;                                          // vector 0
    int vocab, shift, n_vec;
    __device__ __forceinline__ Row() {}
    __device__ __forceinline__ Row(const T* row, int v) : vocab(v) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(row);
        base = reinterpret_cast<const char*>(at & ~(uintptr_t)15);
        shift = (int)((at & 15) / sizeof(T));
        n_vec = (v + shift + VE - 1) / VE;
    }
    __device__ __forceinline__ int first(int j) const { return j * VE - shift; }
    __device__ __forceinline__ const char* address(int j) const { return base + (int64_t)j * 16; }
    __device__ __forceinline__ uint4 load(int j) const;        // with -inf outside of the row
    __device__ __forceinline__ bool whole(int j) const { return j * VE >= shift && (j + 1) * VE - shift <= vocab; }
};
template <typename T>
__device__ __forceinline__ uint4 no_entries() {
    const uint32_t w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    return make_uint4(w, w, w, w);
}
// A vector at address `at` whose entries are first, first + 1, ... of a row, with -inf outside of the row. `v`: as it lies in memory, or, where it reaches beyond
// the buffer, nothing: its entries are read one by one.
template <typename T>
__device__ __noinline__ uint4 edge_of(const char* at, int first, int vocab, uint4 v, bool in_memory) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < Row<T>::VE; ++e) {
        const int i = first + e;
        const bool in = i >= 0 && i < vocab;
        if constexpr (sizeof(T) == 4) {
            if (!in) w[e] = 0xff800000u;
            else if (!in_memory) w[e] = reinterpret_cast<const uint32_t*>(at)[e];
        } else {
            uint32_t h = (w[e / 2] >> (16 * (e & 1))) & 0xffffu;
            if (!in) h = 0xff80u;
            else if (!in_memory) h = reinterpret_cast<const uint16_t*>(at)[e];
            w[e / 2] = e & 1 ? (w[e / 2] & 0xffffu) | h << 16 : (w[e / 2] & 0xffff0000u) | h;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T>
__device__ __forceinline__ uint4 Row<T>::load(int j) const {
    if (whole(j)) return *reinterpret_cast<const uint4*>(address(j));
    return edge_of<T>(address(j), first(j), vocab, no_entries<T>(), false);
}

// largest entry of a vector; NaN has no say
__device__ __forceinline__ float vec_max(const uint4& v, float) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
}
__device__ __forceinline__ float vec_max(const uint4& v, __nv_bfloat16) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
}

// ---- copies to shared memory under way --------------------------------------------------------------------------------
template <int OFFSET = 0>
__device__ __forceinline__ void copy_async16(uint32_t smem, const void* gmem) {
    asm volatile("cp.async.ca.shared.global [%0+%2], [%1+%2], 16;" ::"r"(smem), "l"(gmem), "n"(OFFSET) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }      // all but the latest N groups have landed

// ---- statistics ----------------------------------------------------------------------------------------------------
// (z - m) c and (z - m) / T by way of half the difference, which is the same but for numbers below 2^-125: the difference of two logits may pass fp32's
// range where c or 1 / T brings it back.
__device__ __forceinline__ float difference_times(float z, float m, float c) { return 2.f * (fmaf(z, 0.5f, -0.5f * m) * c); }
__device__ __forceinline__ float difference_over(float z, float m, float t) { return 2.f * (fmaf(z, 0.5f, -0.5f * m) / t); }
// m: maximum, s: sum of 2^((z - m) c), w: sum of 2^((z - m) c) (z - m) c
struct Stat {
    float m, s, w;
};
// to a maximum `to` that is not smaller
__device__ __forceinline__ Stat raised(const Stat& a, float to, float c) {
    if (a.m == to) return a;
    const float d = a.m == -CUDART_INF_F ? FAR : fmaxf(difference_times(a.m, to, c), FAR), f = fast_exp2(d);
    return Stat{to, a.s * f, (a.w + a.s * d) * f};
}
// of a warp's lanes (of each LANES neighbouring ones): the maximum first, then one rescaling
template <int LANES>
__device__ __forceinline__ Stat lanes_merged(const Stat& a, float c) {
    float m = a.m;
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    Stat t = raised(a, m, c);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
        t.s += __shfl_xor_sync(0xffffffffu, t.s, o);
        t.w += __shfl_xor_sync(0xffffffffu, t.w, o);
    }
    return t;
}
// two fp32 operations by one instruction
__device__ __forceinline__ unsigned long long pair(float a, float b) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 halves(unsigned long long p) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
    return r;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// A thread's running sums of 2^y and 2^y y, those of even and odd entries apart, y = (z - m) c + rest: m is the largest entry of a warp's tile, and it is not
// raised before an entry's term is above 2^3, so that tiles after the first seldom do. (Where m is far below the maximum, the sum of 2^y y is all but
// taken off again in the end: terms of 2^14 cost the entropy a decimal.) A tile's terms are added up on their own first. y = z c - r by one fused operation, with r = m c rounded and rest
// = m c - r, which is exact; the size of m does not touch the terms. Entries below LOW, -inf among them, count as LOW: their terms are 0, and
// y has to be finite. Where any of that does not hold (a maximum near LOW or that large that `rest` is no small number, a temperature of an extreme size), `plain`
// terms take the differences one by one.
constexpr float LOW = -1.2676506002282294e30f;                 // -2^100
__device__ __forceinline__ uint4 not_below_low(const uint4& v, float) {
    const auto one = [](uint32_t z) {
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(z)), "f"(LOW));
        return __float_as_uint(r);
    };
    return make_uint4(one(v.x), one(v.y), one(v.z), one(v.w));
}
__device__ __forceinline__ uint4 not_below_low(const uint4& v, __nv_bfloat16) {
    const auto two = [](uint32_t z) {
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(z), "r"(0xf180f180u));
        return r;
    };
    return make_uint4(two(v.x), two(v.y), two(v.z), two(v.w));
}
struct Running {
    float m, limit, rest, neg_r;                               // limit: from which on m is raised
    bool plain;
    unsigned long long s, w;
    __device__ __forceinline__ void reset() {
        m = limit = -CUDART_INF_F;
        rest = neg_r = 0.f;
        plain = true;
        s = w = 0;
    }
    __device__ __forceinline__ void raise(float to, float c) {
        const float old = m, old_rest = rest, r = to * c;
        m = to;
        limit = to + 3.f / c;
        plain = !(fabsf(r) < 1048576.f && c < 1.0e8f && c > 1.0e-20f);
        neg_r = -r;
        rest = plain ? 0.f : fmaf(to, c, -r);
        const float d = old == -CUDART_INF_F ? FAR : fmaxf(difference_times(old, to, c), FAR) - old_rest + rest, f = fast_exp2(d);
        const float2 a = halves(s), b = halves(w);
        s = pair(a.x * f, a.y * f);
        w = pair((b.x + a.x * d) * f, (b.y + a.y * d) * f);
    }
    template <typename T>
    __device__ __forceinline__ void add(const uint4 (&raw)[UNROLL], float c) {
        constexpr int N = 16 / (int)sizeof(T);
        const unsigned long long cc = pair(c, c), rr = pair(neg_r, neg_r);
        unsigned long long ts = 0, tw = 0;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float f[N];
            unpack16(not_below_low(raw[u], T()), f, T());
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                const unsigned long long y = fma2(pair(f[e], f[e + 1]), cc, rr);
                const float2 yy = halves(y);
                const unsigned long long x = pair(fast_exp2(yy.x), fast_exp2(yy.y));
                ts = add2(ts, x);
                tw = fma2(x, y, tw);
            }
        }
        s = add2(s, ts);
        w = add2(w, tw);
    }
    template <typename T>
    __device__ __forceinline__ void add_plain(const uint4& v, float c) {
        constexpr int N = 16 / (int)sizeof(T);
        float f[N];
        unpack16(v, f, T());
        float2 a = halves(s), b = halves(w);
        const float base = m == -CUDART_INF_F ? 0.f : m;       // every term is 0 then
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float y = difference_times(f[e], base, c), x = fast_exp2(y);
            a.x += x;
            b.x = fmaf(x, fmaxf(y, FAR), b.x);
        }
        s = pair(a.x, a.y);
        w = pair(b.x, b.y);
    }
    // with `top`, the thread's largest entry, in the place of a smaller m
    __device__ __forceinline__ Stat total(float top, float c) const {
        const float2 a = halves(s), b = halves(w);
        const float f = fast_exp2(-rest), sum = a.x + a.y;
        return raised(Stat{m, sum * f, (b.x + b.y - sum * rest) * f}, fmaxf(m, top), c);
    }
};

// ---- a token that is all but certain ----------------------------------------------------------------------------------
// Beside the largest entry's term, 1, the others lose all decimals below 2^-24, and with them ln S = ln(1 + rest) and the entropy where the rest is small. Below a sum
// of 1 + 2^-5, the sums of a stretch are therefore told without that one term. Only the thread that has seen the largest entry has it in its own sums: its warp reads
// that thread's vectors once more and adds up all but it. Rows that need it pay: of only such rows 4096 x 32000 bf16 with 20 alternatives 70.7 -> 78 us, 2048 x
// 151936 107.5 -> 111, 32 x 151936 7.2 -> 7.8. (Taken out of its tile during the pass, where m is raised to it, the entry costs less there and all other rows 1 to 7 %: 4096 x 5003
// 32.3 -> 34.7.)
constexpr float CERTAIN = 1.03125f;
template <typename T, class C>
__device__ __forceinline__ void without_largest(const T* z, int vocab, int lo_j, int hi_j, float m, Stat own, float c, const Stat* of_warps, Stat* all, uint32_t has) {
    constexpr int THREADS = C::THREADS, WARPS = C::WARPS;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, owner = __ffs(has) - 1;
    const Row<T> row(z, vocab);
    Stat x = raised(own, m, c);
    if (lane == owner) x.s = x.w = 0.f;
    // (the other warps' sums are added by a lane each)
    if (lane < WARPS && lane != warp) {
        const Stat y = raised(of_warps[lane], m, c);
        x.s += y.s;
        x.w += y.w;
    }
    for (int j = lo_j + warp * 32 + owner + lane * THREADS; j < hi_j; j += 32 * THREADS) {
        float f[Row<T>::VE];
        unpack16(row.load(j), f, T());
#pragma unroll
        for (int e = 0; e < Row<T>::VE; ++e) {
            const float y = difference_times(f[e], m, c), t = f[e] == m ? 0.f : fast_exp2(y);
            x.s += t;
            x.w = fmaf(t, fmaxf(y, FAR), x.w);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
        x.w += __shfl_xor_sync(0xffffffffu, x.w, o);
    }
    if (lane == 0) *all = x;
}

// ---- candidates for the alternatives ---------------------------------------------------------------------------------
// An entry is ordered by (value, lower index first) as one 64-bit key, so that no two are equal and the result does not depend on
// the order in which threads find them. -0 counts as 0; -inf and NaN are no alternatives and have no key.
__device__ __forceinline__ uint32_t ordered(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ unsigned long long key_of(float z, int i) { return (unsigned long long)ordered(z) << 32 | (0xffffffffu - (uint32_t)i); }
__device__ __forceinline__ float value_of(unsigned long long key) { return unordered((uint32_t)(key >> 32)); }
__device__ __forceinline__ int index_of(unsigned long long key) { return (int)(0xffffffffu - (uint32_t)key); }
constexpr uint32_t ORDERED_NONE = 0x007fffffu;                 // ordered(-inf)
constexpr unsigned long long NO_KEY = (unsigned long long)ORDERED_NONE << 32 | 0xffffffffu;      // not below any key of -inf, below all others

__host__ __device__ __forceinline__ int most_of(int n_top) { return n_top + n_top / 4 + 8; }      // entries that a bound on the n_top-th largest may leave
__host__ __device__ __forceinline__ int capacity_of(int n_top, int threads) { return most_of(n_top) + threads; }      // of the list: a turn's entries fit behind one that has been cut
// what a CTA of so many threads takes: of more than half of its threads' largest entries the bound below is a weak one, and each given token has a thread
constexpr bool takes(int threads, int n_top, int n_tokens) { return 2 * n_top <= threads && n_tokens <= threads; }
// Cells of a thread: its part of a row in as many runs of tiles. Of more cells fewer vectors are read again, but a cell has a tile at least, and shared memory
// is taken from L1, which the copies under way need (see `many_cells`).
__host__ __device__ __forceinline__ int cells_of(bool many) { return many ? 16 : 8; }
static_assert(takes(256, LP_MAX_TOP, LP_MAX_TOKENS) && 32 + 32 / 4 + 8 <= 64 && 16 * 256 <= 65536, "the most that a bound leaves has a thread each; cells in 16 bits");

constexpr int BIN_BITS = 6, BINS = 1 << BIN_BITS;                   // of the range of the threads' largest entries

// The search for a stretch's n_top largest entries, after the pass over it that has left the largest entry of every thread and of each of its cells. At least
// n_top threads' largest entries bound the n_top-th largest of the stretch from below, and little else is above a bound that few of them are (`bound`).
// What is, lies in a few cells, which are read again (from L2, mostly) by all threads together. The pass itself so needs no barrier and looks at no
// entry twice; taking candidates out as they come by cost a barrier a tile and more than the reading of the row.
template <class C>
struct Candidates {
    static constexpr int THREADS = C::THREADS, WARPS = C::WARPS;
    unsigned long long* list;      // [capacity] keys
    unsigned long long* few;       // [most]
    uint16_t* cells;               // [n_cells][THREADS] largest entries as bf16, rounded up
    uint16_t* found;               // [most * n_cells] cells to be read again: cell * THREADS + thread
    int* count;                    // entries of list, of found
    uint32_t* ends;                // [2][WARPS]
    int* bins;                     // [BINS]
    int n_top, most, capacity, n_cells;
    unsigned long long floor;      // keys that are not above it are none of the n_top largest
    float floor_z;

    __device__ __forceinline__ void raise(unsigned long long to) {
        floor = to;
        // (a bound between the two zeros, which are equal as values, stands below both)
        floor_z = (uint32_t)(to >> 32) == 0x7fffffffu ? -1.4e-45f : value_of(to);
    }
    // all threads, between barriers: the list loses entries that are not among its n_top largest until at most `most` are left
    __device__ void cut() {
        const int n = *count;
        if (n <= most) return;
        const unsigned long long mine = (int)threadIdx.x < n ? list[threadIdx.x] : 0;
        const auto above = [&](unsigned long long k) {
            int a = __syncthreads_count(mine > k);
            for (int i = THREADS; i < n; i += THREADS) a += __syncthreads_count(i + (int)threadIdx.x < n && list[i + threadIdx.x] > k);
            return a;
        };
        unsigned long long lo = floor, hi = ~0ull;             // (not all entries above the floor need be in the list)
        for (int left = above(lo); left > most;) {             // more than `most` above lo, fewer than n_top above hi
            const unsigned long long mid = lo + (hi - lo) / 2;
            const int a = above(mid);
            if (a < n_top) {
                hi = mid;
            } else {
                lo = mid;
                left = a;
            }
        }
        if (threadIdx.x == 0) *count = 0;
        __syncthreads();
        if (mine > lo) few[atomicAdd(count, 1)] = mine;
        for (int i = THREADS + threadIdx.x; i < n; i += THREADS)
            if (list[i] > lo) few[atomicAdd(count, 1)] = list[i];
        __syncthreads();
        if ((int)threadIdx.x < *count) list[threadIdx.x] = few[threadIdx.x];
        raise(lo);
        __syncthreads();
    }
    __device__ __forceinline__ float cell_top(int cell) const { return __uint_as_float((uint32_t)cells[cell * THREADS + threadIdx.x] << 16); }
    // k-th vector of a cell
    __device__ __forceinline__ static int vector_of(int lo, int per_cell, int cell, int thread, int k) {
        return lo + (cell * per_cell + k) * THREADS + thread;
    }
    // all threads: a floor that at least n_top of the threads' largest entries lie above, and at most `most`. Found between bins of the values' range, then by halving
    // between values, and where too many are equal, between keys. Returns whether this thread's entries may lie above it.
    template <typename T>
    __device__ bool bound(const Row<T>& row, int lo_j, int hi_j, int per_cell, float top) {
        raise(NO_KEY);
        const bool hit = top > -CUDART_INF_F;
        const uint32_t mine = hit ? ordered(top) : 0;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const uint32_t top_of_warp = __reduce_max_sync(0xffffffffu, mine), least = __reduce_min_sync(0xffffffffu, mine);
        if (lane == 0) {
            ends[warp] = top_of_warp;
            ends[WARPS + warp] = least;
        }
        if (threadIdx.x < BINS) bins[threadIdx.x] = 0;
        int above = __syncthreads_count(hit);
        if (above <= most) return hit;
        uint32_t hi = __reduce_max_sync(0xffffffffu, ends[lane % WARPS]), lo = __reduce_min_sync(0xffffffffu, ends[WARPS + lane % WARPS]);
        lo = max(lo, ORDERED_NONE + 1) - 1;                    // more than `most` above lo, none above hi
        // counted by bins of the range, the bins' sums from the top: mostly a bin's border does
        const int shift = max(0, 32 - __clz(hi - lo - 1) - BIN_BITS);
        if (mine > lo) atomicAdd(bins + ((mine - lo - 1) >> shift), 1);
        __syncthreads();
        {
            static_assert(BINS == 64, "two bins a lane");
            const int upper = bins[BINS - 1 - 2 * lane], lower = bins[BINS - 2 - 2 * lane];
            int sum = upper + lower;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int other = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += other;
            }
            const int at = __ffs(__ballot_sync(0xffffffffu, sum >= n_top)) - 1;      // (all of them are more than n_top)
            const int to_lower = __shfl_sync(0xffffffffu, sum, at), to_upper = to_lower - __shfl_sync(0xffffffffu, lower, at);
            const bool in_upper = to_upper >= n_top;
            const uint32_t bin = BINS - 1 - 2 * at - !in_upper, from = lo + (bin << shift);
            above = in_upper ? to_upper : to_lower;
            hi = hi - from > 1u << shift ? from + (1u << shift) : hi;      // (their sum may pass 32 bits)
            lo = from;
        }
        if (above <= most) {
            raise((unsigned long long)lo << 32 | 0xffffffffu);
            return mine > lo;
        }
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            above = __syncthreads_count(mine > mid);
            if (above < n_top) { hi = mid; continue; }
            lo = mid;
            if (above <= most) {
                raise((unsigned long long)lo << 32 | 0xffffffffu);
                return mine > lo;
            }
        }
        // ties: fewer than n_top lie above the value `hi`, more than `most` at or above it. Of those at it the first place in the row decides.
        unsigned long long best = mine > hi ? ~(unsigned long long)threadIdx.x : 0;
        if (mine == hi) {
            int at = -1;
            for (int cell = 0; at < 0 && cell < n_cells; ++cell) {      // (what is rounded up may be smaller)
                if (!(cell_top(cell) >= top)) continue;
                for (int k = 0; at < 0 && k < per_cell; ++k) {
                    const int j = vector_of(lo_j, per_cell, cell, threadIdx.x, k);
                    if (j >= hi_j) break;
                    float f[Row<T>::VE];
                    unpack16(row.load(j), f, T());
#pragma unroll
                    for (int e = Row<T>::VE - 1; e >= 0; --e)
                        if (f[e] == top) at = row.first(j) + e;
                }
            }
            // (not there any more: a row that another stream writes to meanwhile. The keys have to differ all the same, or the halving would not end)
            if (at < 0) at = max(0, row.first(vector_of(lo_j, per_cell, 0, threadIdx.x, 0)));
            best = key_of(top, at);
        }
        unsigned long long l = (unsigned long long)lo << 32 | 0xffffffffu, h = (unsigned long long)hi << 32 | 0xffffffffu;
        while (true) {
            const unsigned long long mid = l + (h - l) / 2;
            above = __syncthreads_count(best > mid);
            if (above < n_top) { h = mid; continue; }
            l = mid;
            if (above <= most) break;
        }
        raise(l);
        return best > l;
    }
    // entries of the found cells' vectors [from, to) that are above the floor go to the list, as far as there is room: `count` may rise above capacity
    template <typename T>
    __device__ __forceinline__ void append(const Row<T>& row, int lo_j, int hi_j, int per_cell, int from, int to) {
        constexpr int AT_ONCE = 2;
        for (int i0 = from + (int)threadIdx.x; i0 < to; i0 += AT_ONCE * THREADS) {
            uint4 v[AT_ONCE];
            int j[AT_ONCE];
#pragma unroll
            for (int q = 0; q < AT_ONCE; ++q) {
                const int i = i0 + q * THREADS, c = i < to ? found[i / per_cell] : 0;
                j[q] = i < to ? vector_of(lo_j, per_cell, c / THREADS, c % THREADS, i % per_cell) : hi_j;
                v[q] = j[q] < hi_j ? row.load(j[q]) : no_entries<T>();
            }
#pragma unroll
            for (int q = 0; q < AT_ONCE; ++q) {
                float f[Row<T>::VE];
                unpack16(v[q], f, T());
                uint32_t hits = 0;
#pragma unroll
                for (int e = 0; e < Row<T>::VE; ++e) hits |= f[e] >= floor_z ? 1u << e : 0u;
                for (; hits; hits &= hits - 1) {
                    const int e = __ffs(hits) - 1;
                    float z = f[0];
#pragma unroll
                    for (int k = 1; k < Row<T>::VE; ++k) z = e == k ? f[k] : z;
                    const unsigned long long key = key_of(z, row.first(j[q]) + e);
                    if (key > floor) {
                        const int at = atomicAdd(count, 1);
                        if (at < capacity) list[at] = key;
                    }
                }
            }
        }
    }
    // all threads, after the pass over vectors [lo_j, hi_j): the n_top largest keys are among the at most THREADS of the list; returns how many those are. per_cell: vectors
    // of a cell, top: the thread's largest entry
    template <typename T>
    __device__ int search(const Row<T>& row, int lo_j, int hi_j, int per_cell, float top) {
        if (threadIdx.x < 2) count[threadIdx.x] = 0;
        if (bound(row, lo_j, hi_j, per_cell, top)) {           // (begins with a barrier)
            for (int c = 0; c < n_cells; ++c) {
                const float z = cell_top(c);
                if (z >= floor_z && key_of(z, max(0, row.first(vector_of(lo_j, per_cell, c, threadIdx.x, 0)))) > floor) found[atomicAdd(count + 1, 1)] = (uint16_t)(c * THREADS + threadIdx.x);
            }
        }
        __syncthreads();
        const int n = count[1] * per_cell;
        append(row, lo_j, hi_j, per_cell, 0, n);
        __syncthreads();
        if (*count > capacity) {                               // too many at once (a row whose large entries lie in few threads): in turns with room for all
            __syncthreads();
            if (threadIdx.x == 0) *count = 0;
            __syncthreads();
            constexpr int TURN = THREADS / Row<T>::VE;         // vectors
            for (int i = 0; i < n; i += TURN) {
                if (*count + THREADS > capacity) cut();
                __syncthreads();
                append(row, lo_j, hi_j, per_cell, i, min(n, i + TURN));
                __syncthreads();
            }
        }
        if (*count > THREADS) cut();
        return *count;
    }
};
// Lanes that share a key's comparisons: as many as there are threads for
template <int THREADS>
__device__ __forceinline__ int lanes_a_key(int n) { return n <= THREADS / 8 ? 8 : n <= THREADS / 4 ? 4 : n <= THREADS / 2 ? 2 : 1; }
// The place of key `mine` among n keys, largest first: by `lanes` neighbouring lanes, of which this is the part-th; all of them get it
__device__ __forceinline__ int rank_of(const unsigned long long* list, int n, unsigned long long mine, int part, int lanes) {
    int above = 0;
#pragma unroll 4
    for (int i = part; i < n; i += lanes) above += list[i] > mine;
    for (int o = lanes >> 1; o > 0; o >>= 1) above += __shfl_xor_sync(0xffffffffu, above, o);
    return above;
}
template <int THREADS>
__device__ __forceinline__ void set_cell(uint16_t* cells, int cell, float top) {
    const uint32_t b = __float_as_uint(top);                   // (towards +inf: of a negative number the rest is cut off; NaN stays NaN in a cell that then counts as none)
    cells[cell * THREADS + threadIdx.x] = (uint16_t)((b & 0x80000000u ? b : b + 0xffffu) >> 16);
}

struct ForwardParams {
    const void* logits;
    const char* end;               // behind the last row
    const int32_t* tokens;
    float *logprob, *stats, *entropy, *top_logprob;
    int32_t *top_ids, *status;
    int64_t ld;
    int32_t n_rows, vocab, n_tokens, n_top;
    float temperature, c;          // c = log2(e) / T
    bool many;                     // cells
};

// What a CTA of a cluster tells the others about its stretch of the row
struct Told {
    float m, s, w;
    int n;                         // entries of its list, and 2^16 if m is not in its sums
};

__device__ __forceinline__ void st_cluster_u64(const void* local_smem, uint32_t rank, unsigned long long v) {      // the same variable in CTA `rank`
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(ptx::mapa_shared(ptx::smem_u32(local_smem), rank)), "l"(v) : "memory");
}

// Shared memory behind the tiles under way, in 8-byte words: cells, list, few, what the CTAs of a cluster tell each other (twice 8 bytes each) and their keys, found
struct Layout {
    int cells, list, few, told, keys, found, words;
    __host__ __device__ Layout(int n_top, bool many, int cs, int threads) {
        const int most = n_top > 0 ? most_of(n_top) : 0, n_cells = n_top > 0 ? cells_of(many) : 0;
        cells = 0;
        told = cells + n_cells * threads / 4;
        list = told + (cs > 1 ? 2 * cs : 0);
        few = list + (n_top > 0 ? capacity_of(n_top, threads) : 0);
        keys = few + most;
        found = keys + (cs > 1 ? cs * n_top : 0);
        words = found + most * n_cells / 4;
    }
};

// The search as a call of its own: its registers are not the pass's
template <typename T, class C>
__device__ __noinline__ int search_stretch(const T* z, int vocab, int lo_j, int hi_j, int per_cell, float top, int n_top, bool many, int cs, unsigned long long* words,
                                           int* count, uint32_t* ends) {
    const Layout at(n_top, many, cs, C::THREADS);
    Candidates<C> cand;
    cand.list = words + at.list;
    cand.few = words + at.few;
    cand.cells = reinterpret_cast<uint16_t*>(words + at.cells);
    cand.found = reinterpret_cast<uint16_t*>(words + at.found);
    cand.count = count;
    cand.ends = ends;
    cand.bins = reinterpret_cast<int*>(ends + 2 * C::WARPS);
    cand.n_top = n_top;
    cand.most = most_of(n_top);
    cand.capacity = capacity_of(n_top, C::THREADS);
    cand.n_cells = cells_of(many);
    return cand.search(Row<T>(z, vocab), lo_j, hi_j, per_cell, top);
}

// A CTA's stretch of a row: vectors [lo, hi)
template <typename T, int CS>
struct Stretch {
    Row<T> row;
    int lo, hi;
    __device__ __forceinline__ Stretch(const ForwardParams& p, int rank, int r) : row(reinterpret_cast<const T*>(p.logits) + (int64_t)r * p.ld, p.vocab) {
        const int per = (row.n_vec + CS - 1) / CS;
        lo = min(rank * per, row.n_vec);
        hi = min(row.n_vec, lo + per);
    }
};
// Tiles [from, from + count) of a stretch, all of whose vectors are among [first, last)
template <int TILE>
struct Span {
    int from;
    uint32_t count;
    __device__ __forceinline__ Span() {}
    __device__ __forceinline__ Span(int lo, int first, int last) : from(lo < first), count((uint32_t)max(0, (last - lo) / TILE - from)) {}      // (first: 0 or 1)
    __device__ __forceinline__ bool has(int k) const { return (uint32_t)(k - from) < count; }
};

// A cluster of CS CTAs per row, a CTA per stretch of its vectors. One CTA a row: it goes on with another row, whose first tiles are then already under way;
// several: the grid has a cluster for each row.
template <typename T, int CS, class C>
__global__ void __launch_bounds__(C::THREADS, C::PER_SM) token_logprobs_kernel(const ForwardParams p) {
    constexpr int THREADS = C::THREADS, WARPS = C::WARPS, TILE = C::TILE, TILE_BYTES = C::TILE_BYTES;
    extern __shared__ uint4 ring[];                        // [STAGES][TILE]: a thread reads what it has copied itself
    __shared__ Stat sh[WARPS], rest;
    __shared__ uint32_t ends[2 * WARPS + BINS];            // and the search's bins
    __shared__ int count[2];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, rank = CS > 1 ? (int)ptx::cluster_ctarank() : 0;
    unsigned long long* words = reinterpret_cast<unsigned long long*>(ring + STAGES * TILE);
    const Layout at(p.n_top, p.many, CS, THREADS);
    Told* told = reinterpret_cast<Told*>(words + at.told);
    unsigned long long* keys = words + at.keys;
    unsigned long long* list = words + at.list;
    uint16_t* cells = reinterpret_cast<uint16_t*>(words + at.cells);
    const int n_cells = cells_of(p.many);
    ptx::pdl_trigger();
    ptx::pdl_wait();
    if constexpr (CS > 1) ptx::cluster_arrive();           // (waited for before the first store into another CTA)
    const int step = gridDim.x / CS;
    const char* begin = reinterpret_cast<const char*>(p.logits);
    const auto in_memory = [&](const char* a) { return a >= begin && a + 16 <= p.end; };
    // the next tile to be requested: the k-th of row r's stretch, whose part for this thread begins at `from`; `plain` ones lie inside of the buffer
    int ahead_r = blockIdx.x / CS, ahead_k = 0, ahead_tiles = 0;
    const char* ahead_at = nullptr;
    Span<TILE> plain;
    const auto look_ahead = [&]() {                        // at row ahead_r
        const Stretch<T, CS> n(p, rank, ahead_r);
        ahead_k = 0;
        ahead_tiles = (n.hi - n.lo + TILE - 1) / TILE;
        ahead_at = n.row.address(n.lo) + tid * 16;
        plain = Span<TILE>(n.lo, n.row.base < begin, min(n.hi, n.row.n_vec - (n.row.address(n.row.n_vec) > p.end)));
    };
    look_ahead();                                          // (the grid has no more clusters than there are rows)
    const uint32_t slots = ptx::smem_u32(ring + tid);
    uint32_t fill = slots;                                 // its place in the ring of two
    const auto request = [&]() {
        while (ahead_k == ahead_tiles && ahead_r < p.n_rows) {
            ahead_r += step;
            if (ahead_r < p.n_rows) look_ahead();
        }
        if (ahead_r < p.n_rows) {
            static_assert(UNROLL == 4 && STAGES == 2, "");
            if (plain.has(ahead_k)) {
                copy_async16<0 * THREADS * 16>(fill, ahead_at);
                copy_async16<1 * THREADS * 16>(fill, ahead_at);
                copy_async16<2 * THREADS * 16>(fill, ahead_at);
                copy_async16<3 * THREADS * 16>(fill, ahead_at);
            } else {
                const Stretch<T, CS> n(p, rank, ahead_r);
                const int j = n.lo + ahead_k * TILE + tid;
#pragma unroll
                for (int u = 0; u < UNROLL; ++u)
                    if (j + u * THREADS < n.hi && in_memory(ahead_at + u * THREADS * 16)) copy_async16(fill + u * THREADS * 16, ahead_at + u * THREADS * 16);
            }
            ++ahead_k;
            ahead_at += TILE_BYTES;
        }
        copy_commit();
        fill = 2 * slots + TILE_BYTES - fill;
    };
    for (int i = 0; i < STAGES; ++i) request();
    int use = tid;                                         // place of the next tile to be worked on
    for (int r = blockIdx.x / CS; r < p.n_rows; r += step) {
        const Stretch<T, CS> cur(p, rank, r);
        const Row<T>& row = cur.row;
        // a given token's logit (every CTA holds the row's result in the end; the first one writes it)
        const int tok = tid < p.n_tokens && rank == 0 ? p.tokens[(int64_t)r * p.n_tokens + tid] : -1;
        Running t;
        t.reset();
        float peak = -CUDART_INF_F, cell_top = -CUDART_INF_F;
        const int tiles = (cur.hi - cur.lo + TILE - 1) / TILE, tiles_a_cell = (tiles + n_cells - 1) / n_cells, per_cell = tiles_a_cell * UNROLL;
        const Span<TILE> whole(cur.lo, row.shift > 0, min(cur.hi, (p.vocab + row.shift) / Row<T>::VE));      // tiles inside of the row
        int cell = 0, in_cell = 0;
        for (int k = 0; k < tiles; ++k) {
            copy_wait<STAGES - 1>();
            uint4 raw[UNROLL];
            if (whole.has(k)) {
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) raw[u] = ring[use + u * THREADS];
            } else {
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) {
                    const int j = cur.lo + k * TILE + u * THREADS + tid;
                    raw[u] = no_entries<T>();
                    if (j < cur.hi) {
                        raw[u] = ring[use + u * THREADS];
                        if (!row.whole(j)) raw[u] = edge_of<T>(row.address(j), row.first(j), p.vocab, raw[u], in_memory(row.address(j)));
                    }
                }
            }
            float top = vec_max(raw[0], T());
#pragma unroll
            for (int u = 1; u < UNROLL; ++u) top = fmaxf(top, vec_max(raw[u], T()));
            if (__any_sync(0xffffffffu, top > t.limit)) {  // (lanes of a warp have the same m)
                const uint32_t most = __reduce_max_sync(0xffffffffu, top > -CUDART_INF_F ? ordered(top) : ORDERED_NONE);
                t.raise(unordered(most), p.c);
            }
            peak = fmaxf(peak, top);
            if (p.n_top > 0) {
                cell_top = fmaxf(cell_top, top);
                if (++in_cell == tiles_a_cell || k + 1 == tiles) {
                    set_cell<THREADS>(cells, cell++, cell_top);
                    cell_top = -CUDART_INF_F;
                    in_cell = 0;
                }
            }
            use = 2 * tid + TILE - use;
            request();                                     // into the place that has just been read
            if (!t.plain) {
                t.add<T>(raw, p.c);
            } else {
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) t.add_plain<T>(raw[u], p.c);
            }
        }
        if (p.n_top > 0)
            for (; cell < n_cells; ++cell) set_cell<THREADS>(cells, cell, -CUDART_INF_F);
        float z_tok = 0.f;
        if (tok >= p.vocab && p.status) atomicOr(p.status, DFLASH_DEV_BAD_TOKEN);
        if (tok >= 0 && tok < p.vocab) z_tok = as_f(reinterpret_cast<const T*>(p.logits)[(int64_t)r * p.ld + tok]);
        // ---- the CTA's results: warp, CTA
        const Stat seen = t.total(peak, p.c);
        Stat x = lanes_merged<32>(seen, p.c);
        if (lane == 0) sh[warp] = x;
        int n_list = 0;
        if (p.n_top > 0) n_list = search_stretch<T, C>(reinterpret_cast<const T*>(p.logits) + (int64_t)r * p.ld, p.vocab, cur.lo, cur.hi, per_cell, peak, p.n_top, p.many, CS, words, count, ends);
        else __syncthreads();
        x = lanes_merged<WARPS>(sh[lane % WARPS], p.c);
        float ones = 0.f;                                  // largest entries that are not in the sums
        if (x.s < CERTAIN && fabsf(x.m) < CUDART_INF_F) {
            const uint32_t has = __ballot_sync(0xffffffffu, peak == x.m);      // one lane of one warp, or the sum were 2
            if (has) without_largest<T, C>(reinterpret_cast<const T*>(p.logits) + (int64_t)r * p.ld, p.vocab, cur.lo, cur.hi, x.m, seen, p.c, sh, &rest, has);
            __syncthreads();
            x = rest;
            ones = 1.f;
        }
        const int lanes = lanes_a_key<THREADS>(n_list), own = tid / lanes;
        const unsigned long long key = own < n_list ? list[own] : 0;
        const int rank_in_list = p.n_top > 0 ? rank_of(list, n_list, key, tid % lanes, lanes) : 0;
        const int place = own < n_list && tid % lanes == 0 ? rank_in_list : p.n_top;
        n_list = min(n_list, p.n_top);
        if constexpr (CS > 1) {
            __syncthreads();
            if (place < p.n_top) list[place] = key;
            __syncthreads();
        }
        // ---- the cluster's
        if constexpr (CS > 1) {
            ptx::cluster_wait();                           // every CTA runs
            if (tid < CS) {
                const Told mine{x.m, x.s, x.w, n_list | (ones > 0.f ? 1 << 16 : 0)};
                const unsigned long long* w = reinterpret_cast<const unsigned long long*>(&mine);
                st_cluster_u64(told + rank, tid, w[0]);
                st_cluster_u64(reinterpret_cast<const char*>(told + rank) + 8, tid, w[1]);
            }
            for (int i = tid; i < CS * n_list; i += THREADS) st_cluster_u64(keys + rank * p.n_top + i / CS, i % CS, list[i / CS]);
            __syncwarp();
            ptx::cluster_sync_all();                       // no CTA writes into another one after this
            float m = told[0].m;
#pragma unroll
            for (int q = 1; q < CS; ++q) m = fmaxf(m, told[q].m);
            x = Stat{m, 0.f, 0.f};
            ones = 0.f;
#pragma unroll
            for (int q = 0; q < CS; ++q) {
                const float one = told[q].n >> 16 ? 1.f : 0.f;
                const Stat y = raised(Stat{told[q].m, told[q].s + (told[q].m == m ? 0.f : one), told[q].w}, m, p.c);
                x.s += y.s;
                x.w += y.w;
                ones += told[q].m == m ? one : 0.f;
            }
        }
        // (a row that holds NaN has a sum of NaN; one of -inf and NaN has no maximum, but is not empty either)
        const bool empty = x.m == -CUDART_INF_F && x.s == 0.f;
        const float sum = ones + x.s, log_sum = empty ? 0.f : ones == 1.f ? log1pf(x.s) : logf(sum);
        if (rank == 0) {
            if (tid == 0) {
                if (p.stats) *reinterpret_cast<float2*>(p.stats + 2 * (int64_t)r) = make_float2(x.m, log_sum);
                if (p.entropy) p.entropy[r] = empty ? 0.f : log_sum - x.w * LN2 / sum;
            }
            if (tid < p.n_tokens) {
                float lp = 0.f;
                if (tok >= 0 && tok < p.vocab) lp = empty ? -CUDART_INF_F : difference_over(z_tok, x.m, p.temperature) - log_sum;
                p.logprob[(int64_t)r * p.n_tokens + tid] = lp;
            }
        }
        if (p.n_top > 0) {
            int32_t* ids = p.top_ids + (int64_t)r * p.n_top;
            float* lps = p.top_logprob + (int64_t)r * p.n_top;
            int total = n_list;
            if constexpr (CS == 1) {
                if (place < p.n_top) {
                    ids[place] = index_of(key);
                    lps[place] = difference_over(value_of(key), x.m, p.temperature) - log_sum;
                }
            } else {
                // a key's place in the row: its place in the CTA's own list and the number of larger ones in each other list, one lane a list
                total = 0;
#pragma unroll
                for (int q = 0; q < CS; ++q) total += told[q].n & 0xffff;
                const int q = tid % CS;
                for (int i0 = 0; i0 < n_list; i0 += THREADS / CS) {
                    const int i = i0 + tid / CS;
                    int above = 0;
                    unsigned long long k = 0;
                    if (i < n_list) {
                        k = list[i];
                        int b = told[q].n & 0xffff, a = 0;          // keys [0, a) of list q are larger, those from b on are not
                        while (a < b) {
                            const int mid = (a + b) / 2;
                            if (keys[q * p.n_top + mid] > k) a = mid + 1;
                            else b = mid;
                        }
                        above = a;
                    }
#pragma unroll
                    for (int o = CS / 2; o > 0; o >>= 1) above += __shfl_xor_sync(0xffffffffu, above, o);
                    if (q == 0 && i < n_list && above < p.n_top) {
                        ids[above] = index_of(k);
                        lps[above] = difference_over(value_of(k), x.m, p.temperature) - log_sum;
                    }
                }
            }
            for (int i = total + tid; rank == 0 && i < p.n_top; i += THREADS) {      // fewer entries than were asked for
                ids[i] = -1;
                lps[i] = -CUDART_INF_F;
            }
        }
        __syncthreads();                                   // list and sums have been read
    }
}

// Whether a CTA keeps 16 cells a thread instead of 8: where its part of a row has more than 8 tiles, more than 32 alternatives are looked for, and a full SM's CTAs
// stay within 196 KB of shared memory, the last step that leaves L1 more than a few. 2048 x 151936 bf16 (19 tiles) with 33, 48, 64, 80 and 100 alternatives, 8 cells 124, 133, 140,
// 148 and 161 us, 16 cells 126, 132, 138, 143 and 202 (the last passes 196 KB); 544 x 151936 fp32 with 64 68 and 64; 8 tiles, 4096 x 32000 bf16 with 64 in CTAs of 128 threads, 87 and 98.
template <class C>
bool many_cells(int tiles, int n_top, int cs) {
    constexpr int STATIC = 512, PER_CTA = 1024, STEP = 196 * 1024;      // static shared memory, what the system takes of each CTA
    return tiles > 8 && n_top > 32 && C::PER_SM * (STAGES * C::TILE_BYTES + Layout(n_top, true, cs, C::THREADS).words * 8 + STATIC + PER_CTA) <= STEP;
}

// The rows by clusters of CS CTAs. Clusters are placed on as few SMs as hold them, while others idle; so a CTA takes a share of
// the SM's shared memory that leaves room for `per_sm` of them and no more (32 x 151936 bf16, four CTAs a row: 9.8 us with room for four, 6.9 for one).
template <typename T, int CS, class C>
cudaError_t launch_forward(ForwardParams p, int grid, int sm_count, cudaStream_t st) {
    constexpr int SM_SMEM = 228 * 1024, CTA_EXTRA = 2048;      // what an SM has, and what a CTA takes beside its dynamic part, rounded up
    static std::atomic<int> fits[MAX_DEVICES] = {};            // clusters that fit at one CTA per SM; 0: not asked yet. (One variable: two handles may ask at once.)
    p.many = many_cells<C>((p.vocab / Row<T>::VE + C::TILE * CS - 1) / (C::TILE * CS), p.n_top, CS);
    const int dev = current_device_slot(), words = Layout(p.n_top, p.many, CS, C::THREADS).words * 8;
    if (dev < 0) return cudaErrorInvalidDevice;
    const auto kernel = token_logprobs_kernel<T, CS, C>;
    int alone = fits[dev].load(std::memory_order_acquire);
    if (alone == 0) {
        const int most = SM_SMEM - 1024 - CTA_EXTRA;
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e != cudaSuccess) return e;
        alone = sm_count;
        if (CS > 1) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(CS);
            cfg.blockDim = dim3(C::THREADS);
            cfg.dynamicSmemBytes = most;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = CS;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            if (cudaOccupancyMaxActiveClusters(&alone, kernel, &cfg) != cudaSuccess || alone < 1) alone = std::max(1, sm_count / CS);
        }
        fits[dev].store(alone, std::memory_order_release);
    }
    const int per_sm = std::max(1, std::min(C::PER_SM, (p.n_rows + alone - 1) / alone));
    const size_t smem = std::max<size_t>((size_t)STAGES * C::TILE_BYTES + words, per_sm < C::PER_SM ? SM_SMEM / (per_sm + 1) : 0);
    if (CS == 1) return launch_pdl(kernel, dim3(grid), dim3(C::THREADS), smem, st, p);
    return launch_pdl_cluster(kernel, dim3(grid), dim3(C::THREADS), smem, st, CS, p);
}

// How a call is cut up: threads of a CTA, CTAs of a row, CTAs
struct Form {
    int threads, cs, grid;
};
Form forward_form(int es, int n_rows, int vocab, int n_tokens, int n_top, int sm_count) {
    using Wide = Cta<256>;
    // Short rows that are many: smaller CTAs, and so more rows under way an SM. What a row costs beside its tiles (barriers, sums, the search) then overlaps with other rows'
    // work, and less of its last tile is empty. Worth it once there are rows for all CTAs of the next larger size: bf16, 20 alternatives, 64 x 1024 with 256, 128 and
    // 64 threads 5.6, 5.5 and 5.9 us, 1200 x 1024 17.4, 11.5 and 8.0. In long rows the bound from fewer threads leaves larger cells to be read again, of fp32
    // sooner, whose pass HBM holds already: bf16 4096 x 50257 120 and 97 us with 256 and 128, 2048 x 151936 128 and 133 (64 alternatives: 65536 80 and 85,
    // 32000 105 and 98); fp32 4096 x 14000 70 and 57, 32000 101 and 103; with 128 and 64 bf16 4096 x 5003 40 and 29, 16384 44 and 42, fp32 16384 62 and 67.
    const int64_t row = (int64_t)vocab * es, few = (int64_t)(n_top <= 32 ? 112 : 64) << (es == 4 ? 9 : 10);
    const auto alone = [&](int threads, int per_sm) { return Form{threads, 1, std::min(n_rows, per_sm * sm_count)}; };
    if (row <= 32 << 10 && n_rows >= Cta<128>::PER_SM * sm_count && takes(64, n_top, n_tokens)) return alone(64, Cta<64>::PER_SM);
    if (row <= few && n_rows >= Wide::PER_SM * sm_count && takes(128, n_top, n_tokens)) return alone(128, Cta<128>::PER_SM);
    // CTAs per row: what takes the least time by a count of tile times. CTAs that share an SM share its rate, so that what counts is how evenly a turn of
    // CTAs fills the SMs; beside its tiles a turn takes the time of 4 tiles (9 with the search), and a cluster's meeting that of 2 to 4. (A tile time is
    // 0.46 us. 32 x 151936 bf16 by 1, 2, 4 and 8 CTAs a row: 14, 10, 7 and 8 us; 300 rows 26, 25, 27 and 38, with 20 alternatives 31, 32, 37 and 57; 800 rows
    // 57, 49, 61 and 91. The rule is up to a tenth off the best of the four.)
    const int tile = Wide::TILE_BYTES / es, tiles = (vocab + tile - 1) / tile;
    const int64_t slots = (int64_t)Wide::PER_SM * sm_count;
    int cs = 1;
    int64_t least = INT64_MAX;
    for (int s = 1; s <= MAX_CLUSTER && s / 2 < tiles; s *= 2) {
        const int64_t n = (int64_t)n_rows * s, full = n / slots, last = (n % slots + sm_count - 1) / sm_count, each = (tiles + s - 1) / s;
        const int64_t time = (full * Wide::PER_SM + last) * each + (full + (last > 0)) * (n_top > 0 ? 9 : 4) + (s == 1 ? 0 : s == 8 ? 4 : 2);
        if (time < least) {
            least = time;
            cs = s;
        }
    }
    return cs == 1 ? alone(256, Wide::PER_SM) : Form{256, cs, n_rows * cs};
}

template <typename T>
cudaError_t launch_forward(const ForwardParams& p, int sm_count, cudaStream_t st) {
    const Form f = forward_form((int)sizeof(T), p.n_rows, p.vocab, p.n_tokens, p.n_top, sm_count);
    switch (f.threads * f.cs) {
        case 64: return launch_forward<T, 1, Cta<64>>(p, f.grid, sm_count, st);
        case 128: return launch_forward<T, 1, Cta<128>>(p, f.grid, sm_count, st);
        case 256: return launch_forward<T, 1, Cta<256>>(p, f.grid, sm_count, st);
        case 512: return launch_forward<T, 2, Cta<256>>(p, f.grid, sm_count, st);
        case 1024: return launch_forward<T, 4, Cta<256>>(p, f.grid, sm_count, st);
        default: return launch_forward<T, 8, Cta<256>>(p, f.grid, sm_count, st);
    }
}

// ---- gradient ----------------------------------------------------------------------------------------------------------
constexpr int GROUP = 8;                                       // groups of 8 entries a thread
constexpr float GONE = -150.f;                                 // p = 2^y is 0 below, and its factor, which grows with -y, has to stay finite

struct BackwardParams {
    const void* logits;
    const int32_t* tokens;
    const float *stats, *entropy, *d_logprob, *d_entropy;
    void* dlogits;
    int32_t* status;
    int64_t ld, d_ld;
    int32_t vocab, n_tokens, pieces, per_piece;                // entries of a piece: a multiple of GROUP
    float part, c;                 // (z - M) log2(e) / T = (part z - part M) c: halves, whose difference stays in range, where T > 1; the whole elsewhere
    float scale, inv_t;            // gradients are added up times `scale`, a power of two; inv_t = 1 / (T scale)
};

// A group's 16-byte vectors from the border in front of it on: `off` entries lie between the two (OFF: which is not 0, and takes one vector more)
template <typename T, bool OFF>
struct Raw {
    static constexpr int VE = Row<T>::VE, VECS = GROUP / VE + OFF, WORDS = 4 * VECS;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const T* src, int off) {
        const uint4* v = reinterpret_cast<const uint4*>(src - off);
#pragma unroll
        for (int k = 0; k < VECS; ++k) {
            const uint4 x = OFF ? v[k] : __ldcs(v + k);          // (a vector that two groups share comes from L1 the second time)
            w[4 * k] = x.x; w[4 * k + 1] = x.y; w[4 * k + 2] = x.z; w[4 * k + 3] = x.w;
        }
    }
    __device__ __forceinline__ void entries(int off, float (&z)[GROUP]) {
        if constexpr (OFF) {                                   // the same for all groups of a row
            const int words = off * (int)sizeof(T) / 4;
#pragma unroll
            for (int bit = 2; bit > 0; bit >>= 1)
                if (words & bit) {
#pragma unroll
                    for (int k = 0; k < WORDS; ++k) w[k] = k + bit < WORDS ? w[k + bit] : 0;
                }
            if (sizeof(T) == 2 && (off & 1)) {
#pragma unroll
                for (int k = 0; k + 1 < WORDS; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], 16);
            }
        }
#pragma unroll
        for (int k = 0; k < GROUP / VE; ++k) {
            float f[VE];
            unpack16(make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]), f, T());
#pragma unroll
            for (int e = 0; e < VE; ++e) z[k * VE + e] = f[e];
        }
    }
};
__device__ __forceinline__ void store_group(float* dst, const float (&g)[GROUP]) {
    __stcs(reinterpret_cast<float4*>(dst), make_float4(g[0], g[1], g[2], g[3]));
    __stcs(reinterpret_cast<float4*>(dst) + 1, make_float4(g[4], g[5], g[6], g[7]));
}
__device__ __forceinline__ void store_group(__nv_bfloat16* dst, const float (&g)[GROUP]) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(g[2 * e], g[2 * e + 1]);
        w[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    __stcs(reinterpret_cast<uint4*>(dst), make_uint4(w[0], w[1], w[2], w[3]));
}
__device__ __forceinline__ void store_entry(float* dst, float g) { *dst = g; }
__device__ __forceinline__ void store_entry(__nv_bfloat16* dst, float g) { *dst = __float2bfloat16_rn(g); }

// CTA (row, piece of the row)
template <typename T, typename O, int B_THREADS>
__global__ void __launch_bounds__(B_THREADS) token_logprobs_bwd_kernel(const BackwardParams p) {
    constexpr int MOST = B_THREADS < LP_MAX_TOKENS ? B_THREADS : LP_MAX_TOKENS;      // given tokens: a thread each
    __shared__ int4 s_tok[MOST / 4];                           // -1 for none
    __shared__ float4 s_g[MOST / 4];
    __shared__ float s_sum[B_THREADS / 32];
    ptx::pdl_trigger();
    ptx::pdl_wait();
    const int tid = threadIdx.x;
    const int r = blockIdx.x / p.pieces, piece = blockIdx.x % p.pieces;
    const int lo = piece * p.per_piece, hi = min(p.vocab, lo + p.per_piece);
    const T* z = reinterpret_cast<const T*>(p.logits) + (int64_t)r * p.ld;
    O* dz = reinterpret_cast<O*>(p.dlogits) + (int64_t)r * p.d_ld;
    // ---- the row's numbers, all of them requested before any is waited for
    int tok = -1;
    float g = 0.f, z_tok = 0.f;
    const float top = p.stats[2 * (int64_t)r], log_sum = p.stats[2 * (int64_t)r + 1];
    const float gh_in = p.d_entropy ? p.d_entropy[r] : 0.f, h = p.d_entropy ? p.entropy[r] : 0.f;
    if (tid < p.n_tokens) {
        tok = p.tokens[(int64_t)r * p.n_tokens + tid];
        g = p.d_logprob[(int64_t)r * p.n_tokens + tid];
        if (tok >= lo && tok < hi) z_tok = as_f(z[tok]);       // before any store: dlogits may be the logits
        if (tok >= p.vocab) {
            if (p.status && piece == 0) atomicOr(p.status, DFLASH_DEV_BAD_TOKEN);
            tok = -1;
        }
        if (tok < 0) g = 0.f;
    }
    const bool some = g != 0.f;
    g *= p.scale;
    if (tid < MOST) {
        reinterpret_cast<int*>(s_tok)[tid] = tok;
        reinterpret_cast<float*>(s_g)[tid] = g;
    }
    float sum = g;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((tid & 31) == 0) s_sum[tid >> 5] = sum;
    const int any = __syncthreads_or(some);
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < MOST / 32; ++w) sum += s_sum[w];
    const bool off_row = (!any && gh_in == 0.f) || (top == -CUDART_INF_F && log_sum == 0.f);      // nothing comes in, or a row of -inf
    // with y = log2 p = (z - top) c - log_sum / ln 2:  dz = p (a + b y)
    const float part = p.part, part_top = top * part, gh = gh_in * p.scale, sub = log_sum * LOG2E, a = -(sum + gh * h) * p.inv_t, b = -gh * LN2 * p.inv_t;
    auto grad = [&](float v) {
        const float y = fmaf(fmaf(v, part, -part_top), p.c, -sub);
        return fast_exp2(y) * fmaf(b, fmaxf(y, GONE), a);
    };
    // ---- the piece: groups whose stores lie on 16-byte borders; their loads begin `off` entries behind one, and their vectors have to lie inside of the row
    constexpr int AZ = 16 / (int)sizeof(T), AO = 16 / (int)sizeof(O);
    int begin = lo + (AO - (int)((reinterpret_cast<uintptr_t>(dz + lo) & 15) / sizeof(O))) % AO;
    const int off = (int)((reinterpret_cast<uintptr_t>(z + begin) & 15) / sizeof(T));
    while (begin < off) begin += AO > AZ ? AO : AZ;            // (a step that leaves `off` as it is)
    const int last = off ? min(hi, p.vocab - (AZ - off)) : hi, n_group = max(0, (last - begin) / GROUP);
    const auto groups = [&](auto shifted) {
        constexpr bool OFF = decltype(shifted)::value;
        constexpr int U = OFF && sizeof(T) == 4 ? 2 : 4;       // groups of a thread under way
        for (int i0 = 0; i0 < n_group; i0 += U * B_THREADS) {
            Raw<T, OFF> raw[U];
            if (!off_row) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * B_THREADS + tid;
                    if (i < n_group) raw[u].load(z + begin + i * GROUP, off);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * B_THREADS + tid;
                if (i < n_group) {
                    float v[GROUP], d[GROUP];
                    if (!off_row) raw[u].entries(off, v);
#pragma unroll
                    for (int e = 0; e < GROUP; ++e) d[e] = off_row ? 0.f : grad(v[e]);
                    store_group(dz + begin + i * GROUP, d);
                }
            }
        }
    };
    if (off) groups(std::true_type());
    else groups(std::false_type());
    const int rest = begin + n_group * GROUP;                  // entries in front of and behind the groups: all of them where there are none
    for (int i = lo + tid; i < min(begin, hi); i += B_THREADS) store_entry(dz + i, off_row ? 0.f : grad(as_f(z[i])));
    for (int i = rest + tid; i < hi; i += B_THREADS) store_entry(dz + i, off_row ? 0.f : grad(as_f(z[i])));
    // ---- the given tokens' own entries: the first of equal ones adds their gradients up, in the order of the list
    __syncthreads();
    if (!off_row && tok >= lo && tok < hi) {
        float own = 0.f;
        bool earlier = false;
        for (int i = 0; i < p.n_tokens; i += 4) {
            const int4 t = s_tok[i / 4];
            const float4 d = s_g[i / 4];
            own += t.x == tok ? d.x : 0.f;
            own += t.y == tok ? d.y : 0.f;
            own += t.z == tok ? d.z : 0.f;
            own += t.w == tok ? d.w : 0.f;
            earlier |= (t.x == tok && i < tid) || (t.y == tok && i + 1 < tid) || (t.z == tok && i + 2 < tid) || (t.w == tok && i + 3 < tid);
        }
        if (!earlier) store_entry(dz + tok, fmaf(own, p.inv_t, grad(z_tok)));
    }
}

template <typename T, typename O, int B_THREADS>
cudaError_t launch_backward(BackwardParams p, int rows, int sm_count, cudaStream_t st) {
    // pieces of a row: whole tiles, few enough that a CTA's start is little beside its work, enough to fill the GPU
    constexpr int TILE = B_THREADS * 4 * GROUP;
    const int tiles = (p.vocab + TILE - 1) / TILE;
    int per = std::min(tiles, 4);
    while (per > 1 && (int64_t)rows * ((tiles + per - 1) / per) < 8ll * sm_count) --per;
    p.per_piece = per * TILE;
    p.pieces = (p.vocab + p.per_piece - 1) / p.per_piece;
    return launch_pdl(token_logprobs_bwd_kernel<T, O, B_THREADS>, dim3((unsigned)((int64_t)rows * p.pieces)), dim3(B_THREADS), 0, st, p);
}

template <typename T, typename O>
cudaError_t launch_backward(const BackwardParams& p, int rows, int sm_count, cudaStream_t st) {
    // With many rows smaller CTAs overlap what a row costs before its first load and after its last store with other rows' work (64 given tokens, 4096 x 1024 bf16
    // with 256, 128 and 64 threads 22, 14 and 12 us, x 8192 36, 29 and 27; x 151936 with 256 and 128 449 and 428). fp32 gradients of the longest rows are
    // better off in larger ones: one given token, 256 and 128 threads, fp32 logits 4096 x 151936 797 and 829 us, x 32000 177 and 181, x 8192 54 and 48, x 4096 31 and 27,
    // x 2049 24 and 17; bf16 ones 650 and 652, 163 and 159, 50 and 43, 30 and 25, 24 and 16.
    constexpr bool O16 = sizeof(O) == 2;
    if (O16 && p.vocab <= 8192 && rows >= 16 * sm_count && p.n_tokens <= 64) return launch_backward<T, O, 64>(p, rows, sm_count, st);
    if ((O16 || p.vocab <= 4096) && rows >= 8 * sm_count) return launch_backward<T, O, 128>(p, rows, sm_count, st);
    return launch_backward<T, O, 256>(p, rows, sm_count, st);
}

}  // namespace

void token_logprobs_plan(int es, int n_rows, int vocab, int n_tokens, int n_top, int sm_count, int32_t* info) {
    const Form f = forward_form(es, n_rows, vocab, n_tokens, n_top, sm_count);
    info[0] = f.threads; info[1] = f.cs; info[2] = f.grid;
}

int launch_token_logprobs(const Launch& L, const dflash_token_logprobs_args& a) {
    ForwardParams p{};
    p.logits = a.logits; p.tokens = a.tokens; p.logprob = a.logprob; p.stats = a.stats; p.entropy = a.entropy;
    p.top_ids = a.top_ids; p.top_logprob = a.top_logprob; p.status = L.status;
    p.ld = a.row_stride ? a.row_stride : a.vocab; p.n_rows = a.n_rows; p.vocab = a.vocab; p.n_tokens = a.n_tokens; p.n_top = a.n_top;
    p.end = reinterpret_cast<const char*>(a.logits) + ((int64_t)(a.n_rows - 1) * p.ld + a.vocab) * elem_size(a.logits_dtype);
    p.temperature = a.temperature; p.c = (float)(1.4426950408889634 / (double)a.temperature);
    const cudaError_t e = a.logits_dtype == DFLASH_BF16 ? launch_forward<__nv_bfloat16>(p, L.h->sm_count, L.st)
                                                        : launch_forward<float>(p, L.h->sm_count, L.st);
    g_launches += 1;
    return e == cudaSuccess ? DFLASH_OK : DFLASH_ERR_CUDA;
}

int launch_token_logprobs_bwd(const Launch& L, const dflash_token_logprobs_bwd_args& a) {
    BackwardParams p{};
    p.logits = a.logits; p.tokens = a.tokens; p.stats = a.stats; p.entropy = a.entropy; p.d_logprob = a.d_logprob; p.d_entropy = a.d_entropy;
    p.dlogits = a.dlogits; p.status = L.status;
    p.ld = a.row_stride ? a.row_stride : a.vocab; p.d_ld = a.dlogits_row_stride ? a.dlogits_row_stride : a.vocab;
    p.vocab = a.vocab; p.n_tokens = a.n_tokens;
    p.part = a.temperature > 1.f ? 0.5f : 1.f;
    p.c = (float)(1.4426950408889634 / (double)a.temperature / (double)p.part);
    // The sum of a row's gradients may pass fp32's range where 1 / T brings it back. 2^-8 does for the most of them and the largest entropy; a factor that is not
    // below 1 / T takes nothing from those whose share is a normal number.
    p.scale = std::ldexp(1.f, -std::min(8, std::max(0, std::ilogb(a.temperature))));
    p.inv_t = (float)(1.0 / ((double)a.temperature * (double)p.scale));
    const bool in16 = a.logits_dtype == DFLASH_BF16, out16 = a.dlogits_dtype == DFLASH_BF16;
    cudaError_t e;
    if (in16) e = out16 ? launch_backward<__nv_bfloat16, __nv_bfloat16>(p, a.n_rows, L.h->sm_count, L.st) : launch_backward<__nv_bfloat16, float>(p, a.n_rows, L.h->sm_count, L.st);
    else e = out16 ? launch_backward<float, __nv_bfloat16>(p, a.n_rows, L.h->sm_count, L.st) : launch_backward<float, float>(p, a.n_rows, L.h->sm_count, L.st);
    g_launches += 1;
    return e == cudaSuccess ? DFLASH_OK : DFLASH_ERR_CUDA;
}

}  // namespace dflash
