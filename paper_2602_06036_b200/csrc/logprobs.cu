// Log probabilities of given tokens with the entropy and the top alternatives of a row of logits, and their gradient.
// With y = (z - M) / T, M the row's maximum and S = sum exp(y):
//   logprob(v) = y_v - ln S,   entropy = ln S - (sum y exp(y)) / S,
//   dz_v = (1/T) [ sum of g_i over the given tokens i that are v  -  p_v (G + gH (ln p_v + entropy)) ],  G = sum of all g_i, p = exp(logprob).
// Forward: one pass over the logits. Every thread keeps (m, s, w) = (its maximum, sum e, sum e y) of what it has seen, e = exp(y) with its own m,
// and the entries that may be among the row's n_top largest go to a small list in shared memory (see `Candidates`).
// Bound by HBM: 2 or 4 bytes an entry against about 6 issue slots and one exponential.
#include "logprobs.cuh"
#include "softmax_rows.cuh"

#include <cmath>

namespace dflash {
namespace {

constexpr int THREADS = 512, UNROLL = 4, CTAS_PER_SM = 2;      // 16-byte vectors per thread in flight; 32 KB a CTA
constexpr int MAX_CLUSTER = 8;
constexpr int RANK_MAX = 256;                                  // candidates ranked by comparing each with each
constexpr float LN2 = 0.6931471805599453f;
constexpr float FAR = -1.0e4f;                                 // below this many powers of two a term is 0, and its exponent only has to stay finite

// ---- a row as 16-byte vectors -----------------------------------------------------------------------------------
// Vector j holds entries j * VE - shift + (0 .. VE-1): the vectors lie on 16-byte borders whatever the row's start. The first and
// the last one may reach beyond the row: what they hold outside of it is not read and stands for -inf.
template <typename T>
struct Row {
    static constexpr int VE = 16 / (int)sizeof(T);
    const T* z;
    int vocab, shift, n_vec;
    __device__ __forceinline__ Row(const T* row, int v) : z(row), vocab(v) {
        shift = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        n_vec = (v + shift + VE - 1) / VE;
    }
    __device__ __forceinline__ int first(int j) const { return j * VE - shift; }
    __device__ __forceinline__ uint4 load(int j) const {
        const int i0 = first(j);
        if (i0 >= 0 && i0 + VE <= vocab) return __ldcs(reinterpret_cast<const uint4*>(z + i0));
        uint32_t w[4];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = i0 + e >= 0 && i0 + e < vocab ? __float_as_uint(z[i0 + e]) : 0xff800000u;
        } else {
            const uint16_t* h = reinterpret_cast<const uint16_t*>(z);
            auto one = [&](int i) { return (uint32_t)(i >= 0 && i < vocab ? h[i] : (uint16_t)0xff80u); };
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = one(i0 + 2 * e) | one(i0 + 2 * e + 1) << 16;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// largest entry of a vector; NaN has no say
__device__ __forceinline__ float vec_max(const uint4& v, float) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
}
__device__ __forceinline__ float vec_max(const uint4& v, __nv_bfloat16) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
}

// ---- statistics ----------------------------------------------------------------------------------------------------
// m: maximum, s: sum of 2^((z - m) c), w: sum of 2^((z - m) c) (z - m) c
struct Stat {
    float m, s, w;
};
// to a maximum `to` that is not smaller
__device__ __forceinline__ Stat raised(const Stat& a, float to, float c) {
    if (a.m == to) return a;
    const float d = a.m == -CUDART_INF_F ? FAR : fmaxf((a.m - to) * c, FAR), f = fast_exp2(d);
    return Stat{to, a.s * f, (a.w + a.s * d) * f};
}
__device__ __forceinline__ Stat merged(const Stat& a, const Stat& b, float c) {
    const float m = fmaxf(a.m, b.m);
    const Stat x = raised(a, m, c), y = raised(b, m, c);
    return Stat{m, x.s + y.s, x.w + y.w};
}
// entries f[] into the sums; base = m, or 0 as long as m is -inf (every term is 0 then)
template <int N>
__device__ __forceinline__ void add_terms(Stat& t, const float (&f)[N], float base, float c) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float y = (f[e] - base) * c, x = fast_exp2(y);
        t.s += x;
        t.w = fmaf(x, fmaxf(y, FAR), t.w);
    }
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
constexpr unsigned long long NO_KEY = (unsigned long long)0x007fffffu << 32 | 0xffffffffu;      // not below any key of -inf, below all others

// most threads of a tile that may hold candidates; their entries fit behind a full list
__host__ __device__ __forceinline__ int most_threads(int n_top) { return n_top + n_top / 4 + 8; }
template <typename T>
__host__ __device__ __forceinline__ int list_capacity(int n_top) {
    const int a = n_top + most_threads(n_top) * UNROLL * Row<T>::VE;
    return a > RANK_MAX ? a : RANK_MAX;
}

// The list of a CTA: keys above `floor`, of which at least n_top have been seen as soon as floor > NO_KEY. Later tiles hold larger indices, so
// that an entry equal in value to the floor's loses to those: they are compared by value alone.
struct Candidates {
    unsigned long long* list;      // [capacity]
    unsigned long long* few;       // [RANK_MAX]
    int* count;                    // entries of list
    int n_top, capacity;
    unsigned long long floor;
    float floor_z;

    __device__ __forceinline__ void raise(unsigned long long to) {
        floor = to;
        floor_z = value_of(to);
    }
    // all threads: the list becomes its n_top largest keys in falling order
    __device__ void rank() {
        __syncthreads();
        int n = *count;
        const unsigned long long* from = list;
        if (n > RANK_MAX) {        // a lower bound that leaves few enough, found by halving
            unsigned long long lo = 0, hi = ~0ull;
            while (true) {
                const unsigned long long mid = lo + (hi - lo) / 2;
                int above = 0;
                for (int i = 0; i < n; i += THREADS) above += __syncthreads_count(i + (int)threadIdx.x < n && list[i + threadIdx.x] > mid);
                if (above < n_top) { hi = mid; continue; }
                lo = mid;
                if (above <= RANK_MAX) break;
            }
            if (threadIdx.x == 0) *count = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < n; i += THREADS)
                if (list[i] > lo) few[atomicAdd(count, 1)] = list[i];
            __syncthreads();
            n = *count;
            from = few;
        }
        unsigned long long mine = 0;
        int above = 0;
        if ((int)threadIdx.x < n) {
            mine = from[threadIdx.x];
            for (int i = 0; i < n; ++i) above += from[i] > mine;
        }
        __syncthreads();
        if ((int)threadIdx.x < n && above < n_top) list[above] = mine;
        if (threadIdx.x == 0) *count = min(n, n_top);
        __syncthreads();
        if (n >= n_top) raise(list[n_top - 1]);
        __syncthreads();           // (the floor has been read before the next append)
    }
    // all threads, once a tile: `raw` are the thread's vectors tid + u * THREADS of the tile at vector j0, top its largest entry
    template <typename T>
    __device__ void take(const Row<T>& row, const uint4 (&raw)[UNROLL], int j0, float top) {
        constexpr int VE = Row<T>::VE;
        int hits = __syncthreads_count(top > floor_z);
        if (hits == 0) return;
        bool strict = true;        // by value alone
        if (hits > most_threads(n_top)) {
            // The n_top-th largest of the threads' maxima bounds the n_top-th largest entry from below, and few entries lie above it:
            // halve until between n_top and most_threads(n_top) maxima do.
            unsigned long long best = 0;
            if (top > floor_z) {
#pragma unroll
                for (int u = UNROLL - 1; u >= 0; --u) {
                    float f[VE];
                    unpack16(raw[u], f, T());
#pragma unroll
                    for (int e = VE - 1; e >= 0; --e)
                        if (f[e] == top) best = key_of(top, row.first(j0 + u * THREADS + (int)threadIdx.x) + e);
                }
            }
            unsigned long long lo = floor, hi = ~0ull;
            while (true) {
                const unsigned long long mid = lo + (hi - lo) / 2;
                hits = __syncthreads_count(best > mid);
                if (hits < n_top) { hi = mid; continue; }
                lo = mid;
                if (hits <= most_threads(n_top)) break;
            }
            raise(lo);
            strict = false;
        }
        if (*count + hits * UNROLL * VE > capacity) {      // (no thread appends before all have read the count: rank() and the barrier below)
            const unsigned long long f = floor;
            rank();
            if (f >= floor) raise(f);                       // the tile's own bound, where that is the higher one
            else strict = true;                             // the list's n_top-th, an entry of an earlier tile
        }
        __syncthreads();
        if (top >= floor_z) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                float f[VE];
                unpack16(raw[u], f, T());
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    if (f[e] >= floor_z) {
                        const unsigned long long k = key_of(f[e], row.first(j0 + u * THREADS + (int)threadIdx.x) + e);
                        if (strict ? f[e] > floor_z : k > floor) list[atomicAdd(count, 1)] = k;
                    }
                }
            }
        }
    }
};

struct ForwardParams {
    const void* logits;
    const int32_t* tokens;
    float *logprob, *stats, *entropy, *top_logprob;
    int32_t *top_ids, *status;
    int64_t ld;
    int32_t vocab, n_tokens, n_top, capacity;
    float temperature, c;          // c = log2(e) / T
};

// What a CTA of a cluster tells the others about its stretch of the row
struct Told {
    float m, s, w;
    int n;                         // entries of its list
};

__device__ __forceinline__ void st_cluster_u64(const void* local_smem, uint32_t rank, unsigned long long v) {      // the same variable in CTA `rank`
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(ptx::mapa_shared(ptx::smem_u32(local_smem), rank)), "l"(v) : "memory");
}

// A cluster of CS CTAs per row, a CTA per stretch of its vectors.
template <typename T, int CS>
__global__ void __launch_bounds__(THREADS, CTAS_PER_SM) token_logprobs_kernel(const ForwardParams p) {
    extern __shared__ unsigned long long dyn[];            // list [capacity], few [RANK_MAX], then from every CTA: told [CS][2], keys [CS][n_top]
    __shared__ Stat sh[THREADS / 32];
    __shared__ int count;
    ptx::pdl_trigger();
    ptx::pdl_wait();
    if constexpr (CS > 1) ptx::cluster_arrive();           // (waited for before the first store into another CTA)
    const int tid = threadIdx.x, r = blockIdx.x / CS, rank = CS > 1 ? (int)ptx::cluster_ctarank() : 0;
    const T* z = reinterpret_cast<const T*>(p.logits) + (int64_t)r * p.ld;
    const Row<T> row(z, p.vocab);
    const int per = (row.n_vec + CS - 1) / CS, lo = min(rank * per, row.n_vec), hi = min(row.n_vec, lo + per);
    // a given token's logit, early (every CTA holds the row's result in the end; the first one writes it)
    const int tok = tid < p.n_tokens && rank == 0 ? p.tokens[(int64_t)r * p.n_tokens + tid] : -1;
    float z_tok = 0.f;
    if (tok >= p.vocab && p.status) atomicOr(p.status, DFLASH_DEV_BAD_TOKEN);
    if (tok >= 0 && tok < p.vocab) z_tok = as_f(z[tok]);
    Candidates cand;
    cand.list = dyn;
    cand.few = dyn + p.capacity;
    cand.count = &count;
    cand.n_top = p.n_top;
    cand.capacity = p.capacity;
    cand.raise(NO_KEY);
    if (tid == 0) count = 0;
    const uint4 none = sizeof(T) == 4 ? make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u) : make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
    Stat t{-CUDART_INF_F, 0.f, 0.f};
    uint4 next[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) next[u] = lo + u * THREADS + tid < hi ? row.load(lo + u * THREADS + tid) : none;
    for (int j0 = lo; j0 < hi; j0 += UNROLL * THREADS) {
        uint4 raw[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            raw[u] = next[u];
            const int j = j0 + (UNROLL + u) * THREADS + tid;
            next[u] = j < hi ? row.load(j) : none;
        }
        float top = vec_max(raw[0], T());
#pragma unroll
        for (int u = 1; u < UNROLL; ++u) top = fmaxf(top, vec_max(raw[u], T()));
        if (top > t.m) t = raised(t, top, p.c);
        const float base = t.m == -CUDART_INF_F ? 0.f : t.m;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float f[Row<T>::VE];
            unpack16(raw[u], f, T());
            add_terms(t, f, base, p.c);
        }
        if (p.n_top > 0) cand.take(row, raw, j0, top);
    }
    // ---- the CTA's results: warp, CTA
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        t = merged(t, Stat{__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.s, o), __shfl_xor_sync(0xffffffffu, t.w, o)}, p.c);
    if ((tid & 31) == 0) sh[tid >> 5] = t;
    if (p.n_top > 0) cand.rank();
    else __syncthreads();
    t = sh[tid & (THREADS / 32 - 1)];
#pragma unroll
    for (int o = THREADS / 64; o > 0; o >>= 1)
        t = merged(t, Stat{__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.s, o), __shfl_xor_sync(0xffffffffu, t.w, o)}, p.c);
    int n_list = p.n_top > 0 ? count : 0;
    // ---- the cluster's
    Told* told = reinterpret_cast<Told*>(dyn + p.capacity + RANK_MAX);
    unsigned long long* keys = dyn + p.capacity + RANK_MAX + 2 * CS;
    if constexpr (CS > 1) {
        ptx::cluster_wait();                               // every CTA runs
        if (tid < CS) {
            const Told mine{t.m, t.s, t.w, n_list};
            const unsigned long long* w = reinterpret_cast<const unsigned long long*>(&mine);
            st_cluster_u64(told + rank, tid, w[0]);
            st_cluster_u64(reinterpret_cast<const char*>(told + rank) + 8, tid, w[1]);
        }
        for (int i = tid; i < CS * n_list; i += THREADS) st_cluster_u64(keys + rank * p.n_top + i % n_list, i / n_list, cand.list[i % n_list]);
        __syncwarp();
        ptx::cluster_sync_all();                           // no CTA writes into another one after this
        t = Stat{told[0].m, told[0].s, told[0].w};
#pragma unroll
        for (int q = 1; q < CS; ++q) t = merged(t, Stat{told[q].m, told[q].s, told[q].w}, p.c);
    }
    const bool empty = t.m == -CUDART_INF_F;
    // (a row that holds NaN has a sum of NaN; one of -inf and NaN has no maximum, but is not empty either)
    const float log_sum = empty && t.s == 0.f ? 0.f : logf(t.s);
    if (rank == 0) {
        if (tid == 0) {
            if (p.stats) *reinterpret_cast<float2*>(p.stats + 2 * (int64_t)r) = make_float2(t.m, log_sum);
            if (p.entropy) p.entropy[r] = empty && t.s == 0.f ? 0.f : log_sum - t.w * LN2 / t.s;
        }
        if (tid < p.n_tokens) {
            float lp = 0.f;
            if (tok >= 0 && tok < p.vocab) lp = empty && t.s == 0.f ? -CUDART_INF_F : (z_tok - t.m) / p.temperature - log_sum;
            p.logprob[(int64_t)r * p.n_tokens + tid] = lp;
        }
    }
    if (p.n_top > 0) {
        int32_t* ids = p.top_ids + (int64_t)r * p.n_top;
        float* lps = p.top_logprob + (int64_t)r * p.n_top;
        int total = n_list;
        if constexpr (CS == 1) {
            if (tid < n_list) {
                ids[tid] = index_of(cand.list[tid]);
                lps[tid] = (value_of(cand.list[tid]) - t.m) / p.temperature - log_sum;
            }
        } else {
            // a key's place in the row: its place in the CTA's own list and the number of larger ones in each other list, one lane a list
            total = 0;
#pragma unroll
            for (int q = 0; q < CS; ++q) total += told[q].n;
            const int q = tid % CS;
            for (int i0 = 0; i0 < n_list; i0 += THREADS / CS) {
                const int i = i0 + tid / CS;
                int above = 0;
                unsigned long long k = 0;
                if (i < n_list) {
                    k = cand.list[i];
                    int b = told[q].n, a = 0;              // keys [0, a) of list q are larger, those from b on are not
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
                    lps[above] = (value_of(k) - t.m) / p.temperature - log_sum;
                }
            }
        }
        for (int i = total + tid; rank == 0 && i < p.n_top; i += THREADS) {      // fewer entries than were asked for
            ids[i] = -1;
            lps[i] = -CUDART_INF_F;
        }
    }
}

template <typename T, int CS>
cudaError_t launch_forward(const ForwardParams& p, int rows, cudaStream_t st) {
    const size_t smem = p.n_top > 0 ? (size_t)(p.capacity + RANK_MAX + CS * (2 + p.n_top)) * 8 : (size_t)(2 * CS) * 8;
    static bool attr_set[MAX_DEVICES] = {};
    const int dev = current_device_slot();
    if (dev < 0) return cudaErrorInvalidDevice;
    if (!attr_set[dev]) {
        const int most = (list_capacity<T>(LP_MAX_TOP) + RANK_MAX + CS * (2 + LP_MAX_TOP)) * 8;
        const cudaError_t e = cudaFuncSetAttribute(token_logprobs_kernel<T, CS>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e != cudaSuccess) return e;
        attr_set[dev] = true;
    }
    if (CS == 1) return launch_pdl(token_logprobs_kernel<T, CS>, dim3(rows), dim3(THREADS), smem, st, p);
    return launch_pdl_cluster(token_logprobs_kernel<T, CS>, dim3(rows * CS), dim3(THREADS), smem, st, CS, p);
}

template <typename T>
cudaError_t launch_forward(ForwardParams p, int rows, int sm_count, cudaStream_t st) {
    p.capacity = p.n_top > 0 ? list_capacity<T>(p.n_top) : 0;
    if (p.n_top == 0) p.capacity = -RANK_MAX;              // (no list: what the CTAs tell each other comes first)
    // CTAs per row: as many as it takes to fill the GPU, as long as each has a tile of its own
    const int tiles = (p.vocab + UNROLL * THREADS * Row<T>::VE - 1) / (UNROLL * THREADS * Row<T>::VE);
    int cs = 1;
    while (cs < MAX_CLUSTER && cs < tiles && (int64_t)rows * cs < CTAS_PER_SM * sm_count) cs *= 2;
    switch (cs) {
        case 1: return launch_forward<T, 1>(p, rows, st);
        case 2: return launch_forward<T, 2>(p, rows, st);
        case 4: return launch_forward<T, 4>(p, rows, st);
        default: return launch_forward<T, 8>(p, rows, st);
    }
}

// ---- gradient ----------------------------------------------------------------------------------------------------------
constexpr int B_THREADS = 256, B_UNROLL = 4, GROUP = 8;        // groups of 8 entries a thread, 4 of them under way

struct BackwardParams {
    const void* logits;
    const int32_t* tokens;
    const float *stats, *entropy, *d_logprob, *d_entropy;
    void* dlogits;
    int32_t* status;
    int64_t ld, d_ld;
    int32_t vocab, n_tokens, pieces, per_piece;                // entries of a piece: a multiple of GROUP
    float inv_t, c;
};

template <typename T>
__device__ __forceinline__ void load_group(const T* src, float (&z)[GROUP]) {
    constexpr int VE = Row<T>::VE;
#pragma unroll
    for (int k = 0; k < GROUP / VE; ++k) {
        float f[VE];
        unpack16(__ldcs(reinterpret_cast<const uint4*>(src) + k), f, T());
#pragma unroll
        for (int e = 0; e < VE; ++e) z[k * VE + e] = f[e];
    }
}
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
template <typename T, typename O>
__global__ void __launch_bounds__(B_THREADS) token_logprobs_bwd_kernel(const BackwardParams p) {
    __shared__ int s_tok[LP_MAX_TOKENS];
    __shared__ float s_g[LP_MAX_TOKENS], s_sum[B_THREADS / 32];
    ptx::pdl_trigger();
    ptx::pdl_wait();
    const int tid = threadIdx.x;
    const int r = blockIdx.x / p.pieces, piece = blockIdx.x % p.pieces;
    const int lo = piece * p.per_piece, hi = min(p.vocab, lo + p.per_piece);
    const T* z = reinterpret_cast<const T*>(p.logits) + (int64_t)r * p.ld;
    O* dz = reinterpret_cast<O*>(p.dlogits) + (int64_t)r * p.d_ld;
    // ---- the row's numbers
    int tok = -1;
    float g = 0.f, z_tok = 0.f;
    if (tid < p.n_tokens) {
        tok = p.tokens[(int64_t)r * p.n_tokens + tid];
        if (tok >= p.vocab) {
            if (p.status && piece == 0) atomicOr(p.status, DFLASH_DEV_BAD_TOKEN);
            tok = -1;
        }
        if (tok >= 0) g = p.d_logprob[(int64_t)r * p.n_tokens + tid];
        if (tok >= lo && tok < hi) z_tok = as_f(z[tok]);       // before any store: dlogits may be the logits
        s_tok[tid] = tok;
        s_g[tid] = g;
    }
    float sum = g;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((tid & 31) == 0) s_sum[tid >> 5] = sum;
    const int any = __syncthreads_or(g != 0.f);
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < LP_MAX_TOKENS / 32; ++w) sum += s_sum[w];
    const float top = p.stats[2 * (int64_t)r], log_sum = p.stats[2 * (int64_t)r + 1];
    const float gh = p.d_entropy ? p.d_entropy[r] : 0.f, h = p.d_entropy ? p.entropy[r] : 0.f;
    const bool off = (!any && gh == 0.f) || (top == -CUDART_INF_F && log_sum == 0.f);      // nothing comes in, or a row of -inf
    // with y = log2 p = (z - top) c - log_sum / ln 2:  dz = p (a + b y)
    const float sub = log_sum * LOG2E, a = -(sum + gh * h) * p.inv_t, b = -gh * LN2 * p.inv_t;
    auto grad = [&](float v) {
        const float y = fmaf(v - top, p.c, -sub);
        return fast_exp2(y) * fmaf(b, fmaxf(y, FAR), a);
    };
    // ---- the piece: groups whose loads and stores both lie on 16-byte borders start at entry `first`, if there is such a place
    constexpr int AZ = 16 / (int)sizeof(T), AO = 16 / (int)sizeof(O), AM = AZ > AO ? AZ : AO;
    const int pz = (int)((reinterpret_cast<uintptr_t>(z + lo) & 15) / sizeof(T)), po = (int)((reinterpret_cast<uintptr_t>(dz + lo) & 15) / sizeof(O));
    int first = 0;
    while (first < AM && ((pz + first) % AZ != 0 || (po + first) % AO != 0)) ++first;
    const bool vec = first < AM;
    const int begin = vec ? min(lo + first, hi) : hi, n_group = (hi - begin) / GROUP;
    for (int i0 = 0; i0 < n_group; i0 += B_UNROLL * B_THREADS) {
        float v[B_UNROLL][GROUP];
        if (!off) {
#pragma unroll
            for (int u = 0; u < B_UNROLL; ++u) {
                const int i = i0 + u * B_THREADS + tid;
                if (i < n_group) load_group(z + begin + i * GROUP, v[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < B_UNROLL; ++u) {
            const int i = i0 + u * B_THREADS + tid;
            if (i < n_group) {
                float d[GROUP];
#pragma unroll
                for (int e = 0; e < GROUP; ++e) d[e] = off ? 0.f : grad(v[u][e]);
                store_group(dz + begin + i * GROUP, d);
            }
        }
    }
    const int rest = begin + n_group * GROUP;                  // entries in front of and behind the groups: all of them where there are none
    for (int i = lo + tid; i < begin && vec; i += B_THREADS) store_entry(dz + i, off ? 0.f : grad(as_f(z[i])));
    for (int i = (vec ? rest : lo) + tid; i < hi; i += B_THREADS) store_entry(dz + i, off ? 0.f : grad(as_f(z[i])));
    // ---- the given tokens' own entries: the first of equal ones adds their gradients up, in the order of the list
    __syncthreads();
    if (!off && tok >= lo && tok < hi) {
        float own = 0.f;
        bool earlier = false;
        for (int i = 0; i < p.n_tokens; ++i) {
            if (s_tok[i] == tok) {
                earlier |= i < tid;
                own += s_g[i];
            }
        }
        if (!earlier) store_entry(dz + tok, fmaf(own, p.inv_t, grad(z_tok)));
    }
}

template <typename T, typename O>
cudaError_t launch_backward(BackwardParams p, int rows, int sm_count, cudaStream_t st) {
    // pieces of a row: whole tiles, few enough that a CTA's start is little beside its work, enough to fill the GPU
    constexpr int TILE = B_THREADS * B_UNROLL * GROUP;
    const int tiles = (p.vocab + TILE - 1) / TILE;
    int per = std::min(tiles, 4);
    while (per > 1 && (int64_t)rows * ((tiles + per - 1) / per) < 8ll * sm_count) --per;
    p.per_piece = per * TILE;
    p.pieces = (p.vocab + p.per_piece - 1) / p.per_piece;
    return launch_pdl(token_logprobs_bwd_kernel<T, O>, dim3((unsigned)((int64_t)rows * p.pieces)), dim3(B_THREADS), 0, st, p);
}

}  // namespace

int launch_token_logprobs(const Launch& L, const dflash_token_logprobs_args& a) {
    ForwardParams p{};
    p.logits = a.logits; p.tokens = a.tokens; p.logprob = a.logprob; p.stats = a.stats; p.entropy = a.entropy;
    p.top_ids = a.top_ids; p.top_logprob = a.top_logprob; p.status = L.status;
    p.ld = a.row_stride ? a.row_stride : a.vocab; p.vocab = a.vocab; p.n_tokens = a.n_tokens; p.n_top = a.n_top;
    p.temperature = a.temperature; p.c = (float)(1.4426950408889634 / (double)a.temperature);
    const cudaError_t e = a.logits_dtype == DFLASH_BF16 ? launch_forward<__nv_bfloat16>(p, a.n_rows, L.h->sm_count, L.st)
                                                        : launch_forward<float>(p, a.n_rows, L.h->sm_count, L.st);
    g_launches += 1;
    return e == cudaSuccess ? DFLASH_OK : DFLASH_ERR_CUDA;
}

int launch_token_logprobs_bwd(const Launch& L, const dflash_token_logprobs_bwd_args& a) {
    BackwardParams p{};
    p.logits = a.logits; p.tokens = a.tokens; p.stats = a.stats; p.entropy = a.entropy; p.d_logprob = a.d_logprob; p.d_entropy = a.d_entropy;
    p.dlogits = a.dlogits; p.status = L.status;
    p.ld = a.row_stride ? a.row_stride : a.vocab; p.d_ld = a.dlogits_row_stride ? a.dlogits_row_stride : a.vocab;
    p.vocab = a.vocab; p.n_tokens = a.n_tokens;
    p.inv_t = (float)(1.0 / (double)a.temperature); p.c = (float)(1.4426950408889634 / (double)a.temperature);
    const bool in16 = a.logits_dtype == DFLASH_BF16, out16 = a.dlogits_dtype == DFLASH_BF16;
    cudaError_t e;
    if (in16) e = out16 ? launch_backward<__nv_bfloat16, __nv_bfloat16>(p, a.n_rows, L.h->sm_count, L.st) : launch_backward<__nv_bfloat16, float>(p, a.n_rows, L.h->sm_count, L.st);
    else e = out16 ? launch_backward<float, __nv_bfloat16>(p, a.n_rows, L.h->sm_count, L.st) : launch_backward<float, float>(p, a.n_rows, L.h->sm_count, L.st);
    g_launches += 1;
    return e == cudaSuccess ? DFLASH_OK : DFLASH_ERR_CUDA;
}

}  // namespace dflash
