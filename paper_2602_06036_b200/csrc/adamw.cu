// AdamW over many tensors at once, with clipping by the norm of all gradients and states of 32 or 8 bits:
//   g' = grad * grad_scale * min(1, max_norm / (norm + 1e-6)),   m = b1 m + (1 - b1) g',   v = b2 v + (1 - b2) g'^2,
//   w = w - lr wd w - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps).
// The tensors are described in the launch's parameters (no table in device memory to keep), as many as fit one launch. A launch cuts them into
// chunks of CHUNK entries and every CTA takes chunks in turn. Bound by HBM: 2 to 4 bytes of gradient, 4 to 10 of weights and 16 (or 4.1) of states an entry.
// Measured without clipping for 2.5e8 weights, share of the copy rate: 32-bit states 0.94 to 0.97, 8-bit ones 0.90 beside master copies, 0.67 without (65
// instructions an entry, a third of them roots, divisions and roundings that have to be exact, hold it then). What is under way decides: four blocks
// of a warp and two CTAs an SM against two and four: 0.95 and 0.92, 8 bits 0.90 and 0.77. Clipping adds the reading of the gradients: 2.0e9 bytes 400 us.
// Norm: a launch in front adds the squares up, a partial sum a CTA; each CTA of the step adds the partial sums up itself, in their order, which
// costs less than a third launch and gives all of them, and every run, the same number.
// Borders: four neighbouring entries take one access of each buffer where such groups lie on their borders in all of them, counted from the tensor's start or from up
// to three entries in front of it (pieces of flat buffers). Elsewhere, and at a tensor's ends, a lane takes entries 32 apart one by one: 6.7e6 bf16 weights in 160
// pieces with 8-bit states 41 us instead of 25.
// 8-bit states: e4m3 codes of m and of sqrt(v), with one fp32 scale (the largest magnitude / 448) for 128 entries. A float code keeps its 4
// significant bits over a factor of 2^15 below the largest of its 128 (half a step: 2^-4 of the value), where an 8-bit linear code loses all entries
// below 1/254 of it; sqrt(v) spans half as many powers of two as v. The update of a step uses m and v before their rounding. A root that is not
// 0 is never rounded to 0, which would make its next step m / eps.
#include "adamw.cuh"
#include "ptx_sm100.cuh"

#include <cuda_fp8.h>
#include <math_constants.h>

#include <algorithm>
#include <cmath>
#include <limits>
#include <type_traits>

namespace dflash {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32, PER_LANE = 4;
constexpr int BLOCK = 32 * PER_LANE;                    // entries of a warp's turn, and of an 8-bit state that share a scale
constexpr int UNROLL = 4;                               // blocks of a warp under way
constexpr int CHUNK = WARPS * UNROLL * BLOCK;           // 4096
constexpr int CTAS_PER_SM = 2, NORM_CTAS_PER_SM = 4;
constexpr int NORM_UNROLL = 4, NORM_BYTES = NORM_UNROLL * THREADS * 16;      // of a chunk of gradients
constexpr int MAX_TENSORS = 320;                        // descriptors of a launch: 30 KB of its 32 KB of parameters
constexpr int FEW_TENSORS = 32;                         // a launch of that many carries 3 KB, which takes 1 us less

enum Weights { W_F32 = 0, W_BF16 = 1, W_MASTER = 2 };      // fp32, bf16, bf16 with a master copy in fp32

struct Tensor {
    void* param;
    const void* grad;
    float* master;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t n;
    float lr_wd, step_size;                             // lr * weight_decay; lr / (1 - b1^t), or both without lr and t where those live on the device
    int32_t kind;                                       // Weights * 4 + (gradients bf16) * 2 + (states of 8 bits)
    int32_t wide;                                       // entries in groups of four lie on borders that allow one access each,
    int32_t lead;                                       // those that start `lead` entries in front of the first one
};
template <int N>
struct Table {
    Tensor t[N];
    int64_t first[N + 1];                               // spans in front of each tensor
    int32_t n, span;                                    // a span: so many chunks one behind the other
};
struct StepParams {
    const double* partial;                              // [n_partial] sums of squared gradients, or nullptr: no norm
    int32_t n_partial;
    float* norm_out;
    const float* lr;                                    // nullptr: in the table
    const int32_t* step;
    double ln_b1, ln_b2;
    float b1, b2, one_b1, one_b2, eps, rsqrt_bc2, grad_scale, max_norm;
    int32_t* status;
};

static_assert(sizeof(Table<MAX_TENSORS>) + sizeof(StepParams) <= 32764, "the parameters of a launch");

template <int N>
__device__ __forceinline__ int tensor_of(const Table<N>& tab, int64_t chunk, int a) {
    if (chunk < tab.first[a + 1]) return a;             // (as for the chunk before)
    int b = tab.n;                                      // first[a] <= chunk < first[b]
    while (b - a > 1) {
        const int mid = (a + b) / 2;
        if (tab.first[mid] <= chunk) a = mid;
        else b = mid;
    }
    return a;
}

// ---- the four entries of a lane in a block: neighbouring ones (WIDE: all of them there and on their border), or lane, lane + 32, ... (some may be outside) ----
template <bool WIDE>
__device__ __forceinline__ int entry(int e) { return WIDE ? (int)(threadIdx.x & 31) * 4 + e : (int)(threadIdx.x & 31) + 32 * e; }

template <bool WIDE>
__device__ __forceinline__ void load4(const float* p, int from, int to, float (&f)[4]) {
    if constexpr (WIDE) {
        const float4 v = __ldcs(reinterpret_cast<const float4*>(p) + (threadIdx.x & 31));
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = entry<false>(e) >= from && entry<false>(e) < to ? p[entry<false>(e)] : 0.f;
    }
}
template <bool WIDE>
__device__ __forceinline__ void load4(const __nv_bfloat16* p, int from, int to, float (&f)[4]) {
    if constexpr (WIDE) {
        const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p) + (threadIdx.x & 31));
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = entry<false>(e) >= from && entry<false>(e) < to ? __bfloat162float(p[entry<false>(e)]) : 0.f;
    }
}
template <bool WIDE>
__device__ __forceinline__ void store4(float* p, int from, int to, const float (&f)[4]) {
    if constexpr (WIDE) {
        __stcs(reinterpret_cast<float4*>(p) + (threadIdx.x & 31), make_float4(f[0], f[1], f[2], f[3]));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (entry<false>(e) >= from && entry<false>(e) < to) p[entry<false>(e)] = f[e];
    }
}
template <bool WIDE>
__device__ __forceinline__ void store4(__nv_bfloat16* p, int from, int to, const float (&f)[4]) {
    if constexpr (WIDE) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
        __stcs(reinterpret_cast<uint2*>(p) + (threadIdx.x & 31), make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b)));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (entry<false>(e) >= from && entry<false>(e) < to) p[entry<false>(e)] = __float2bfloat16_rn(f[e]);
    }
}
template <bool WIDE>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int to) {
    if constexpr (WIDE) return __ldcs(reinterpret_cast<const uint32_t*>(p) + (threadIdx.x & 31));
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (entry<false>(e) < to) w |= (uint32_t)p[entry<false>(e)] << (8 * e);
    return w;
}
template <bool WIDE>
__device__ __forceinline__ void store_codes(uint8_t* p, int to, uint32_t w) {
    if constexpr (WIDE) {
        __stcs(reinterpret_cast<uint32_t*>(p) + (threadIdx.x & 31), w);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (entry<false>(e) < to) p[entry<false>(e)] = (uint8_t)(w >> (8 * e));
    }
}
__device__ __forceinline__ void decode(uint32_t w, float scale, float (&f)[4]) {
    const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xffffu), __NV_E4M3);
    const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3);
    const float2 x = __half22float2(__half2(a)), y = __half22float2(__half2(b));
    f[0] = x.x * scale; f[1] = x.y * scale; f[2] = y.x * scale; f[3] = y.y * scale;
}
__device__ __forceinline__ uint32_t encode(const float (&f)[4]) {
    const uint32_t a = __nv_cvt_float2_to_fp8x2(make_float2(f[0], f[1]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t b = __nv_cvt_float2_to_fp8x2(make_float2(f[2], f[3]), __NV_SATFINITE, __NV_E4M3);
    return a | b << 16;
}
// The scale of a block whose largest magnitude is `top` (all lanes), and what its entries are multiplied by. A block that holds NaN or an
// infinity gets the scale NaN, one below 2^-117 the scale 0 (its own would no longer be a normal number).
__device__ __forceinline__ float scale_of(float top, float& inv) {
    const float scale = top < 6.0185e-36f ? 0.f : top * (1.f / 448.f);
    inv = scale > 0.f ? 1.f / scale : 0.f;
    return top < CUDART_INF_F ? scale : CUDART_NAN_F;
}
// largest magnitude, as its bits: magnitudes order like them, infinities and then NaN above all numbers
__device__ __forceinline__ uint32_t block_top(const float (&f)[4]) {
    uint32_t t = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) t = max(t, __float_as_uint(f[e]) & 0x7fffffffu);
    return __reduce_max_sync(0xffffffffu, t);
}
// a / b for b of a normal number's size (2 ulp)
__device__ __forceinline__ float quotient(float a, float b) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(b));
    return a * r;
}

// What a thread needs of a tensor, at its warp's first block of a chunk
template <int KIND>
struct Place {
    static constexpr int W = KIND >> 2;
    static constexpr bool G16 = KIND & 2, S8 = KIND & 1, MASTER = W == W_MASTER, P16 = W != W_F32;
    using G = std::conditional_t<G16, __nv_bfloat16, float>;
    using P = std::conditional_t<P16, __nv_bfloat16, float>;
    using S = std::conditional_t<S8, uint8_t, float>;
    const G* grad;
    P* param;
    float* master;
    S *m, *v;
    float *m_scale, *v_scale;
    __device__ __forceinline__ Place(const Tensor& t, int64_t at)
        : grad(reinterpret_cast<const G*>(t.grad) + at), param(reinterpret_cast<P*>(t.param) + at), master(MASTER ? t.master + at : nullptr),
          m(reinterpret_cast<S*>(t.m) + at), v(reinterpret_cast<S*>(t.v) + at), m_scale(S8 ? t.m_scale + at / BLOCK : nullptr), v_scale(S8 ? t.v_scale + at / BLOCK : nullptr) {}
    __device__ __forceinline__ void next_chunk() {
        grad += CHUNK; param += CHUNK; m += CHUNK; v += CHUNK;
        if constexpr (MASTER) master += CHUNK;
        if constexpr (S8) { m_scale += CHUNK / BLOCK; v_scale += CHUNK / BLOCK; }
    }
};
struct Rates {
    float gs, lr_wd, step_size, rsqrt_bc2;
};

// The warp's blocks of one chunk; at: their first entry's place in the tensor of n. WIDE: all of them lie inside.
// Products and sums of the states are rounded one by one, as the formula is written: a code that lies between two is then rounded alike by whatever else computes it so.
template <int KIND, bool WIDE>
__device__ __forceinline__ void step_blocks(const Place<KIND>& q, int64_t at, int64_t n, const StepParams& p, const Rates& r) {
    constexpr bool S8 = Place<KIND>::S8, MASTER = Place<KIND>::MASTER;
    const int lane = threadIdx.x & 31;
    // entries of block u that lie inside: [from(u), to(u))
    const auto from = [&](int u) { return WIDE ? 0 : (int)max(-(at + u * BLOCK), (int64_t)0); };
    const auto to = [&](int u) { return WIDE ? BLOCK : (int)max(min(n - (at + u * BLOCK), (int64_t)BLOCK), (int64_t)0); };
    float g[UNROLL][4], w[UNROLL][4], m[UNROLL][4], v[UNROLL][4];
    uint32_t cm[UNROLL], cv[UNROLL];
    float sm[UNROLL], sv[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const int o = u * BLOCK;
        load4<WIDE>(q.grad + o, from(u), to(u), g[u]);
        if constexpr (MASTER) load4<WIDE>(q.master + o, from(u), to(u), w[u]);
        else load4<WIDE>(q.param + o, from(u), to(u), w[u]);
        if constexpr (S8) {
            cm[u] = load_codes<WIDE>(q.m + o, to(u));
            cv[u] = load_codes<WIDE>(q.v + o, to(u));
            sm[u] = to(u) > 0 ? q.m_scale[u] : 0.f;
            sv[u] = to(u) > 0 ? q.v_scale[u] : 0.f;
        } else {
            load4<WIDE>(q.m + o, from(u), to(u), m[u]);
            load4<WIDE>(q.v + o, from(u), to(u), v[u]);
        }
    }
    uint32_t tops[2 * UNROLL];                          // largest magnitudes of m, and roots of v, of each block
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const int o = u * BLOCK;
        if constexpr (S8) {
            decode(cm[u], sm[u], m[u]);
            decode(cv[u], sv[u], v[u]);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] *= v[u][e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = __fmul_rn(g[u][e], r.gs);
            m[u][e] = __fadd_rn(__fmul_rn(p.b1, m[u][e]), __fmul_rn(p.one_b1, x));
            v[u][e] = __fadd_rn(__fmul_rn(p.b2, v[u][e]), __fmul_rn(p.one_b2, __fmul_rn(x, x)));
            const float root = sqrtf(v[u][e]);
            w[u][e] = fmaf(-r.lr_wd, w[u][e], w[u][e]) - quotient(r.step_size * m[u][e], fmaf(root, r.rsqrt_bc2, p.eps));
            if constexpr (S8) v[u][e] = root;
        }
        if constexpr (MASTER) store4<WIDE>(q.master + o, from(u), to(u), w[u]);
        // (the weights that the model reads: their rounding to bf16 is not fed back where there is a master copy)
        store4<WIDE>(q.param + o, from(u), to(u), w[u]);
        if constexpr (S8) {
            tops[2 * u] = block_top(m[u]);
            tops[2 * u + 1] = block_top(v[u]);
        } else {
            store4<WIDE>(q.m + o, from(u), to(u), m[u]);
            store4<WIDE>(q.v + o, from(u), to(u), v[u]);
        }
    }
    if constexpr (S8) {
        // a share of the lanes works out each scale, and what entries are multiplied by
        constexpr int SHARE = 32 / (2 * UNROLL);
        uint32_t top = tops[0];
#pragma unroll
        for (int k = 1; k < 2 * UNROLL; ++k) top = lane / SHARE == k ? tops[k] : top;
        float inv;
        const float scale = scale_of(__uint_as_float(top), inv);
        if (lane % SHARE == 0 && to(lane / SHARE / 2) > 0) (lane / SHARE % 2 ? q.v_scale : q.m_scale)[lane / SHARE / 2] = scale;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const float im = __shfl_sync(0xffffffffu, inv, 2 * u * SHARE), iv = __shfl_sync(0xffffffffu, inv, (2 * u + 1) * SHARE);
            const float least = iv > 0.f ? 0.001953125f : 0.f;      // 2^-9: the smallest code
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[u][e] *= im;
                v[u][e] = v[u][e] > 0.f ? fmaxf(v[u][e] * iv, least) : 0.f;
            }
            store_codes<WIDE>(q.m + u * BLOCK, to(u), encode(m[u]));
            store_codes<WIDE>(q.v + u * BLOCK, to(u), encode(v[u]));
        }
    }
}

// `chunks` chunks from entry `at` of the tensor on
template <int KIND>
__device__ __forceinline__ void step_chunks(const Tensor& t, int64_t at, int chunks, const StepParams& p, const Rates& r) {
    const int first = (threadIdx.x >> 5) * UNROLL * BLOCK;
    const int64_t n = t.n;
    const bool can = t.wide;
    Place<KIND> q(t, at + first);
    for (; chunks > 0 && at < n; --chunks, at += CHUNK, q.next_chunk()) {
        if (can && at >= 0 && at + CHUNK <= n) step_blocks<KIND, true>(q, at + first, n, p, r);
        else step_blocks<KIND, false>(q, at + first, n, p, r);
    }
}

// sum over the CTA in a fixed order; every thread gets it
__device__ __forceinline__ double cta_sum(double x, double* sh) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < WARPS; ++k) s += sh[k];
    return s;
}

template <int N>
__global__ void __launch_bounds__(THREADS, CTAS_PER_SM) adamw_kernel(const __grid_constant__ Table<N> tab, const __grid_constant__ StepParams p) {
    __shared__ double sh[WARPS];
    __shared__ float s_bc[2];
    ptx::pdl_trigger();
    ptx::pdl_wait();
    float gs = p.grad_scale;
    if (p.partial) {
        double x = 0.0;
        for (int i = threadIdx.x; i < p.n_partial; i += THREADS) x += p.partial[i];
        const float norm = (float)(sqrt(cta_sum(x, sh)) * fabs((double)p.grad_scale));
        const bool fine = norm < CUDART_INF_F;
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            if (p.norm_out) *p.norm_out = norm;
            if (!fine && p.status) atomicOr(p.status, DFLASH_DEV_NOT_FINITE);
        }
        if (!fine) return;                              // every CTA alike: the step is left out
        if (p.max_norm > 0.f) gs *= fminf(1.f, p.max_norm / (norm + 1e-6f));
    }
    float lr = 1.f, rsqrt_bc2 = p.rsqrt_bc2;
    if (p.lr || p.step) {                               // what of the bias correction and the rate lives on the device
        if (threadIdx.x == 0) {
            const double t = p.step ? (double)max(*p.step, 1) : 1.0;
            s_bc[0] = (p.lr ? *p.lr : 1.f) * (p.step ? (float)(-1.0 / expm1(t * p.ln_b1)) : 1.f);
            s_bc[1] = p.step ? (float)rsqrt(-expm1(t * p.ln_b2)) : p.rsqrt_bc2;
        }
        __syncthreads();
        lr = s_bc[0];
        rsqrt_bc2 = s_bc[1];
    }
    const float wd_lr = p.lr ? *p.lr : 1.f;
    const int64_t chunks = tab.first[tab.n];
    int k = 0;
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        k = tensor_of(tab, c, k);
        const Tensor& t = tab.t[k];
        const int64_t at = (c - tab.first[k]) * CHUNK * tab.span - t.lead;
        const Rates r{gs, t.lr_wd * wd_lr, t.step_size * lr, rsqrt_bc2};
        switch (t.kind) {
#define DFLASH_ADAMW_CASE(K) case K: step_chunks<K>(t, at, tab.span, p, r); break;
            DFLASH_ADAMW_CASE(0) DFLASH_ADAMW_CASE(1) DFLASH_ADAMW_CASE(2) DFLASH_ADAMW_CASE(3)
            DFLASH_ADAMW_CASE(4) DFLASH_ADAMW_CASE(5) DFLASH_ADAMW_CASE(6) DFLASH_ADAMW_CASE(7)
            DFLASH_ADAMW_CASE(8) DFLASH_ADAMW_CASE(9) DFLASH_ADAMW_CASE(10) DFLASH_ADAMW_CASE(11)
#undef DFLASH_ADAMW_CASE
        }
    }
}

__device__ __forceinline__ void add_square(float& s, float x) { s = fmaf(x, x, s); }
__device__ __forceinline__ void add_square(double& s, float x) {
    const float q = x * x;                                  // (one that fp32 does not hold stays infinite: nor could the second moment hold it)
    s += q < CUDART_INF_F ? (double)x * (double)x : (double)q;
}
// sum, in S, of the squares of the entries [from, to) of 16-byte vectors at p, NORM_UNROLL a thread and THREADS apart
template <typename S, typename G, bool WIDE>
__device__ __forceinline__ S squares(const G* p, int64_t from, int64_t to) {
    constexpr int VE = 16 / (int)sizeof(G);
    S s = 0;
    uint4 raw[NORM_UNROLL];
#pragma unroll
    for (int u = 0; u < NORM_UNROLL; ++u) {
        const int64_t i = (int64_t)(u * THREADS + threadIdx.x) * VE;
        raw[u] = make_uint4(0, 0, 0, 0);
        if (WIDE || (i >= from && i + VE <= to)) {
            raw[u] = *reinterpret_cast<const uint4*>(p + i);       // (read again by the step: kept in L2 as far as it goes)
        } else {
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                if (i + e < from || i + e >= to) continue;
                add_square(s, (float)p[i + e]);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < NORM_UNROLL; ++u) {
        const uint32_t w[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (sizeof(G) == 4) {
                add_square(s, __uint_as_float(w[k]));
            } else {
                add_square(s, __uint_as_float(w[k] << 16));
                add_square(s, __uint_as_float(w[k] & 0xffff0000u));
            }
        }
    }
    return s;
}

// sum of the squares of the gradients in this CTA's chunks, each thread's and chunk's added up in S, those sums in double
template <typename S, int N>
__device__ __forceinline__ double cta_squares(const Table<N>& tab, double* sh) {
    double sum = 0.0;
    const int64_t chunks = tab.first[tab.n];
    int k = 0;
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        k = tensor_of(tab, c, k);
        const Tensor& t = tab.t[k];
        const int es = t.kind & 2 ? 2 : 4, size = NORM_BYTES / es;
        const int64_t at = (c - tab.first[k]) * size - t.lead, from = -at, to = t.n - at;
        const bool wide = from <= 0 && to >= size;
        const char* p = reinterpret_cast<const char*>(t.grad) + at * es;
        S s;
        if (t.kind & 2) s = wide ? squares<S, __nv_bfloat16, true>(reinterpret_cast<const __nv_bfloat16*>(p), from, to) : squares<S, __nv_bfloat16, false>(reinterpret_cast<const __nv_bfloat16*>(p), from, to);
        else s = wide ? squares<S, float, true>(reinterpret_cast<const float*>(p), from, to) : squares<S, float, false>(reinterpret_cast<const float*>(p), from, to);
        sum += (double)s;
    }
    return cta_sum(sum, sh);
}

// partial[blockIdx.x] = sum of the squares of the gradients in this CTA's chunks. In the table a chunk has NORM_BYTES, and `lead` entries lie between
// a gradient's start and the 16-byte border in front of it. The 16 or 32 squares of a thread and chunk are added up in fp32, whose range they may pass together
// (32 of 5e18) and below which squares vanish: of a sum of 2^-90 on, that is nothing. Where the sum is none such, all of them are taken in double.
template <int N>
__global__ void __launch_bounds__(THREADS, NORM_CTAS_PER_SM) adamw_norm_kernel(const __grid_constant__ Table<N> tab, double* __restrict__ partial) {
    __shared__ double sh[WARPS];
    ptx::pdl_trigger();
    ptx::pdl_wait();
    double sum = cta_squares<float>(tab, sh);
    if (!(sum >= 8.0779357e-28 && sum < CUDART_INF)) {      // (all threads have the same sum)
        __syncthreads();
        sum = cta_squares<double>(tab, sh);
    }
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

template <int N>
int launch_tables(const Launch& L, const dflash_adamw_args& a) {
    const int launches = std::max(1, (a.n_tensors + N - 1) / N);
    const bool norm = a.max_grad_norm > 0.0 || a.grad_norm;
    StepParams p{};
    p.norm_out = a.grad_norm; p.lr = a.lr_dev; p.step = a.step_dev;
    p.ln_b1 = a.beta1 > 0.0 ? std::log(a.beta1) : -INFINITY;
    p.ln_b2 = a.beta2 > 0.0 ? std::log(a.beta2) : -INFINITY;
    p.b1 = (float)a.beta1; p.b2 = (float)a.beta2; p.one_b1 = (float)(1.0 - a.beta1); p.one_b2 = (float)(1.0 - a.beta2);
    p.eps = (float)a.eps; p.grad_scale = (float)a.grad_scale; p.max_norm = a.max_grad_norm > 0.0 ? std::max((float)a.max_grad_norm, std::numeric_limits<float>::denorm_min()) : 0.f; p.status = L.status;
    const double bc1 = a.step_dev ? 1.0 : -std::expm1(a.step * p.ln_b1), bc2 = a.step_dev ? 1.0 : -std::expm1(a.step * p.ln_b2);
    p.rsqrt_bc2 = (float)(1.0 / std::sqrt(bc2));
    const double lr = a.lr_dev ? 1.0 : a.lr;
    const auto table = [&](int l, bool for_norm, Table<N>& tab) {
        const int from = l * N, n = std::min(N, a.n_tensors - from);
        int64_t chunks = 0, entries = 0;
        for (int i = 0; i < n; ++i) entries += a.tensors[from + i].n;
        // four chunks one behind the other share a look at the table and the addresses, where that leaves every CTA several turns
        tab.span = entries >= (int64_t)64 * CHUNK * CTAS_PER_SM * L.h->sm_count ? 4 : 1;
        for (int i = 0; i < n; ++i) {
            const dflash_adamw_tensor& s = a.tensors[from + i];
            Tensor& t = tab.t[i];
            const bool p16 = s.param_dtype == DFLASH_BF16, g16 = s.grad_dtype == DFLASH_BF16, s8 = s.state_bits == 8;
            t.param = s.param; t.grad = s.grad; t.master = s.master; t.m = s.exp_avg; t.v = s.exp_avg_sq;
            t.m_scale = s.exp_avg_scale; t.v_scale = s.exp_avg_sq_scale; t.n = s.n;
            t.lr_wd = (float)(lr * s.weight_decay * s.lr_scale);
            t.step_size = (float)(lr * s.lr_scale / bc1);
            t.kind = (s.master ? W_MASTER : p16 ? W_BF16 : W_F32) * 4 + g16 * 2 + s8;
            // entries in front of the first one to the next border, by the weights; the same has to do for the others. (The blocks of an 8-bit state start with the
            // tensor.)
            const int pb = p16 ? 2 : 4, gb = g16 ? 2 : 4, sb = s8 ? 1 : 4;
            t.lead = s8 ? 0 : (int)((reinterpret_cast<uintptr_t>(s.param) / pb) & 3);
            const auto border = [&](const void* q, int bytes) { return !q || (reinterpret_cast<uintptr_t>(q) - (uintptr_t)t.lead * bytes) % (4 * bytes) == 0; };
            t.wide = border(s.param, pb) && border(s.grad, gb) && border(s.master, 4) && border(s.exp_avg, sb) && border(s.exp_avg_sq, sb);
            if (!t.wide) t.lead = 0;
            if (for_norm) t.lead = (int)((reinterpret_cast<uintptr_t>(s.grad) & 15) / gb);
            const int64_t size = for_norm ? NORM_BYTES / gb : (int64_t)CHUNK * tab.span;
            tab.first[i] = chunks;
            chunks += s.n > 0 ? (s.n + t.lead + size - 1) / size : 0;
        }
        tab.first[n] = chunks;
        tab.n = n;
        return chunks;
    };
    const auto grid = [&](int64_t chunks, int per_sm) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(chunks, (int64_t)L.h->sm_count * per_sm)); };
    Table<N> tab;
    if (norm) {
        double* partial = reinterpret_cast<double*>(a.workspace);
        p.partial = partial;
        for (int l = 0; l < launches; ++l) {
            const unsigned g = grid(table(l, true, tab), NORM_CTAS_PER_SM);
            if (launch_pdl(adamw_norm_kernel<N>, dim3(g), dim3(THREADS), 0, L.st, tab, partial + p.n_partial) != cudaSuccess) return DFLASH_ERR_CUDA;
            p.n_partial += (int)g;
            g_launches += 1;
        }
    }
    for (int l = 0; l < launches; ++l) {
        const int64_t chunks = table(l, false, tab);
        if (launch_pdl(adamw_kernel<N>, dim3(grid(chunks, CTAS_PER_SM)), dim3(THREADS), 0, L.st, tab, p) != cudaSuccess) return DFLASH_ERR_CUDA;
        p.norm_out = nullptr;
        g_launches += 1;
    }
    return DFLASH_OK;
}

}  // namespace

int64_t adamw_workspace_bytes(int sm_count, int n_tensors) {
    const int64_t launches = std::max(1, (n_tensors + MAX_TENSORS - 1) / MAX_TENSORS);
    return align_up(launches * sm_count * NORM_CTAS_PER_SM * (int64_t)sizeof(double), 256);
}

int launch_adamw(const Launch& L, const dflash_adamw_args& a) {
    return a.n_tensors <= FEW_TENSORS ? launch_tables<FEW_TENSORS>(L, a) : launch_tables<MAX_TENSORS>(L, a);
}

}  // namespace dflash
