// What the feed-forward operators (ozimmu_layers.h) share: element types, matrix instructions, activations, and the
// epilogue of a product.  HIP only.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ozimmu_layers.h"
#include "gemm_dev.h"

namespace oz {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));

// 16 bytes of elements: what a lane feeds to the matrix instructions per half of a step of 128 bytes of k.
template <class T>
struct Chunk {
    static constexpr int E = 16 / (int)sizeof(T);
    typedef T V __attribute__((ext_vector_type(E)));
};

// c += p q over the k of one chunk per lane.  Operands of 16 bits: one 16x16x32 instruction, lane l holds row l % 16 and
// k 8 (l / 16) ... + 7.  32 bits: four 16x16x4 instructions, lane l's element i standing for k 4 (l / 16) + i; which k an
// instruction takes does not matter as long as both operands agree.  Sums in 32 bits.
// Result: lane l, register i = entry (4 (l / 16) + i, l % 16) of the 16 x 16 block, rows from p, columns from q.
__device__ __forceinline__ v4f mma(v4u p, v4u q, v4f c, bf16)
{
    typedef Chunk<bf16>::V V;
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, p), __builtin_bit_cast(V, q), c, 0, 0, 0);
}
__device__ __forceinline__ v4f mma(v4u p, v4u q, v4f c, f16)
{
    typedef Chunk<f16>::V V;
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, p), __builtin_bit_cast(V, q), c, 0, 0, 0);
}
__device__ __forceinline__ v4f mma(v4u p, v4u q, v4f c, float)
{
    const v4f a = __builtin_bit_cast(v4f, p), b = __builtin_bit_cast(v4f, q);
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

// 16 bytes from an address that is aligned to the element only, `n` elements of them there (the others 0)
template <class T>
__device__ __forceinline__ v4u load_chunk(const T *p, int n)
{
    constexpr int E = Chunk<T>::E;
    union { v4u v; T e[E]; } r;
    if (n >= E) {
        __builtin_memcpy(&r.v, p, 16);
    } else {
        r.v = v4u{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < n) r.e[i] = p[i];
    }
    return r.v;
}

// Activations, in 32 bits.  Operands of 32 bits take the library's exponential, error function and division; those of 16
// bits the instructions for 2^x and 1 / x (two units off at most) and a polynomial, whose errors are a hundredth of the
// rounding that follows: 8192 x 8192 values of an epilogue with the library's erf cost 110 us, so 40.
template <bool FINE>
__device__ __forceinline__ float exp_of(float x)
{
    if constexpr (FINE) return expf(x);
    else return __builtin_amdgcn_exp2f(x * 1.44269504088896f);
}
template <bool FINE>
__device__ __forceinline__ float logistic(float x)
{
    if constexpr (FINE) return 1.0f / (1.0f + expf(-x));
    else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.44269504088896f));
}

// Phi(z) and phi(z) of the normal distribution.  16 bits: Phi(-|z|) = exp(-z^2 / 2) R(|z|), R = exp(z^2 / 2) erfc(z / sqrt 2) / 2
// as a polynomial of t = 1 / (1 + 0.36 |z|) fitted for the least relative error, 9e-7 (so small values keep their digits).
template <bool FINE>
__device__ __forceinline__ void normal(float z, float &Phi, float &phi)
{
    if constexpr (FINE) {
        Phi = 0.5f * erfcf(z * -0.70710678118654752f);
        phi = 0.39894228040143268f * expf(-0.5f * z * z);
    } else {
        const float t = __builtin_amdgcn_rcpf(1.0f + 0.36f * fabsf(z)), e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448f);
        float r = 0.04705653339624405f;
        r = __builtin_fmaf(r, t, -0.179765522480011f);
        r = __builtin_fmaf(r, t, 0.18095506727695465f);
        r = __builtin_fmaf(r, t, 0.026548659428954124f);
        r = __builtin_fmaf(r, t, 0.13971948623657227f);
        r = __builtin_fmaf(r, t, 0.14177241921424866f);
        r = __builtin_fmaf(r, t, 0.14371304214000702f);
        r = r * t * e;
        Phi = z > 0.0f ? 1.0f - r : r;
        phi = 0.39894228040143268f * e;
    }
}

// (gelu_tanh: (1 + tanh u) / 2 = 1 / (1 + exp(-2u)))
template <class T>
__device__ __forceinline__ float activate(int act, float z)
{
    constexpr bool FINE = sizeof(T) == 4;
    switch (act) {
        case OZIMMU_ACT_RELU: return z < 0.0f ? 0.0f : z;               // (a NaN stays one)
        case OZIMMU_ACT_GELU: {
            float Phi, phi;
            normal<FINE>(z, Phi, phi);
            return z * Phi;
        }
        case OZIMMU_ACT_GELU_TANH: return z * logistic<FINE>(1.5957691216057308f * (z + 0.044715f * z * z * z));
        case OZIMMU_ACT_SILU: return z * logistic<FINE>(z);
    }
    return z;
}

// ... and their slopes
template <class T>
__device__ __forceinline__ float activation_slope(int act, float z)
{
    constexpr bool FINE = sizeof(T) == 4;
    switch (act) {
        case OZIMMU_ACT_RELU: return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;
        case OZIMMU_ACT_GELU: {
            float Phi, phi;
            normal<FINE>(z, Phi, phi);
            return Phi + z * phi;
        }
        case OZIMMU_ACT_GELU_TANH: {
            const float s = logistic<FINE>(1.5957691216057308f * (z + 0.044715f * z * z * z));
            const float near = z * s * (1.0f - s) * 2.0f;             // (0 where the square overflows)
            return near == 0.0f ? s : s + near * 0.79788456080286536f * (1.0f + 0.134145f * z * z);
        }
        case OZIMMU_ACT_SILU: {
            const float s = logistic<FINE>(z);
            return s * (1.0f + z * (1.0f - s));
        }
    }
    return 1.0f;
}

// What happens to the sums of a product: y = act(sum + bias) + residual, `pre` = sum + bias.  Entry (q, p) of the result
// stands at out[q * ldo + p]: p runs along the contiguous side.
struct Epilogue {
    const void *bias, *residual;          // may be null
    void *pre, *out;                      // pre may be null
    int ldr, ldpre, ldo;
    int np, nq;
    int act;
    int wide;                             // every row of 8 entries that starts at a multiple of 8 is aligned to its size, up to 16 bytes
};

template <class T, int N>
__device__ __forceinline__ void load_row(const T *p, float (&v)[N])
{
    typedef T V __attribute__((ext_vector_type(N)));
    const V x = *(const V *)p;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)x[i];
}
template <class T, int N>
__device__ __forceinline__ void store_row(T *p, const float (&v)[N])
{
    typedef T V __attribute__((ext_vector_type(N)));
    V x;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (T)v[i];
    *(V *)p = x;
}

// ... past the caches: the results of the largest tiles, which are not read again before they have left them anyway, and leave the L2s to
// the operands (8192 x 4096 x 8192 bf16: dx 396 us with plain stores, 386 so; with gelu and pre 456 and 451)
template <class T, int N>
__device__ __forceinline__ void stream_row(T *p, const float (&v)[N])
{
    typedef T V __attribute__((ext_vector_type(N)));
    V x;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (T)v[i];
    if constexpr (sizeof(V) == 16) {
        __builtin_nontemporal_store(__builtin_bit_cast(v4u, x), (v4u *)p);
    } else {
        typedef T H __attribute__((ext_vector_type(N / 2)));
        __builtin_nontemporal_store(__builtin_bit_cast(v4u, (H)__builtin_shufflevector(x, x, 0, 1, 2, 3)), (v4u *)p);
        __builtin_nontemporal_store(__builtin_bit_cast(v4u, (H)__builtin_shufflevector(x, x, 4, 5, 6, 7)), (v4u *)p + 1);
    }
}

// N = 8 (p a multiple of 8) entries of row q
template <class T>
__device__ __forceinline__ void finish_row(const Epilogue &e, int q, int p, float (&v)[8])
{
    if (e.wide && p + 8 <= e.np) {
        float t[8];
        if (e.bias) {
            load_row((const T *)e.bias + p, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        if (e.pre) store_row((T *)e.pre + (size_t)q * e.ldpre + p, v);
        if (e.act)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = activate<T>(e.act, v[i]);
        if (e.residual) {
            load_row((const T *)e.residual + (size_t)q * e.ldr + p, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        store_row((T *)e.out + (size_t)q * e.ldo + p, v);
    } else {
        float b[8], r[8];                           // (all loads before the first store, which might be to the same place)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool in = p + i < e.np;
            b[i] = in && e.bias ? (float)((const T *)e.bias)[p + i] : 0.0f;
            r[i] = in && e.residual ? (float)((const T *)e.residual)[(size_t)q * e.ldr + p + i] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (p + i >= e.np) continue;
            float x = v[i] + b[i];
            if (e.pre) ((T *)e.pre)[(size_t)q * e.ldpre + p + i] = (T)x;
            x = activate<T>(e.act, x);
            if (e.residual) x += r[i];
            ((T *)e.out)[(size_t)q * e.ldo + p + i] = (T)x;
        }
    }
}

// ---- launchers, one set per element type (product_bf16.hip, product_f16.hip, product_f32.hip)

// D[q][p] = sum over k of P Q.  An operand's rows (p or q) are contiguous along k (`k_rows`), or its entries of one k are
// contiguous along p or q.
struct Product {
    const void *P, *Q;
    int ldp, ldq;
    bool p_k_rows, q_k_rows;
    int nk;
    // what the operands hold: rows (p or q) and k; more than np, nq and nk where they are padded with zeros
    int p_rows, q_rows, p_nk, q_nk;
    Epilogue e;
};

// The bias gradient: column sums of `rows` rows of partial sums.  64 columns a work-group, always in the same order.
struct BiasGrad {
    const float *sums;                    // [rows][n]
    void *db;                             // null: none
    int rows, n;
};
inline int bias_grad_blocks(const BiasGrad &b) { return b.db ? (b.n + 63) / 64 : 0; }
template <class T>
__device__ __forceinline__ void bias_grad(const BiasGrad &b, int block, float *part)    // part: 256 floats of LDS
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = block * 64 + lane;
    float s = 0.0f;
    if (c < b.n)
#pragma unroll 8
        for (int r = wave; r < b.rows; r += 4) s += b.sums[(size_t)r * b.n + c];
    part[threadIdx.x] = s;
    __syncthreads();
    if (wave == 0 && c < b.n) ((T *)b.db)[c] = (T)((part[lane] + part[64 + lane]) + (part[128 + lane] + part[192 + lane]));
}

// HIP takes less than 2^32 work-items along a dimension of a grid: rows of at most kGridRow work-groups (of up to 512; a multiple of
// the XCDs), one behind the other along y or z.
constexpr unsigned kGridRow = 1u << 22;
inline unsigned grid_row(long long groups) { return groups < kGridRow ? (unsigned)groups : kGridRow; }
inline unsigned grid_rows(long long groups) { return (unsigned)((groups + kGridRow - 1) / kGridRow); }

enum Tile { kTile256, kTile128, kTile64, kTileFew };      // edge; few_tokens_kernel
struct ProductPlan {
    int tile;
    int splits, steps;       // the contraction in `splits` parts of `steps` steps of 128 bytes
    bool direct;             // copied to LDS without registers
    double us;               // estimated
};

}  // namespace oz
