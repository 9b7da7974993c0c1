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

// Operands of 8 bits: one 16x16x64 instruction, lane l holds row l % 16 and k 16 (l / 16) ... + 15.  Sums are whole numbers of 32 bits, exact for
// up to 131071 products; where sums of either kind pass through the same places (registers, LDS, memory) they stand there as bits.
__device__ __forceinline__ v4f mma(v4u p, v4u q, v4f c, int8_t)
{
    return __builtin_bit_cast(v4f, __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, p), __builtin_bit_cast(v4i, q), __builtin_bit_cast(v4i, c), 0, 0, 0));
}
// a + b of operands of type T
template <class T>
__device__ __forceinline__ float add_sums(float a, float b)
{
    if constexpr (sizeof(T) == 1) return __int_as_float(__float_as_int(a) + __float_as_int(b));
    else return a + b;
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

// ... of a row whose entries in front of p number `before`: those of 8 bits that end within a chunk are taken with the 16 bytes that end where the row
// does, where it is as long, and moved (sixteen loads of a byte otherwise)
template <class T>
__device__ __forceinline__ v4u load_chunk(const T *p, int n, int before)
{
    if constexpr (sizeof(T) == 1) {
        if (n <= 0) return v4u{0, 0, 0, 0};
        if (before + n >= 16) {
            const int beyond = n < 16 ? 16 - n : 0, shift = 8 * beyond;
            unsigned long long x[2];
            __builtin_memcpy(x, p - beyond, 16);
            if (shift >= 64) {
                x[0] = x[1] >> (shift - 64);
                x[1] = 0;
            } else if (shift > 0) {
                x[0] = (x[0] >> shift) | (x[1] << (64 - shift));
                x[1] >>= shift;
            }
            return v4u{(unsigned)x[0], (unsigned)(x[0] >> 32), (unsigned)x[1], (unsigned)(x[1] >> 32)};
        }
    }
    return load_chunk(p, n);
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

// ... of a product of operands S.  Where these are of 8 bits the product takes half as long, and 67 million gelus of results in 16 bits a quarter
// of its time (8192 x 4096 x 8192: 276 us, 237 without).  There Phi(-|z|) = 2^p(|z|) with one polynomial, fitted for the least error of p up to 5: 4e-6
// of the value up to 4, 1e-5 up to 6, and 6e-7 of y at most; beyond, p runs away to minus infinity, faster than the logarithm, and the value (below
// 6e-9, and below float16's range) is off by up to 1e-13: bfloat16 loses digits from z = -7 on and has none from -9 on.  Keeping them as normal() does takes
// three terms more, or a second polynomial behind a look at each 8 values: 8192 x 256 -> 8192 79 or 78 us instead of 74, 4096 of k 1 % more.
// y = max(z, 0) - |z| Phi(-|z|) (an infinite |z| is taken as a large one, or 0 would have to outweigh it).
template <class S, class T>
__device__ __forceinline__ float activate_sum(int act, float z)
{
    if constexpr (sizeof(S) == 1 && sizeof(T) == 2) {
        if (act == OZIMMU_ACT_GELU) {
            const float x = fabsf(z);
            float p = -1.8195439679402625e-06f;
            p = __builtin_fmaf(p, x, 6.133275019237772e-05f);
            p = __builtin_fmaf(p, x, -0.00092875468544662f);
            p = __builtin_fmaf(p, x, 0.00850219652056694f);
            p = __builtin_fmaf(p, x, -0.053950950503349304f);
            p = __builtin_fmaf(p, x, -0.4584710896015167f);
            p = __builtin_fmaf(p, x, -1.1512492895126343f);
            p = __builtin_fmaf(p, x, -0.9999953508377075f);
            return __builtin_fmaf(-fminf(x, 0x1p100f), __builtin_amdgcn_exp2f(p), fmaxf(z, 0.0f));
        }
    }
    return activate<T>(act, z);
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
    // operands of 8 bits: the rows' scales, sum * q_scale[q] * p_scale[p] takes the sum's place; gradients: sum * q_scale[q], where it is not null
    const float *q_scale, *p_scale;
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

// eight elements, at any alignment of their type; `n` of them there (the others 0)
template <class T>
struct Eight {
    typedef T V __attribute__((ext_vector_type(8)));
    V v;
    __device__ __forceinline__ void load(const T *p, int n)
    {
        if (n >= 8) {
            __builtin_memcpy(&v, p, sizeof v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : (T)0;
        }
    }
    __device__ __forceinline__ float operator[](int i) const { return (float)v[i]; }
};

template <class T>
__device__ __forceinline__ void store8(T *p, int n, const float (&x)[8])
{
    typename Eight<T>::V v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (T)x[i];
    if (n >= 8) {
        __builtin_memcpy(p, &v, sizeof v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = v[i];
    }
}

// The sum of operands of type T, scaled, and the bias: of 8 bits the whole number to the nearest float, its product with the token's scale, and that
// with the feature's together with the bias, each rounded once.
template <class T>
__device__ __forceinline__ float scaled(float sum, float q_scale, float p_scale, float bias)
{
    if constexpr (sizeof(T) == 1) return __builtin_fmaf((float)__float_as_int(sum) * q_scale, p_scale, bias);
    else return sum * q_scale + bias;
}

// What 8 entries of a row want of the scales and the bias (operands of 8 bits): loaded early, or in finish_row
template <class T>
struct RowVectors {
    float x, scale[8], bias[8];
    __device__ __forceinline__ void load(const Epilogue &e, int q, int p)
    {
        x = e.q_scale[q];
        load_columns(e, p);
    }
    __device__ __forceinline__ void load_columns(const Epilogue &e, int p)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) bias[i] = 0.0f;
        if (e.wide && p + 8 <= e.np) {              // (both loads before either's wait)
            load_row(e.p_scale + p, scale);
            if (e.bias) load_row((const T *)e.bias + p, bias);
        } else {
            Eight<float> s;
            Eight<T> b;
            s.load(e.p_scale + p, e.np - p);
            if (e.bias) b.load((const T *)e.bias + p, e.np - p);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                scale[i] = s[i];
                if (e.bias) bias[i] = b[i];
            }
        }
    }
};

// The values before the activation, `pre` and what follows, of N = 8 (p a multiple of 8) entries of row q: sums of operands of type S.
template <class S, class T>
__device__ __forceinline__ void finish_values(const Epilogue &e, int q, int p, float (&v)[8])
{
    if (sizeof(S) == 1 || (e.wide && p + 8 <= e.np)) {
        // (8 entries at any alignment, or what there is of them: of operands of 8 bits; the others take aligned rows only)
        const int n = sizeof(S) == 1 ? e.np - p : 8;
        Eight<T> t;
        if (e.residual) t.load((const T *)e.residual + (size_t)q * e.ldr + p, n);
        if (e.pre) store8((T *)e.pre + (size_t)q * e.ldpre + p, n, v);
        if (e.act)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = activate_sum<S, T>(e.act, v[i]);
        if (e.residual)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        store8((T *)e.out + (size_t)q * e.ldo + p, n, v);
    } else {
        float r[8];                                 // (all loads before the first store, which might be to the same place)
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = p + i < e.np && e.residual ? (float)((const T *)e.residual)[(size_t)q * e.ldr + p + i] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (p + i >= e.np) continue;
            if (e.pre) ((T *)e.pre)[(size_t)q * e.ldpre + p + i] = (T)v[i];
            float z = activate<T>(e.act, v[i]);
            if (e.residual) z += r[i];
            ((T *)e.out)[(size_t)q * e.ldo + p + i] = (T)z;
        }
    }
}

template <class S, class T>
__device__ __forceinline__ void finish_row(const Epilogue &e, int q, int p, float (&v)[8], const RowVectors<T> &with)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = scaled<S>(v[i], with.x, with.scale[i], with.bias[i]);
    finish_values<S, T>(e, q, p, v);
}

// N = 8 (p a multiple of 8) entries of row q: sums of operands of type S, results of type T
template <class S, class T = S>
__device__ __forceinline__ void finish_row(const Epilogue &e, int q, int p, float (&v)[8])
{
    if constexpr (sizeof(S) == 1) {
        RowVectors<T> with;
        with.load(e, q, p);
        finish_row<S, T>(e, q, p, v, with);
        return;
    }
    if (e.q_scale) {
        const float x = e.q_scale[q];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= x;
    }
    if (e.bias) {
        if (e.wide && p + 8 <= e.np) {
            float t[8];
            load_row((const T *)e.bias + p, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (p + i < e.np) v[i] += (float)((const T *)e.bias)[p + i];
        }
    }
    finish_values<S, T>(e, q, p, v);
}

// A scale as m 2^e, 1/2 <= m < 1, and its sign with the power: code * power is exact in 16 bits (8 binary digits; float16: where it is in its range),
// so that of an operand held in 8 bits only m has to go elsewhere: into dz, which with m below 1 stays in its type's range.  (Half of that range was lost with
// each operand in 8 bits where m was 1 to 2.)  The power is 2^8 (bfloat16: 2^120) at most, so that no code's value leaves the range, and m takes the rest of
// larger scales.  Scales that are 0 or not finite stay whole.
struct SplitScale {
    float m, power;
};
template <class T>
__device__ __forceinline__ SplitScale split_scale(float s)
{
    constexpr int kMost = std::is_same_v<T, f16> ? 8 : 120;
    if (s == 0.0f || !(fabsf(s) < __uint_as_float(0x7f800000u))) return SplitScale{1.0f, s};
    const int e = __builtin_amdgcn_frexp_expf(s), over = e > kMost ? e - kMost : 0;
    return SplitScale{__builtin_ldexpf(fabsf(__builtin_amdgcn_frexp_mantf(s)), over), __builtin_ldexpf(s < 0.0f ? -1.0f : 1.0f, e - over)};
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
// the XCDs), one behind the other along y or z; half as many (kGridRow1024) of larger ones.
constexpr unsigned kGridRow = 1u << 22, kGridRow1024 = kGridRow / 2;
inline unsigned grid_row(long long groups, unsigned row = kGridRow) { return groups < row ? (unsigned)groups : row; }
inline unsigned grid_rows(long long groups, unsigned row = kGridRow) { return (unsigned)((groups + row - 1) / row); }

enum Tile { kTile256, kTile128, kTile64, kTileFew, kTile32 };      // edge; few_tokens_kernel; 32 x 64 (both gradients in one launch, 32 bits)
struct ProductPlan {
    int tile;
    int splits, steps;       // the contraction in `splits` parts of `steps` steps of 128 bytes
    bool direct;             // copied to LDS without registers
    double us;               // estimated
};

}  // namespace oz
