// What the kernels over whole rows share (norm.hip, norm_grad.hip): sums and maxima over a row, rows in 8 bits.  Both are bound by memory
// (8192 x 8192 bf16 to 8 bits 36 us, 5.6 TB/s); of a single row's 2.4 us nearly all is the launch and one trip to memory, so one barrier is all they have.
#pragma once
#include "layers.h"

namespace oz {

// f over the 64 lanes' values of a wavefront, the same in each: among 16 by exchanges inside the vector unit
template <class X, class F>
__device__ __forceinline__ X over_lanes(X x, F f)
{
    auto with = [&](unsigned o) { x = f(x, __builtin_bit_cast(X, o)); };
    with(__builtin_amdgcn_mov_dpp(__builtin_bit_cast(unsigned, x), 0xb1, 0xf, 0xf, true));      // lane ^ 1
    with(__builtin_amdgcn_mov_dpp(__builtin_bit_cast(unsigned, x), 0x4e, 0xf, 0xf, true));      // lane ^ 2
    with(__builtin_amdgcn_mov_dpp(__builtin_bit_cast(unsigned, x), 0x141, 0xf, 0xf, true));     // 7 - lane within 8
    with(__builtin_amdgcn_mov_dpp(__builtin_bit_cast(unsigned, x), 0x140, 0xf, 0xf, true));     // 15 - lane within 16
    with(__builtin_amdgcn_ds_swizzle(__builtin_bit_cast(unsigned, x), 0x401f));                 // lane ^ 16
    with(__shfl_xor(__builtin_bit_cast(unsigned, x), 32));
    return x;
}
__device__ __forceinline__ float lanes_sum(float x) { return over_lanes(x, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ unsigned lanes_top(unsigned x) { return over_lanes(x, [](unsigned a, unsigned b) { return a > b ? a : b; }); }

// two sums, or a sum and a maximum, over a row's L threads; `slots`: L / 64 pairs of LDS of this use alone
struct SumAndTop {
    float sum;
    unsigned top;
};
template <int L>
__device__ __forceinline__ SumAndTop over_row(float sum, unsigned top, SumAndTop *slots)
{
    sum = lanes_sum(sum);
    top = lanes_top(top);
    if constexpr (L > 64) {
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = SumAndTop{sum, top};
        __syncthreads();
        sum = 0.0f;
        top = 0;
#pragma unroll
        for (int w = 0; w < L / 64; ++w) {
            const SumAndTop s = slots[w];
            sum += s.sum;
            top = s.top > top ? s.top : top;
        }
    }
    return SumAndTop{sum, top};
}

// 8 values of a row from `at` on, of a row that has 8: at its end the 8 that end there, which ends() moves to their places, with zeros behind
// them.  (No decision stands before the load, behind which
// the next would wait: gradients of 8000 x 7001 bf16 130 -> 114 us, 40000 x 800 74 -> 66.)
template <class T>
__device__ __forceinline__ void load_to_end(Eight<T> &v, const T *row, int at, int width)
{
    __builtin_memcpy(&v.v, row + (at < width - 8 ? at : width - 8), sizeof v.v);
}
template <class T>
__device__ __forceinline__ void ends(Eight<T> &v, int at, int width)
{
    const int over = at - (width - 8);
    if (over <= 0) return;
#pragma unroll
    for (int by = 4; by > 0; by /= 2)
        if (over & by)
#pragma unroll
            for (int i = 0; i < 8; ++i) v.v[i] = i + by < 8 ? v.v[i + by < 8 ? i + by : 0] : (T)0;
    if (over >= 8) v.v = (T)0;
}

// Bits of |x|: ordered as the magnitudes are, infinities and then NaN above all numbers.
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
constexpr unsigned kInfinity = 0x7f800000u;

// A row in 8 bits: code = t (127 / top) rounded to nearest, ties to even, |code| <= 127; scale = top / 127.  127 / top and the product
// with it are rounded in 32 bits, so that the codes follow from t bit by bit.  Rows whose largest magnitude is below 2^-100
// (127 / top might leave the range) are held as zeros; one with a value that is not finite has no scale: NaN.
struct RowScale {
    float inverse, scale;
};
__device__ __forceinline__ RowScale row_scale(unsigned top)
{
    const float t = __uint_as_float(top);
    if (top >= kInfinity) return RowScale{0.0f, __uint_as_float(0x7fc00000u)};
    if (t < 0x1p-100f) return RowScale{0.0f, 0.0f};
    return RowScale{127.0f / t, t * (1.0f / 127.0f)};
}

// |x| < 2^22 rounded to the nearest whole number, in the low bits of a float's 32
__device__ __forceinline__ unsigned whole_bits(float x) { return __float_as_uint(x + 12582912.0f); }

__device__ __forceinline__ void store_codes(int8_t *p, int n, const float (&t)[8], const RowScale &s)
{
    unsigned b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float q = t[i] * s.inverse;                             // (rounded by itself: no fused multiply-add)
        asm("" : "+v"(q));
        b[i] = whole_bits(q);
    }
    if (s.inverse == 0.0f)                                      // (values that are not finite among them)
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = 0;
    v2u c;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        c[i] = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u) | __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x04000c0cu);
    if (n >= 8) {
        __builtin_memcpy(p, &c, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (int8_t)(c[i / 4] >> (8 * (i & 3)));
    }
}

// Where the mean of h^2, or its sum with eps, leaves the range of 32 bits, h times this takes its place, and eps times its square.
constexpr float kSmaller = 0x1p-80f;
// the mean of the squares + eps, of h times `factor`
__device__ __forceinline__ float mean_of(float squares, int width, float eps, float factor = 1.0f)
{
    return squares / (float)width + eps * factor * factor;
}
__device__ __forceinline__ bool in_range(float mean) { return mean < __uint_as_float(kInfinity); }       // (a NaN is not)
__device__ __forceinline__ float inverse_root(float mean) { return 1.0f / sqrtf(mean); }

}  // namespace oz
