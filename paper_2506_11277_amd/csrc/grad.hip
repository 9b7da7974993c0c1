// Gradient of the values before the activation, dz = dy * act'(pre), and the bias gradient: the sum of dz over the tokens.
//
// Bound by memory: dy and pre are read once, dz is written once; the column sums ride along in registers.  A work-group
// owns 512 columns of grad_rows() tokens, its four wavefronts every fourth token; sums meet in LDS, then, one row per
// work-group of tokens, with the products of dx and dw or in a kernel of their own, always in the same order.
// 8192 x 8192 bf16 with gelu, 403 MB: 74 us, 5.4 TB/s (the library's erf: 110).
#include "norm_dev.h"
#include "pad_dev.h"

namespace oz {
namespace {

// Rows first + wave, ... of a work-group's columns.  (ACT and EIGHT decided once: with a decision for each value, and loads behind decisions, the launch
// takes 7.9 us instead of 5.5 for 500 x 384 f32, silu, and its copies.)
//
// dz of operands in 16 bits, x or w of which is held in 8: dz m[t] n[o] with the m and n of their scales (split_scale), which leaves
// the operands exact and the products' rows to be divided by m[t] (dx) and n[o] (dw).
template <class T, int ACT, bool EIGHT>
__device__ __forceinline__ void grad_rows_of(const GradInput &a, long long first, long long last, bool first_strip, int lane, int c, int n, const float (&factor)[8], float (&sum)[8])
{
    constexpr int R = 2;
    for (long long r0 = first; r0 < last; r0 += 4 * R) {
        // (as they are in memory: as floats they would leave fewer wavefronts a SIMD)
        Eight<T> dy[R];
        Eight<std::conditional_t<EIGHT, int8_t, T>> pre[R];
        float m[R], z_scale[R];
#pragma unroll
        for (int y = 0; y < R; ++y) {
            const long long r = r0 + 4 * y < last ? r0 + 4 * y : r0;
            dy[y].load((const T *)a.dy + (size_t)r * a.lddy + c, n);
            if constexpr (ACT != OZIMMU_ACT_NONE) {
                pre[y].load((const std::conditional_t<EIGHT, int8_t, T> *)a.pre + (size_t)r * a.ldpre + c, n);
                if constexpr (EIGHT) z_scale[y] = a.pre_scale[r];
            }
            m[y] = a.x_scale ? a.x_scale[r] : 1.0f;
        }
#pragma unroll
        for (int y = 0; y < R; ++y) {
            const long long r = r0 + 4 * y;
            if (r >= last) break;
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] = dy[y][i];
                if constexpr (ACT != OZIMMU_ACT_NONE) d[i] *= activation_slope<T>(ACT, EIGHT ? pre[y][i] * z_scale[y] : pre[y][i]);
                sum[i] += d[i];
            }
            if (!a.dz) continue;
            if (a.x_scale) {
                const float f = split_scale(m[y]).m;
                if (first_strip && lane == 0) a.x_inverse[r] = 1.0f / f;
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] *= f * factor[i];
            } else if (a.w_scale) {
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] *= factor[i];
            }
            T *to = (T *)a.dz + (size_t)r * a.lddz + c;
            store_row(to, d);                            // (rows of dz are the workspace's, on 16 bytes, zeros behind them)
        }
    }
}

template <class T, bool EIGHT>
__device__ __forceinline__ void grad_rows_as(const GradInput &a, long long first, long long last, bool first_strip, int lane, int c, int n, const float (&factor)[8], float (&sum)[8])
{
    switch (a.act) {
        case OZIMMU_ACT_RELU: return grad_rows_of<T, OZIMMU_ACT_RELU, EIGHT>(a, first, last, first_strip, lane, c, n, factor, sum);
        case OZIMMU_ACT_GELU: return grad_rows_of<T, OZIMMU_ACT_GELU, EIGHT>(a, first, last, first_strip, lane, c, n, factor, sum);
        case OZIMMU_ACT_GELU_TANH: return grad_rows_of<T, OZIMMU_ACT_GELU_TANH, EIGHT>(a, first, last, first_strip, lane, c, n, factor, sum);
        case OZIMMU_ACT_SILU: return grad_rows_of<T, OZIMMU_ACT_SILU, EIGHT>(a, first, last, first_strip, lane, c, n, factor, sum);
    }
    grad_rows_of<T, OZIMMU_ACT_NONE, EIGHT>(a, first, last, first_strip, lane, c, n, factor, sum);
}

template <class T>
__device__ __forceinline__ void grad_input(const GradInput &a, int strip, int group, float (*part)[512])
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int c = strip * 512 + lane * 8, n = a.n_out - c;
    const long long first = (long long)group * a.rows, last = first + a.rows < a.tokens ? first + a.rows : a.tokens;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, factor[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) factor[i] = a.w_scale && i < n ? a.w_scale[c + i] : 1.0f;
    if (a.w_scale)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            factor[i] = split_scale(factor[i]).m;
            if (i < n && group == 0 && wave == 0) a.w_inverse[c + i] = 1.0f / factor[i];
        }
    if (n > 0) {
        if (a.pre_scale) grad_rows_as<T, true>(a, first + wave, last, strip == 0, lane, c, n, factor, sum);
        else grad_rows_as<T, false>(a, first + wave, last, strip == 0, lane, c, n, factor, sum);
    }
    if (!a.sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[wave][lane * 8 + i] = sum[i];
    __syncthreads();
    for (int i = threadIdx.x; i < 512 && strip * 512 + i < a.n_out; i += 256)
        a.sums[(size_t)group * a.n_out + strip * 512 + i] = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
}

// ... and the copies that the products want, in one launch
template <class T>
__global__ __launch_bounds__(256) void grad_input_kernel(GradInput a, PadCopies copies, int strips, long long blocks)
{
    __shared__ float part[4][512];
    const long long b = (long long)blockIdx.y * kGridRow + blockIdx.x;
    if (b < blocks) grad_input<T>(a, (int)((unsigned)b % (unsigned)strips), (int)((unsigned)b / (unsigned)strips), part);
    else pad_chunk<T>(copies, (b - blocks) * 256 + threadIdx.x);
}

template <class T>
__global__ __launch_bounds__(256) void bias_grad_kernel(BiasGrad b)
{
    __shared__ float part[256];
    bias_grad<T>(b, (int)(blockIdx.y * kGridRow + blockIdx.x), part);
}

template <class T>
hipError_t launch(const GradInput &g, const PadCopies &copies, int type, hipStream_t st)
{
    const int strips = (int)((g.n_out + 511LL) / 512);
    const long long blocks = g.dz || g.sums ? (long long)strips * ((g.tokens + (long long)g.rows - 1) / g.rows) : 0, all = blocks + pad_groups(copies, type);
    if (all == 0) return hipSuccess;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    grad_input_kernel<T><<<dim3(grid_row(all), grid_rows(all)), 256, 0, st>>>(g, copies, strips, blocks);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_grad_input(const GradInput &g, const PadCopies &copies, int type, hipStream_t st)
{
    return type == OZIMMU_BF16 ? launch<bf16>(g, copies, type, st) : type == OZIMMU_F16 ? launch<f16>(g, copies, type, st) : launch<float>(g, copies, type, st);
}

hipError_t launch_bias_grad(const BiasGrad &b, int type, hipStream_t st)
{
    const int blocks = bias_grad_blocks(b);
    if (blocks == 0) return hipSuccess;
    const dim3 grid(grid_row(blocks), grid_rows(blocks));
    if (type == OZIMMU_BF16) bias_grad_kernel<bf16><<<grid, 256, 0, st>>>(b);
    else if (type == OZIMMU_F16) bias_grad_kernel<f16><<<grid, 256, 0, st>>>(b);
    else bias_grad_kernel<float><<<grid, 256, 0, st>>>(b);
    return hipGetLastError();
}

}  // namespace oz
