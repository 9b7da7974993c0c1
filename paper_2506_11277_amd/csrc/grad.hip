// Gradient of the values before the activation, dz = dy * act'(pre), and the bias gradient: the sum of dz over the tokens.
//
// Bound by memory: dy and pre are read once, dz is written once; the column sums ride along in registers.  A work-group
// owns 512 columns of grad_rows() tokens, its four wavefronts every fourth token; sums meet in LDS, then, one row per
// work-group of tokens, with the products of dx and dw or in a kernel of their own, always in the same order.
// 8192 x 8192 bf16 with gelu, 403 MB: 74 us, 5.4 TB/s (the library's erf: 110).
#include "pad_dev.h"

namespace oz {
namespace {

template <class T>
__device__ __forceinline__ void load8(const T *p, int n, bool wide, float (&v)[8])
{
    if (wide && n >= 8) {
        load_row(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
    }
}

// ... held in 8 bits, with their row's scale
__device__ __forceinline__ void load8(const int8_t *p, int n, float scale, float (&v)[8])
{
    if (n >= 8) {
        typedef int8_t V __attribute__((ext_vector_type(8)));
        V x;
        __builtin_memcpy(&x, p, 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)x[i] * scale;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] * scale : 0.0f;
    }
}

// dz of operands in 16 bits, x or w of which is held in 8: dz m[t] n[o] with the m and n of their scales' (split_scale), which leaves
// the operands exact and the products' rows to be divided by m[t] (dx) and n[o] (dw).
template <class T>
__device__ __forceinline__ void grad_input(const GradInput &a, int strip, int group, float (*part)[512])
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int c = strip * 512 + lane * 8, n = a.n_out - c;
    const long long first = (long long)group * a.rows, last = first + a.rows < a.tokens ? first + a.rows : a.tokens;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, factor[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        factor[i] = 1.0f;
        if (a.w_scale && i < n) {
            factor[i] = split_scale(a.w_scale[c + i]).m;
            if (group == 0 && wave == 0) a.w_inverse[c + i] = 1.0f / factor[i];
        }
    }
    if (n > 0)
#pragma unroll 2
        for (long long r = first + wave; r < last; r += 4) {
            float d[8], z[8];
            load8((const T *)a.dy + (size_t)r * a.lddy + c, n, a.wide, d);
            if (a.act) {
                if (a.pre_scale) load8((const int8_t *)a.pre + (size_t)r * a.ldpre + c, n, a.pre_scale[r], z);
                else load8((const T *)a.pre + (size_t)r * a.ldpre + c, n, a.wide, z);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] *= activation_slope<T>(a.act, z[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += d[i];
            if (a.dz) {
                if (a.x_scale) {
                    const float m = split_scale(a.x_scale[r]).m;
                    if (strip == 0 && lane == 0) a.x_inverse[r] = 1.0f / m;
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] *= m * factor[i];
                } else if (a.w_scale) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] *= factor[i];
                }
                T *to = (T *)a.dz + (size_t)r * a.lddz + c;
                store_row(to, d);                           // (rows of dz are the workspace's, on 16 bytes, zeros behind them)
            }
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
    if (b < blocks) grad_input<T>(a, (int)(b % strips), (int)(b / strips), part);
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
