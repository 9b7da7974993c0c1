// Gradient of the values before the activation, dz = dy * act'(pre), and the bias gradient: the sum of dz over the tokens.
//
// Bound by memory: dy and pre are read once, dz is written once; the column sums ride along in registers.  A work-group
// owns 512 columns of grad_rows() tokens, its four wavefronts every fourth token; sums meet in LDS, then, one row per
// work-group of tokens, with the products of dx and dw or in a kernel of their own, always in the same order.
// 8192 x 8192 bf16 with gelu, 403 MB: 74 us, 5.4 TB/s (the library's erf: 110).
#include "layers.h"

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

template <class T>
__global__ __launch_bounds__(256) void grad_input_kernel(GradInput a)
{
    __shared__ float part[4][512];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int c = blockIdx.x * 512 + lane * 8, n = a.n_out - c;
    const int first = blockIdx.y * a.rows, last = first + a.rows < a.tokens ? first + a.rows : a.tokens;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (n > 0)
#pragma unroll 2
        for (int r = first + wave; r < last; r += 4) {
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
                T *to = (T *)a.dz + (size_t)r * a.lddz + c;
                store_row(to, d);                           // (rows of dz are the workspace's, on 16 bytes, zeros behind them)
            }
        }
    if (!a.sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[wave][lane * 8 + i] = sum[i];
    __syncthreads();
    for (int i = threadIdx.x; i < 512 && blockIdx.x * 512 + i < a.n_out; i += 256)
        a.sums[(size_t)blockIdx.y * a.n_out + blockIdx.x * 512 + i] = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
}

template <class T>
__global__ __launch_bounds__(256) void bias_grad_kernel(BiasGrad b)
{
    __shared__ float part[256];
    bias_grad<T>(b, (int)(blockIdx.y * kGridRow + blockIdx.x), part);
}

template <class T>
hipError_t launch(const GradInput &g, hipStream_t st)
{
    const int groups = (g.tokens + g.rows - 1) / g.rows;
    if (groups == 0) return hipSuccess;
    if (groups > 65535) return hipErrorInvalidValue;
    grad_input_kernel<T><<<dim3((g.n_out + 511) / 512, groups), 256, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_grad_input(const GradInput &g, int type, hipStream_t st)
{
    return type == OZIMMU_BF16 ? launch<bf16>(g, st) : type == OZIMMU_F16 ? launch<f16>(g, st) : launch<float>(g, st);
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
