// Gradient of the values before the activation, dz = dy * act'(pre), and the bias gradient: the sum of dz over the tokens.
//
// Bound by memory: dy and pre are read once, dz is written once; the column sums ride along in registers.  A work-group
// owns 512 columns of grad_rows() tokens, its four wavefronts every fourth token; sums meet in LDS, then, one row per
// work-group of tokens, with the products of dx and dw or in a kernel of their own, always in the same order.
// 8192 x 8192 bf16 with gelu, 403 MB: 73 to 77 us between products, 5.2 to 5.5 TB/s (the library's erf: 110); from 8 bits, with 8192 x 4096 of x to bf16 beside it, 435 MB: 85 us.
#include "pad_dev.h"

namespace oz {
namespace {

// Rows first, first + 4, ... of a lane's 8 columns from c on, `n` of them there.  (With a decision on the activation for each value, and loads behind
// decisions, the launch takes 7.9 us instead of 6.0 for 500 x 384 f32, silu, and its copies.)
// FULL: 8 of them in all lanes (8192 x 4096 bf16 from 8 bits, without dz, 36.2 -> 34.6 us, 16384 x 2048 with dz and dx 60.4 -> 59.1).
//
// Whole strips of 16 bits with nothing in 8: as many loads as a compute unit can have on their way at once are more than memory serves well (8192 x 8192,
// where all work-groups are resident), so that a row's dy and pre are asked for in turn.  Of gelu and its tanh form, whose arithmetic is as long as a
// load, the next row's dy comes during it.  dz, and dx of 8 columns, of 8192 x 8192 bf16 with relu 109.5 -> 104.4 us, silu 111.3 -> 105.6, gelu
// 114.0 -> 109.0 (dy in turn, and nothing during the arithmetic: 119.6), gelu_tanh 111.1 -> 107.1; 8192 x 4096 with gelu 60.5 -> 58.2.
//
// dz of operands in 16 bits, x or w of which is held in 8 (SPLIT): dz m[t] n[o] with the m and n of their scales (split_scale), which leaves
// the operands exact and the products' rows to be divided by m[t] (dx) and n[o] (dw).
template <class T, int ACT, bool EIGHT, bool SPLIT, bool FULL>
__device__ __forceinline__ void grad_rows_of(const GradInput &a, long long first, long long last, bool writes_inverse, int c, int n, const float (&factor)[8], float (&sum)[8])
{
    typedef std::conditional_t<EIGHT, int8_t, T> Pre;
    constexpr bool kTurns = FULL && !EIGHT && !SPLIT && sizeof(T) == 2 && ACT != OZIMMU_ACT_NONE;
    constexpr bool kAhead = kTurns && (ACT == OZIMMU_ACT_GELU || ACT == OZIMMU_ACT_GELU_TANH);
    Eight<T> next;
    if (kAhead && first < last) next.load((const T *)a.dy + (size_t)first * a.lddy + c, 8);
    for (long long r = first; r < last; r += 4) {
        Eight<T> dy;
        Eight<Pre> pre;
        float scale = 1.0f, m = 1.0f, d[8];
        if constexpr (kAhead) dy = next;
        else dy.load((const T *)a.dy + (size_t)r * a.lddy + c, FULL ? 8 : n);
        if constexpr (ACT != OZIMMU_ACT_NONE) {
            if constexpr (kTurns && !kAhead) asm volatile("" : "+v"(dy.v));             // (a wait for it)
            pre.load((const Pre *)a.pre + (size_t)r * a.ldpre + c, FULL ? 8 : n);
            if constexpr (EIGHT) scale = a.pre_scale[r];
            if constexpr (kAhead) {
                asm volatile("" : "+v"(pre.v));
                next.load((const T *)a.dy + (size_t)(r + 4 < last ? r + 4 : r) * a.lddy + c, 8);
                asm volatile("" ::: "memory");                                          // (the load stays in front of the arithmetic)
            }
        }
        if (SPLIT && a.x_scale) m = split_scale<T>(a.x_scale[r]).m;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            d[i] = dy[i];
            if constexpr (ACT != OZIMMU_ACT_NONE) d[i] *= activation_slope<T>(ACT, EIGHT ? pre[i] * scale : pre[i]);
            sum[i] += d[i];
            if constexpr (SPLIT) d[i] *= m * factor[i];
        }
        if (SPLIT && a.x_scale && writes_inverse) a.x_inverse[r] = 1.0f / m;
        if (!FULL && n < 8)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= n) d[i] = 0.0f;                    // (0 times an infinite scale is none)
        // (rows of dz are the workspace's, on 16 bytes, zeros behind them)
        if (a.dz) store_row((T *)a.dz + (size_t)r * a.lddz + c, d);
    }
}

template <class T, int ACT, bool EIGHT, bool SPLIT>
__device__ __forceinline__ void grad_input(const GradInput &a, int strip, int group, float (*part)[512])
{
    // (the rows are a wavefront's: their addresses are scalars)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int c = strip * 512 + lane * 8, n = a.n_out - c;
    const long long first = (long long)group * a.rows, last = first + a.rows < a.tokens ? first + a.rows : a.tokens;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, factor[8];
    if constexpr (SPLIT) {
#pragma unroll
        for (int i = 0; i < 8; ++i) factor[i] = a.w_scale && i < n ? a.w_scale[c + i] : 0.0f;       // (0: m = 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            factor[i] = split_scale<T>(factor[i]).m;
            if (a.w_scale && i < n && group == 0 && wave == 0) a.w_inverse[c + i] = 1.0f / factor[i];
        }
    }
    if ((strip + 1LL) * 512 <= a.n_out) grad_rows_of<T, ACT, EIGHT, SPLIT, true>(a, first + wave, last, strip == 0 && lane == 0, c, n, factor, sum);
    else if (n > 0) grad_rows_of<T, ACT, EIGHT, SPLIT, false>(a, first + wave, last, strip == 0 && lane == 0, c, n, factor, sum);
    if (!a.sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[wave][lane * 8 + i] = sum[i];
    __syncthreads();
    for (int i = threadIdx.x; i < 512 && strip * 512 + i < a.n_out; i += 256)
        a.sums[(size_t)group * a.n_out + strip * 512 + i] = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
}

// ... and the copies that the products want, in one launch
template <class T, int ACT, bool EIGHT, bool SPLIT>
__global__ __launch_bounds__(256) void grad_input_kernel(GradInput a, PadCopies copies, int strips, long long blocks)
{
    __shared__ float part[4][512];
    const long long b = (long long)blockIdx.y * kGridRow + blockIdx.x;
    if (b < blocks) grad_input<T, ACT, EIGHT, SPLIT>(a, (int)((unsigned)b % (unsigned)strips), (int)((unsigned)b / (unsigned)strips), part);
    else pad_chunk<T>(copies, (b - blocks) * 256 + threadIdx.x);
}

template <class T>
__global__ __launch_bounds__(256) void bias_grad_kernel(BiasGrad b)
{
    __shared__ float part[256];
    bias_grad<T>(b, (int)(blockIdx.y * kGridRow + blockIdx.x), part);
}

template <class T, bool EIGHT, bool SPLIT>
hipError_t launch_as(const GradInput &g, const PadCopies &copies, int strips, long long blocks, long long all, hipStream_t st)
{
    const dim3 grid(grid_row(all), grid_rows(all));
    switch (g.act) {
        case OZIMMU_ACT_RELU: grad_input_kernel<T, OZIMMU_ACT_RELU, EIGHT, SPLIT><<<grid, 256, 0, st>>>(g, copies, strips, blocks); break;
        case OZIMMU_ACT_GELU: grad_input_kernel<T, OZIMMU_ACT_GELU, EIGHT, SPLIT><<<grid, 256, 0, st>>>(g, copies, strips, blocks); break;
        case OZIMMU_ACT_GELU_TANH: grad_input_kernel<T, OZIMMU_ACT_GELU_TANH, EIGHT, SPLIT><<<grid, 256, 0, st>>>(g, copies, strips, blocks); break;
        case OZIMMU_ACT_SILU: grad_input_kernel<T, OZIMMU_ACT_SILU, EIGHT, SPLIT><<<grid, 256, 0, st>>>(g, copies, strips, blocks); break;
        default: grad_input_kernel<T, OZIMMU_ACT_NONE, false, SPLIT><<<grid, 256, 0, st>>>(g, copies, strips, blocks);
    }
    return hipGetLastError();
}

template <class T>
hipError_t launch(const GradInput &g, const PadCopies &copies, int type, hipStream_t st)
{
    const int strips = (int)((g.n_out + 511LL) / 512);
    const long long blocks = g.dz || g.sums ? (long long)strips * ((g.tokens + (long long)g.rows - 1) / g.rows) : 0, all = blocks + pad_groups(copies, type);
    if (all == 0) return hipSuccess;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    // (scales go into dz in 16 bits only)
    if constexpr (sizeof(T) == 2)
        if (g.x_scale || g.w_scale)
            return g.pre_scale ? launch_as<T, true, true>(g, copies, strips, blocks, all, st) : launch_as<T, false, true>(g, copies, strips, blocks, all, st);
    return g.pre_scale ? launch_as<T, true, false>(g, copies, strips, blocks, all, st) : launch_as<T, false, false>(g, copies, strips, blocks, all, st);
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
