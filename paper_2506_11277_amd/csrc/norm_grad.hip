// Gradients of the root-mean-square norm y = h r w, r = 1 / sqrt(mean of h^2 + eps): with g = dy w and n = h r
//   dx = r (g - n mean(g n)) + add,   dw = the sum of dy n over the tokens.
//
// Bound by memory: a work-group takes one row after the other, its values in registers, so that they are read once; the
// sums of dw stay in registers from row to row, and leave them as one row of partial sums for each work-group, which a
// second kernel adds up, always in the same order.  Rows beyond what registers hold are read twice, and dw is summed
// by columns in a pass of its own.
// 8192 x 8192 bf16 with `add`: 98 us for the rows (5.5 TB/s) and 4.9 for the partial sums, where a copy of as many bytes
// takes 110; 7863 x 24 f32: 11 us, of which the two launches are nearly all.
#include "norm_dev.h"

namespace oz {
namespace {

struct TwoSums {
    float a, b;
};
template <int L>
__device__ __forceinline__ TwoSums sums_over_row(float a, float b, TwoSums *slots)
{
    a = lanes_sum(a);
    b = lanes_sum(b);
    if constexpr (L > 64) {
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = TwoSums{a, b};
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < L / 64; ++w) {
            const TwoSums s = slots[w];
            a += s.a;
            b += s.b;
        }
    }
    return TwoSums{a, b};
}

// what a row's gradients need of it: r, and mean(g n) r; of h 2^-80 where `factor` is 2^-80
struct RowGrad {
    float r, mean, factor;
};
__device__ __forceinline__ RowGrad row_grad(float mean, const TwoSums &s, int width, float factor)
{
    const float r = inverse_root(mean);
    return RowGrad{r, s.b * r / (float)width, factor};
}
// (r of h itself is r factor; g and n are of ordinary size, whatever h is)
__device__ __forceinline__ float input_grad(const RowGrad &s, float h, float g)
{
    const float n = h * s.factor * s.r;
    return (g - n * s.mean) * (s.r * s.factor);
}

// SHORT: rows of less than 8 values, and of 32 bits for 1024 threads, which have no registers for more.  Rows of up to 2048 values: the next one
// is on its way while one's gradients are formed (40000 x 800 bf16 66 -> 51 us, 30000 x 1500 82 -> 77, 20000 x 512 24 -> 20; of 8192 values that
// takes the registers of a second work-group, 107 -> 112).
template <class T, int L, int C, bool ADD, bool SHORT>
__global__ __launch_bounds__(L < 256 ? 256 : L) void norm_grad_kernel(NormGradArgs a)
{
    constexpr int ROWS = L < 256 ? 256 / L : 1;
    __shared__ TwoSums slots[3][L / 64];
    __shared__ float part[L < 256 ? 256 * 8 : 1];
    const int t = L < 256 ? threadIdx.x & (L - 1) : threadIdx.x, which = L < 256 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L) : 0;
    float dw[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[c][i] = 0.0f;
    Eight<T> rw[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * L + t) * 8;
        if (a.weight) rw[c].load((const T *)a.weight + at, a.width - at);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) rw[c].v[i] = (T)1.0f;
    }
    struct Row {
        Eight<T> h[C], d[C], add[ADD ? C : 1];
    };
    auto load = [&](Row &x, long long row) __attribute__((always_inline)) {
        const T *h = (const T *)a.h + (size_t)row * a.ldh, *d = (const T *)a.dy + (size_t)row * a.lddy, *add = (const T *)a.add + (size_t)row * a.ldadd;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * L + t) * 8;
            if constexpr (SHORT) {
                x.h[c].load(h + at, a.width - at);
                x.d[c].load(d + at, a.width - at);
                if constexpr (ADD) x.add[c].load(add + at, a.width - at);
            } else {
                load_to_end(x.h[c], h, at, a.width);
                load_to_end(x.d[c], d, at, a.width);
                if constexpr (ADD) load_to_end(x.add[c], add, at, a.width);
            }
        }
    };
    constexpr bool kAhead = L * C <= 256;
    int turn = 0;
    auto gradients = [&](Row &x, long long row) __attribute__((always_inline)) {
        if constexpr (!SHORT)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int at = (c * L + t) * 8;
                ends(x.h[c], at, a.width);
                ends(x.d[c], at, a.width);
                if constexpr (ADD) ends(x.add[c], at, a.width);
            }
        auto statistics = [&](float factor, TwoSums *to) __attribute__((always_inline)) {
            float squares = 0.0f, products = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float h = x.h[c][i] * factor;
                    squares = __builtin_fmaf(h, h, squares);
                    products = __builtin_fmaf(x.d[c][i] * rw[c][i], h, products);
                }
            return sums_over_row<L>(squares, products, to);
        };
        // (two sets of slots in turn: a row's are read before anyone is behind the next row's barrier)
        RowGrad s;
        const TwoSums first = statistics(1.0f, slots[turn]);
        const float mean = mean_of(first.a, a.width, a.eps);
        if (__builtin_expect(in_range(mean), 1)) {
            s = row_grad(mean, first, a.width, 1.0f);
        } else {
            if constexpr (L > 64) __syncthreads();
            const TwoSums second = statistics(kSmaller, slots[2]);
            s = row_grad(mean_of(second.a, a.width, a.eps, kSmaller), second, a.width, kSmaller);
            if constexpr (L > 64) __syncthreads();
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * L + t) * 8;
            float dx[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = x.d[c][i], h = x.h[c][i];
                dx[i] = input_grad(s, h, d * rw[c][i]);
                if constexpr (ADD) dx[i] += x.add[c][i];
                dw[c][i] = __builtin_fmaf(d, h * s.factor * s.r, dw[c][i]);
            }
            if (a.dx) store8((T *)a.dx + (size_t)row * a.lddx + at, a.width - at, dx);
        }
        turn ^= 1;
    };
    const long long step = (long long)gridDim.x * ROWS;
    long long row = (long long)blockIdx.x * ROWS + which;
    if (row < a.rows) {
        if constexpr (kAhead) {
            Row x, next;
            load(x, row);
            for (; row + step < a.rows; row += step) {
                load(next, row + step);
                gradients(x, row);
                x = next;
            }
            gradients(x, row);
        } else {
            for (; row < a.rows; row += step) {
                Row x;
                load(x, row);
                gradients(x, row);
            }
        }
    }
    if (!a.sums) return;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * L + t) * 8;
        if constexpr (L < 256) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) part[(which * L + t) * 8 + i] = dw[c][i];
            __syncthreads();
            if (which == 0)
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int q = 1; q < ROWS; ++q) dw[c][i] += part[(q * L + t) * 8 + i];
        }
        if (which == 0) store8(a.sums + (size_t)blockIdx.x * a.width + at, a.width - at, dw[c]);
    }
}

// Rows of any width: dx, and for the sums by columns r and the factor that h is taken with.
template <class T>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormGradArgs a)
{
    constexpr int L = 1024;
    __shared__ TwoSums slots[2][L / 64];
    const long long row = (long long)blockIdx.y * kGridRow1024 + blockIdx.x;
    if (row >= a.rows) return;
    const T *hs = (const T *)a.h + (size_t)row * a.ldh, *ds = (const T *)a.dy + (size_t)row * a.lddy, *w = (const T *)a.weight;
    const T *add = a.add ? (const T *)a.add + (size_t)row * a.ldadd : nullptr;
    auto values = [&](int at, float (&h)[8], float (&g)[8]) __attribute__((always_inline)) {
        Eight<T> rh, rd, rw;
        rh.load(hs + at, a.width - at);
        rd.load(ds + at, a.width - at);
        if (w) rw.load(w + at, a.width - at);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[i] = rh[i];
            g[i] = w ? rd[i] * rw[i] : rd[i];
        }
    };
    auto statistics = [&](float factor, TwoSums *to) __attribute__((always_inline)) {
        float squares = 0.0f, products = 0.0f;
        for (int at = threadIdx.x * 8; at < a.width; at += L * 8) {
            float h[8], g[8], a = 0.0f, b = 0.0f;
            values(at, h, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = h[i] * factor;
                a = __builtin_fmaf(v, v, a);
                b = __builtin_fmaf(g[i], v, b);
            }
            squares += a;
            products += b;
        }
        return sums_over_row<L>(squares, products, to);
    };
    RowGrad s;
    const TwoSums first = statistics(1.0f, slots[0]);
    const float mean = mean_of(first.a, a.width, a.eps);
    if (in_range(mean)) {
        s = row_grad(mean, first, a.width, 1.0f);
    } else {
        const TwoSums second = statistics(kSmaller, slots[1]);
        s = row_grad(mean_of(second.a, a.width, a.eps, kSmaller), second, a.width, kSmaller);
    }
    if (a.dx)
        for (int at = threadIdx.x * 8; at < a.width; at += L * 8) {
            float h[8], g[8];
            values(at, h, g);
            Eight<T> ra;
            if (add) ra.load(add + at, a.width - at);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[i] = input_grad(s, h[i], g[i]);
                if (add) h[i] += ra[i];
            }
            store8((T *)a.dx + (size_t)row * a.lddx + at, a.width - at, h);
        }
    if (a.factors && threadIdx.x == 0) ((float2 *)a.factors)[row] = float2{s.r, s.factor};
}

// the sums of dw over `group` tokens, 512 columns a work-group
template <class T>
__global__ __launch_bounds__(256) void norm_grad_columns_kernel(NormGradArgs a, int group)
{
    __shared__ float part[4][512];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c = blockIdx.x * 512 + lane * 8;
    const long long first = (long long)blockIdx.y * group, last = first + group < a.rows ? first + group : a.rows;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (c < a.width)
        for (long long row = first + wave; row < last; row += 4) {
            Eight<T> rh, rd;
            rh.load((const T *)a.h + (size_t)row * a.ldh + c, a.width - c);
            rd.load((const T *)a.dy + (size_t)row * a.lddy + c, a.width - c);
            const float2 f = ((const float2 *)a.factors)[row];
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = __builtin_fmaf(rd[i], rh[i] * f.y * f.x, sum[i]);
        }
#pragma unroll
    for (int i = 0; i < 8; ++i) part[wave][lane * 8 + i] = sum[i];
    __syncthreads();
    for (int i = threadIdx.x; i < 512; i += 256) {
        const long long col = (long long)blockIdx.x * 512 + i;
        if (col < a.width) a.sums[(size_t)blockIdx.y * a.width + col] = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
    }
}

// dw: the partial sums' rows, 32 columns a work-group, half a wavefront every 32nd row
constexpr int kJoinColumns = 32;
template <class T>
__global__ __launch_bounds__(1024) void norm_grad_join_kernel(const float *sums, T *dw, int rows, int width)
{
    __shared__ float part[32][kJoinColumns];
    const int group = threadIdx.x / kJoinColumns, t = threadIdx.x % kJoinColumns;
    const long long c = ((long long)blockIdx.y * kGridRow1024 + blockIdx.x) * kJoinColumns + t;
    float s = 0.0f;
    if (c < width)
#pragma unroll 8
        for (int r = group; r < rows; r += 32) s += sums[(size_t)r * width + c];
    part[group][t] = s;
    __syncthreads();
    if (group == 0 && c < width) {
#pragma unroll
        for (int g = 1; g < 32; ++g) s += part[g][t];
        dw[c] = (T)s;
    }
}

template <class T, int L, int C>
hipError_t launch_rows(const NormGradArgs &a, int groups, hipStream_t st)
{
    constexpr int threads = L < 256 ? 256 : L;
    constexpr bool tight = L == 1024 && sizeof(T) == 4;
    if constexpr (L * C == 64) {
        if (a.width < 8) {
            if (a.add) norm_grad_kernel<T, L, C, true, true><<<groups, threads, 0, st>>>(a);
            else norm_grad_kernel<T, L, C, false, true><<<groups, threads, 0, st>>>(a);
            return hipGetLastError();
        }
    }
    if (a.add) norm_grad_kernel<T, L, C, true, tight><<<groups, threads, 0, st>>>(a);
    else norm_grad_kernel<T, L, C, false, tight><<<groups, threads, 0, st>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t launch(const NormGradArgs &a, hipStream_t st)
{
    const NormGradPlan plan = plan_norm_grad(a.rows, a.width);
    hipError_t e = hipSuccess;
    if (a.rows > 0 && (a.dx || a.sums)) {
        if (plan.in_registers) {
            // (8192 values, bf16: 104 us with 512 threads a row, 107 with 256; 7001 111, 114; 9370 132 with 1024 as with 512)
            e = a.width <= 512    ? launch_rows<T, 64, 1>(a, plan.parts, st)
                : a.width <= 1024 ? launch_rows<T, 64, 2>(a, plan.parts, st)
                : a.width <= 2048 ? launch_rows<T, 256, 1>(a, plan.parts, st)
                : a.width <= 4096 ? launch_rows<T, 256, 2>(a, plan.parts, st)
                : a.width <= 8192 ? launch_rows<T, 512, 2>(a, plan.parts, st)
                                  : launch_rows<T, 1024, 2>(a, plan.parts, st);
        } else {
            // (where dx takes the place of what the columns are summed from, it is formed behind them)
            const dim3 grid(grid_row(a.rows, kGridRow1024), grid_rows(a.rows, kGridRow1024));
            const bool behind = a.sums && a.dx && (a.dx == a.dy || a.dx == a.h);
            NormGradArgs b = a;
            if (behind) b.dx = nullptr;
            norm_grad_long_kernel<T><<<grid, 1024, 0, st>>>(b);
            e = hipGetLastError();
            if (e == hipSuccess && a.sums) {
                norm_grad_columns_kernel<T><<<dim3((unsigned)((a.width + 511LL) / 512), plan.parts), 256, 0, st>>>(a, plan.group);
                e = hipGetLastError();
            }
            if (e == hipSuccess && behind) {
                b = a;
                b.factors = nullptr;
                norm_grad_long_kernel<T><<<grid, 1024, 0, st>>>(b);
                e = hipGetLastError();
            }
        }
    }
    if (e != hipSuccess || !a.dw) return e;
    const long long groups = (a.width + kJoinColumns - 1LL) / kJoinColumns;
    norm_grad_join_kernel<T><<<dim3(grid_row(groups, kGridRow1024), grid_rows(groups, kGridRow1024)), 1024, 0, st>>>(a.sums, (T *)a.dw, a.rows > 0 ? plan.parts : 0, a.width);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_grad(const NormGradArgs &a, int type, hipStream_t st)
{
    return type == OZIMMU_BF16 ? launch<bf16>(a, st) : type == OZIMMU_F16 ? launch<f16>(a, st) : launch<float>(a, st);
}

}  // namespace oz
