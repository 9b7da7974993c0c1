// Root-mean-square norm of rows, with the residual's addition in front of it and its results in 8 bits behind it:
//   h = x + residual,   y = h r w,   r = 1 / sqrt(mean of h^2 + eps),
// and rows to 8 bits by themselves.  A row's factor r only scales it, so its codes are those of t = h w, and r goes into the scale.
//
// Bound by memory: every value is read once, into registers, and written once.  A row is a wavefront's (no barriers) or
// a work-group's, C groups of 8 values a thread; rows beyond the largest of these are read twice, in a loop.
// 8192 x 8192 bf16 with a residual to 8 bits: 82 us, 16384 x 4096 80 (5.9 TB/s; a copy of as many bytes takes 96); to 8 bits alone: 36 us, of a copy's 41 (30 to 32 where x is in the last-level cache);
// one row of 4096: 2.4 us on the device, a launch and one trip to memory (2.7 on operands that no cache holds).
// h^2 that leaves the range: h 2^-80 and r 2^80 take their places (a product with a power of two is exact).
#include "norm_dev.h"

namespace oz {
namespace {

// SHORT: rows of less than 8 values
template <class T, int L, int C, bool SHORT>
__global__ __launch_bounds__(L < 256 ? 256 : L) void norm_kernel(NormArgs a)
{
    constexpr int ROWS = L < 256 ? 256 / L : 1;
    __shared__ SumAndTop slots[2][L / 64];
    const int t = L < 256 ? threadIdx.x & (L - 1) : threadIdx.x;
    const long long row = ((long long)blockIdx.y * (L > 512 ? kGridRow1024 : kGridRow) + blockIdx.x) * ROWS + (L < 256 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L) : 0);
    if (row >= a.rows) return;
    const T *x = (const T *)a.x + (size_t)row * a.ldx, *res = a.residual ? (const T *)a.residual + (size_t)row * a.ldr : nullptr;
    const T *w = (const T *)a.weight;

    // (all loads before the first store, which may be to the residual's place)
    auto load = [&](Eight<T> &v, const T *from, int at) __attribute__((always_inline)) {
        if constexpr (SHORT) v.load(from + at, a.width - at);
        else load_to_end(v, from, at, a.width);
    };
    auto end = [&](Eight<T> &v, int at) __attribute__((always_inline)) {
        if constexpr (!SHORT) ends(v, at, a.width);
    };
    Eight<T> rx[C], rr[C], rw[C];
#pragma unroll
    for (int c = 0; c < C; ++c) load(rx[c], x, (c * L + t) * 8);
    if (res)
#pragma unroll
        for (int c = 0; c < C; ++c) load(rr[c], res, (c * L + t) * 8);
    if (w)
#pragma unroll
        for (int c = 0; c < C; ++c) load(rw[c], w, (c * L + t) * 8);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * L + t) * 8;
        end(rx[c], at);
        if (res) end(rr[c], at);
        if (w) end(rw[c], at);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) rw[c].v[i] = (T)1.0f;
    }
    float h[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) h[c][i] = rx[c][i];
    if (res)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) h[c][i] += rr[c][i];
    if (a.total)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * L + t) * 8;
            store8((T *)a.total + (size_t)row * a.ldt + at, a.width - at, h[c]);
        }

    auto statistics = [&](SumAndTop *to) __attribute__((always_inline)) {
        float sum = 0.0f;
        unsigned top = 0;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum = __builtin_fmaf(h[c][i], h[c][i], sum);
                const unsigned m = magnitude(h[c][i] * rw[c][i]);
                top = m > top ? m : top;
            }
        return over_row<L>(sum, top, to);
    };
    SumAndTop s = statistics(slots[0]);
    float r = 1.0f;
    if (a.norm) {
        float mean = mean_of(s.sum, a.width, a.eps);
        if (__builtin_expect(!in_range(mean), 0)) {                             // (the same for the whole row)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) h[c][i] *= kSmaller;
            s = statistics(slots[1]);
            mean = mean_of(s.sum, a.width, a.eps, kSmaller);
        }
        r = inverse_root(mean);
    }
    const RowScale scale = row_scale(s.top);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * L + t) * 8;
        float p[8];
        if (a.codes) {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = h[c][i] * rw[c][i];
            store_codes(a.codes + (size_t)row * a.ldc + at, a.width - at, p, scale);
        }
        if (a.y) {                                              // (h r first: h w may leave the range)
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = h[c][i] * r * rw[c][i];
            store8((T *)a.y + (size_t)row * a.ldy + at, a.width - at, p);
        }
    }
    if (a.scale && t == 0) a.scale[row] = scale.scale == 0.0f ? 0.0f : scale.scale * r;         // (no values: r is no number)
}

// ... of any width, its values read twice: once for the statistics and once for the results.
// (Where the sum of the squares leaves the range they are read three times.)
template <class T>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a)
{
    constexpr int L = 1024;
    __shared__ SumAndTop slots[2][L / 64];
    const long long row = (long long)blockIdx.y * kGridRow1024 + blockIdx.x;
    if (row >= a.rows) return;
    const T *x = (const T *)a.x + (size_t)row * a.ldx, *res = a.residual ? (const T *)a.residual + (size_t)row * a.ldr : nullptr;
    const T *w = (const T *)a.weight;
    auto values = [&](int at, float (&h)[8], Eight<T> &rw) __attribute__((always_inline)) {
        Eight<T> rx, rr;
        rx.load(x + at, a.width - at);
        if (res) rr.load(res + at, a.width - at);
        if (w) rw.load(w + at, a.width - at);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[i] = res ? rx[i] + rr[i] : rx[i];
            if (!w) rw.v[i] = (T)1.0f;
        }
    };
    auto statistics = [&](SumAndTop *to, float factor) __attribute__((always_inline)) {
        float sum = 0.0f;
        unsigned top = 0;
        for (int at = threadIdx.x * 8; at < a.width; at += L * 8) {
            float h[8], part = 0.0f;
            Eight<T> rw;
            values(at, h, rw);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = h[i] * factor;
                part = __builtin_fmaf(v, v, part);
                const unsigned m = magnitude(v * rw[i]);
                top = m > top ? m : top;
            }
            sum += part;
        }
        return over_row<L>(sum, top, to);
    };
    SumAndTop s = statistics(slots[0], 1.0f);
    float r = 1.0f, factor = 1.0f;
    if (a.norm) {
        float mean = mean_of(s.sum, a.width, a.eps);
        if (!in_range(mean)) {
            factor = kSmaller;
            s = statistics(slots[1], factor);
            mean = mean_of(s.sum, a.width, a.eps, factor);
        }
        r = inverse_root(mean);
    }
    const RowScale scale = row_scale(s.top);
    for (int at = threadIdx.x * 8; at < a.width; at += L * 8) {
        float h[8];
        Eight<T> rw;
        values(at, h, rw);                                      // (this thread's values: what total replaces, it has read)
        if (a.total) store8((T *)a.total + (size_t)row * a.ldt + at, a.width - at, h);
        float p[8];
        if (a.codes) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = h[i] * factor;
                p[i] = v * rw[i];
            }
            store_codes(a.codes + (size_t)row * a.ldc + at, a.width - at, p, scale);
        }
        if (a.y) {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = h[i] * factor * r * rw[i];
            store8((T *)a.y + (size_t)row * a.ldy + at, a.width - at, p);
        }
    }
    if (a.scale && threadIdx.x == 0) a.scale[row] = scale.scale == 0.0f ? 0.0f : scale.scale * r;
}

template <class T, int L, int C>
hipError_t launch_rows(const NormArgs &a, hipStream_t st)
{
    constexpr int ROWS = L < 256 ? 256 / L : 1;
    const long long groups = ((long long)a.rows + ROWS - 1) / ROWS;
    constexpr unsigned line = L > 512 ? kGridRow1024 : kGridRow;
    const dim3 grid(grid_row(groups, line), grid_rows(groups, line));
    if constexpr (L * C == 64)
        if (a.width < 8) {
            norm_kernel<T, L, C, true><<<grid, 256, 0, st>>>(a);
            return hipGetLastError();
        }
    norm_kernel<T, L, C, false><<<grid, L < 256 ? 256 : L, 0, st>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t launch(const NormArgs &a, hipStream_t st)
{
    if (a.rows == 0) return hipSuccess;
    // (Threads a row, bf16.  Where many rows fill the machine, as few as hold it: 30000 x 1500 to 8 bits 58 us by wavefronts, 65 with 256;
    // 16384 x 4096 80 and the norm alone 39 with 256, 81 and 42 with 512.  Fewer rows, more threads: with a residual to 8 bits 1 x 4096 2.4 us with 512, 2.6 with 256, and 256 x 4096 from memory 4.4, 4.8; 64 x 6000
    // 4.7 with 512, 5.8 with 256.  9370 values 86 us with 512, 131 with 1024; 16384 values 84, 98; 30000 values 96 from registers, 114 in two
    // passes; 20000 values 102 either way.)
    if (a.width <= 512) return launch_rows<T, 64, 1>(a, st);
    if (a.width <= 1024) return launch_rows<T, 64, 2>(a, st);
    if (a.width <= 1536 && a.rows >= 2048) return launch_rows<T, 64, 3>(a, st);
    if (a.width <= 2048) return launch_rows<T, 256, 1>(a, st);
    if (a.width <= 4096) return a.rows <= 256 ? launch_rows<T, 512, 1>(a, st) : launch_rows<T, 256, 2>(a, st);
    if (a.width <= 8192) return launch_rows<T, 512, 2>(a, st);
    if (a.width <= 12288) return launch_rows<T, 512, 3>(a, st);
    if (a.width <= 16384) return launch_rows<T, 512, 4>(a, st);
    if (a.width > 24576 && a.width <= 32768) return launch_rows<T, 1024, 4>(a, st);
    norm_long_kernel<T><<<dim3(grid_row(a.rows, kGridRow1024), grid_rows(a.rows, kGridRow1024)), 1024, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs &a, int type, hipStream_t st)
{
    return type == OZIMMU_BF16 ? launch<bf16>(a, st) : type == OZIMMU_F16 ? launch<f16>(a, st) : launch<float>(a, st);
}

}  // namespace oz
