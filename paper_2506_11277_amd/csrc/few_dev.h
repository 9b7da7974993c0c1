// A linear layer on at most 16 tokens: the weight is read once.  16 output features a work-group, its wavefronts take steps of
// the contraction in turn, their sums meet in LDS.  (From 17 tokens on the tiles are the sooner way: 48 x 8192 x 2048 bf16 13 us
// against 20 here, 64 x 2048 x 8192 9.5 against 20; 16 x 4096 x 4096 9.8 here against 12.3, 1 x 1024 x 4096 4.8 against 7.3.)
#pragma once
#include "stream_dev.h"

namespace oz {

constexpr int kFewWaves = 8;

template <class T, class O, int U>
__global__ __launch_bounds__(64 * kFewWaves) void few_tokens_kernel(Product a, float *partial, int steps_per_split)
{
    constexpr int KE = 8 * Chunk<T>::E;
    __shared__ __attribute__((aligned(16))) float sums[kFewWaves][16 * kStreamLd];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int p0 = (int)(blockIdx.z * kGridRow + blockIdx.x) * 16, row = p0 + (lane & 15);
    if (p0 >= a.e.np) return;
    const T *const w[1] = {(const T *)a.P + (size_t)(row < a.e.np ? row : a.e.np - 1) * a.ldp};
    const bool on[1] = {(lane & 15) < a.e.nq};
    const T *const x[1] = {(const T *)a.Q + (size_t)(on[0] ? lane & 15 : 0) * a.ldq};
    v4f acc[1][1] = {{v4f{0, 0, 0, 0}}};
    const int q = threadIdx.x >> 1, c = (threadIdx.x & 1) * 8, p = p0 + c;
    const bool finishes = q < 16 && q < a.e.nq && p < a.e.np;
    RowVectors<O> with;                             // (their loads beside the weight's, not behind the sums)
    if (sizeof(T) == 1 && finishes && !partial) with.load(a.e, q, p);
    const int all = (a.nk + KE - 1) / KE, first = blockIdx.y * steps_per_split, last = all < first + steps_per_split ? all : first + steps_per_split;
    stream_products<T, 1, 1, U>(acc, w, x, on, first + wave, last, kFewWaves, a.nk, lane);
    put_sums(sums[wave], acc[0][0], lane);
    __syncthreads();
    if (!finishes) return;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < kFewWaves; ++s) {
        const float *from = &sums[s][q * kStreamLd + c];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = add_sums<T>(v[e], from[e]);
    }
    if (partial) store_row(partial + ((size_t)blockIdx.y * a.e.nq + q) * ((a.e.np + 7) & ~7) + p, v);
    else if constexpr (sizeof(T) == 1) finish_row<T, O>(a.e, q, p, v, with);
    else finish_row<T, O>(a.e, q, p, v);
}

template <class T, class O = T>
hipError_t launch_few_tokens(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    const int groups = (a.e.np + 15) / 16;
    const dim3 grid(grid_row(groups), plan.splits, grid_rows(groups));
    float *const to = plan.splits > 1 ? partial : nullptr;
    // (steps whose loads a wavefront issues together: no more than it has; in 8 bits 1 x 1024 -> 4096 has one, which with the scales' loads
    // beside it takes 4.2 us on weights from memory, 5.1 with both behind one another)
    if (sizeof(T) == 1 && plan.steps <= kFewWaves) few_tokens_kernel<T, O, 1><<<grid, 64 * kFewWaves, 0, st>>>(a, to, plan.steps);
    else if (plan.steps > 2 * kFewWaves) few_tokens_kernel<T, O, 4><<<grid, 64 * kFewWaves, 0, st>>>(a, to, plan.steps);
    else few_tokens_kernel<T, O, 2><<<grid, 64 * kFewWaves, 0, st>>>(a, to, plan.steps);
    return hipGetLastError();
}

}  // namespace oz
