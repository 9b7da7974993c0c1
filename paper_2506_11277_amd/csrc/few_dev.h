// A linear layer on at most 64 tokens: the weight is read once.  16 output features a work-group, its wavefronts take steps of
// the contraction in turn, their sums meet in LDS.
#pragma once
#include "stream_dev.h"

namespace oz {

constexpr int kFewWaves = 8;

template <class T, int NX>
__global__ __launch_bounds__(64 * kFewWaves) void few_tokens_kernel(Product a, float *partial, int steps_per_split)
{
    constexpr int KE = 8 * Chunk<T>::E;
    __shared__ __attribute__((aligned(16))) float sums[kFewWaves][NX][16 * kStreamLd];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int p0 = blockIdx.x * 16, row = p0 + (lane & 15);
    const T *const w[1] = {(const T *)a.P + (size_t)(row < a.e.np ? row : a.e.np - 1) * a.ldp};
    const T *x[NX];
    bool on[NX];
#pragma unroll
    for (int j = 0; j < NX; ++j) {
        const int q = 16 * j + (lane & 15);
        on[j] = q < a.e.nq;
        x[j] = (const T *)a.Q + (size_t)(on[j] ? q : 0) * a.ldq;
    }
    v4f acc[1][NX];
#pragma unroll
    for (int j = 0; j < NX; ++j) acc[0][j] = v4f{0, 0, 0, 0};
    const int all = (a.nk + KE - 1) / KE, first = blockIdx.y * steps_per_split, last = all < first + steps_per_split ? all : first + steps_per_split;
    stream_products<T, 1, NX, NX == 1 ? 4 : 2>(acc, w, x, on, first + wave, last, kFewWaves, a.nk, lane);
#pragma unroll
    for (int j = 0; j < NX; ++j) put_sums(sums[wave][j], acc[0][j], lane);
    __syncthreads();
    for (int i = threadIdx.x; i < NX * 32; i += 64 * kFewWaves) {
        const int q = i >> 1, c = (i & 1) * 8, p = p0 + c;
        if (q >= a.e.nq || p >= a.e.np) continue;
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < kFewWaves; ++s) {
            const float *from = &sums[s][q >> 4][(q & 15) * kStreamLd + c];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += from[e];
        }
        if (partial) {
            float *to = partial + ((size_t)blockIdx.y * a.e.nq + q) * ((a.e.np + 7) & ~7) + p;
            *(v4f *)to = v4f{v[0], v[1], v[2], v[3]};
            *(v4f *)(to + 4) = v4f{v[4], v[5], v[6], v[7]};
        } else {
            finish_row<T>(a.e, q, p, v);
        }
    }
}

template <class T, int NX>
hipError_t launch_few(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    few_tokens_kernel<T, NX><<<dim3((a.e.np + 15) / 16, plan.splits), 64 * kFewWaves, 0, st>>>(a, plan.splits > 1 ? partial : nullptr, plan.steps);
    return hipGetLastError();
}

template <class T>
hipError_t launch_few_tokens(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    return a.e.nq <= 16   ? launch_few<T, 1>(a, plan, partial, st)
           : a.e.nq <= 32 ? launch_few<T, 2>(a, plan, partial, st)
           : a.e.nq <= 48 ? launch_few<T, 3>(a, plan, partial, st)
                          : launch_few<T, 4>(a, plan, partial, st);
}

}  // namespace oz
