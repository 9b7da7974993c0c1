// Products with few columns: rows of a weight streamed once, from memory into the matrix instructions' registers.
//
// A wavefront takes 16 rows of the weight (rows of the matrix instruction) and 16 tokens per column block; lane l loads 16
// bytes of row l % 16 at chunk l / 16 of a half step, so a step reads 128 contiguous bytes of each row.  LDS would
// only delay them: no row is used twice.  Bound by memory; what matters is that enough loads are in flight, hence U steps'
// loads are issued before the first of their products (16 x 4096 x 4096 bf16: 33 MB in 9.8 us).
#pragma once
#include "layers_dev.h"

namespace oz {

// acc[i][j] += W_i X_j over the steps first, first + stride, ... < last of an operand of nk entries.  w[i], x[j]: this lane's
// rows.  Lanes whose `on[j]` is false take zeros instead of x[j].
template <class T, int NW, int NX, int U>
__device__ __forceinline__ void stream_products(v4f (&acc)[NW][NX], const T *const (&w)[NW], const T *const (&x)[NX], const bool (&on)[NX], int first,
                                                int last, int stride, int nk, int lane)
{
    constexpr int E = Chunk<T>::E, KE = 8 * E;
    const int g = (lane >> 4) * E;
    for (int t = first; t < last; t += U * stride) {
        v4u a[U][2][NW], b[U][2][NX];
        const int end = t + (U - 1) * stride;
        if (end < last && (end + 1) * KE <= nk) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int k = (t + u * stride) * KE + s * 4 * E + g;
#pragma unroll
                    for (int i = 0; i < NW; ++i) __builtin_memcpy(&a[u][s][i], w[i] + k, 16);
#pragma unroll
                    for (int j = 0; j < NX; ++j) {
                        b[u][s][j] = v4u{0, 0, 0, 0};
                        if (on[j]) __builtin_memcpy(&b[u][s][j], x[j] + k, 16);
                    }
                }
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int k = (t + u * stride) * KE + s * 4 * E + g, n = t + u * stride < last ? nk - k : 0;
#pragma unroll
                    for (int i = 0; i < NW; ++i) a[u][s][i] = load_chunk(w[i] + k, n);
#pragma unroll
                    for (int j = 0; j < NX; ++j) b[u][s][j] = load_chunk(x[j] + k, on[j] ? n : 0);
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < NW; ++i)
#pragma unroll
                    for (int j = 0; j < NX; ++j) acc[i][j] = mma(a[u][s][i], b[u][s][j], acc[i][j], T{});
    }
}

// A wavefront's 16 x 16 sums as 16 rows (columns of the matrix instruction) of 16 floats, rows kStreamLd apart.
constexpr int kStreamLd = 20;
__device__ __forceinline__ void put_sums(float *to, v4f c, int lane) { *(v4f *)(to + (lane & 15) * kStreamLd + 4 * (lane >> 4)) = c; }

}  // namespace oz
