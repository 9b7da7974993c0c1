// Copies of operands in front of a product, a chunk of 16 bytes a thread: to aligned rows, or from 8 bits.  Bound by memory; they ride in the
// launch for dz (948 x 91 -> 768 f16 with x in 8 bits: the call 16 us, with launches of their own 38), or make one themselves.
#pragma once
#include "layers.h"

namespace oz {

// chunk i of the copies, one behind the other
template <class T>
__device__ __forceinline__ void pad_chunk(const PadCopies &a, long long i)
{
    constexpr int E = Chunk<T>::E;
    const long long first = a.c[0].rows * (a.c[0].ldto / E), all = first + a.c[1].rows * (a.c[1].ldto / E);
    if (i >= all) return;
    const bool second = i >= first;
    const PadCopy &c = a.c[second];
    if (second) i -= first;
    const int chunks = c.ldto / E;
    const long long row = i >> 32 ? i / chunks : (long long)((unsigned)i / (unsigned)chunks);      // (64-bit division: as long as the copy)
    const int k = (int)(i - row * chunks) * E;
    T *const to = (T *)c.to + row * c.ldto + k;
    if constexpr (sizeof(T) > 1)
        if (c.scale) {
            const int8_t *const from = (const int8_t *)c.from + row * c.ld + k;
            const float scale = sizeof(T) == 2 ? split_scale<T>(c.scale[row]).power : c.scale[row];
            float v[E];
            if (k + E <= c.cols) {
                typedef int8_t V __attribute__((ext_vector_type(E)));
                V x;
                __builtin_memcpy(&x, from, E);
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = (float)x[e] * scale;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = k + e < c.cols ? (float)from[e] * scale : 0.0f;
            }
            store_row(to, v);
            return;
        }
    *(v4u *)to = load_chunk((const T *)c.from + row * c.ld + k, c.cols - k, k);
}

// work-groups of 256
inline long long pad_groups(const PadCopies &a, int type)
{
    const int e = 16 / (int)element_bytes(type);
    return (a.c[0].rows * (a.c[0].ldto / e) + a.c[1].rows * (a.c[1].ldto / e) + 255) / 256;
}

}  // namespace oz
