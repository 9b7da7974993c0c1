// Copies of operands whose rows are not on 16 bytes, or do not end with a chunk of 16: aligned rows, zeros behind them; and of operands
// that are held in 8 bits with a scale for each row, as the values they stand for, rounded to the type of the product.
//
// Bound by memory: read once, written once, a chunk a thread.  Up to two operands in a launch.
#include "layers.h"

namespace oz {
namespace {

template <class T>
__global__ __launch_bounds__(256) void pad_kernel(PadCopies a)
{
    constexpr int E = Chunk<T>::E;
    long long i = ((long long)blockIdx.y * kGridRow + blockIdx.x) * 256 + threadIdx.x;
    const long long first = a.c[0].rows * (a.c[0].ldto / E), all = first + a.c[1].rows * (a.c[1].ldto / E);
    if (i >= all) return;
    const bool second = i >= first;
    const PadCopy &c = a.c[second];
    if (second) i -= first;
    const int chunks = c.ldto / E;
    const long long row = i / chunks;
    const int k = (int)(i - row * chunks) * E;
    T *const to = (T *)c.to + row * c.ldto + k;
    if constexpr (sizeof(T) > 1)
        if (c.scale) {
            const int8_t *const from = (const int8_t *)c.from + row * c.ld + k;
            const float scale = c.scale[row];
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
    *(v4u *)to = load_chunk((const T *)c.from + row * c.ld + k, c.cols - k);
}

}  // namespace

hipError_t launch_pad(const PadCopies &a, int type, hipStream_t st)
{
    const int e = 16 / (int)element_bytes(type);
    const long long chunks = a.c[0].rows * (a.c[0].ldto / e) + a.c[1].rows * (a.c[1].ldto / e);
    if (chunks == 0) return hipSuccess;
    const long long groups = (chunks + 255) / 256;
    const dim3 grid(grid_row(groups), grid_rows(groups));
    if (type == kType8) pad_kernel<int8_t><<<grid, 256, 0, st>>>(a);
    else if (type == OZIMMU_BF16) pad_kernel<bf16><<<grid, 256, 0, st>>>(a);
    else if (type == OZIMMU_F16) pad_kernel<f16><<<grid, 256, 0, st>>>(a);
    else pad_kernel<float><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace oz
