// Copies of operands whose rows are not on 16 bytes, or do not end with a chunk of 16: aligned rows, zeros behind them.
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
    *(v4u *)((T *)c.to + row * c.ldto + k) = load_chunk((const T *)c.from + row * c.ld + k, c.cols - k);
}

}  // namespace

hipError_t launch_pad(const PadCopies &a, int type, hipStream_t st)
{
    const int e = type == OZIMMU_F32 ? 4 : 8;
    const long long chunks = a.c[0].rows * (a.c[0].ldto / e) + a.c[1].rows * (a.c[1].ldto / e);
    if (chunks == 0) return hipSuccess;
    const long long groups = (chunks + 255) / 256;
    const dim3 grid(grid_row(groups), grid_rows(groups));
    if (type == OZIMMU_BF16) pad_kernel<bf16><<<grid, 256, 0, st>>>(a);
    else if (type == OZIMMU_F16) pad_kernel<f16><<<grid, 256, 0, st>>>(a);
    else pad_kernel<float><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace oz
