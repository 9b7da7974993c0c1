// Copies of operands whose rows are not on 16 bytes, or do not end with a chunk of 16: aligned rows, zeros behind them; and of operands that
// are held in 8 bits: in 32 bits the values that they stand for, in 16 bits code * power of two, which is exact (split_scale).
//
// Bound by memory: read once, written once, a chunk a thread.  Up to two operands in a launch.
#include "pad_dev.h"

namespace oz {
namespace {

template <class T>
__global__ __launch_bounds__(256) void pad_kernel(PadCopies a)
{
    pad_chunk<T>(a, ((long long)blockIdx.y * kGridRow + blockIdx.x) * 256 + threadIdx.x);
}

}  // namespace

hipError_t launch_pad(const PadCopies &a, int type, hipStream_t st)
{
    const long long groups = pad_groups(a, type);
    if (groups == 0) return hipSuccess;
    const dim3 grid(grid_row(groups), grid_rows(groups));
    if (type == kType8) pad_kernel<int8_t><<<grid, 256, 0, st>>>(a);
    else if (type == OZIMMU_BF16) pad_kernel<bf16><<<grid, 256, 0, st>>>(a);
    else if (type == OZIMMU_F16) pad_kernel<f16><<<grid, 256, 0, st>>>(a);
    else pad_kernel<float><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace oz
