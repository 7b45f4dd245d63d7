// Linear layers on 8-bit codes: the launches that leave partial sums of a split k range, and
// the sum of those.

#include "qlin_kernels.h"

namespace aqd {

hipError_t launch_qlin_part(const QlinArgs &a, int shape, hipStream_t stream)
{
    if (a.gate)
        launch_shape<float, true, true>(a, shape, stream);
    else
        launch_shape<float, false, true>(a, shape, stream);
    return hipGetLastError();
}

namespace {

template <typename T>
void combine(const QlinArgs &a, hipStream_t stream)
{
    const long long items = (long long)a.rows * (a.n_pad / 4);   // few: their sums fit the workspace
    const dim3 grid((unsigned)((items + 255) / 256));
    if (a.gate)
        hipLaunchKernelGGL((qlin_combine_kernel<T, true>), grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((qlin_combine_kernel<T, false>), grid, dim3(256), 0, stream, a);
}

}  // namespace

hipError_t launch_qlin_combine(const QlinArgs &a, hipStream_t stream)
{
    if (a.type == AQD_F32)
        combine<float>(a, stream);
    else if (a.type == AQD_F16)
        combine<_Float16>(a, stream);
    else
        combine<__bf16>(a, stream);
    return hipGetLastError();
}

}  // namespace aqd
