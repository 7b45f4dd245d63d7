// Linear layers on 8-bit codes with fp32 outputs.

#include "qlin_kernels.h"

namespace aqd {

hipError_t launch_qlin_f32(const QlinArgs &a, int shape, hipStream_t stream) { return launch_typed<float>(a, shape, stream); }

}  // namespace aqd
