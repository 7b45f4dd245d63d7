// Linear layers on 8-bit codes with fp16 outputs.

#include "qlin_kernels.h"

namespace aqd {

hipError_t launch_qlin_f16(const QlinArgs &a, int shape, hipStream_t stream) { return launch_typed<_Float16>(a, shape, stream); }

}  // namespace aqd
