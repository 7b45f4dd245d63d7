// Linear layers on 8-bit codes with bf16 outputs.

#include "qlin_kernels.h"

namespace aqd {

hipError_t launch_qlin_bf16(const QlinArgs &a, int shape, hipStream_t stream) { return launch_typed<__bf16>(a, shape, stream); }

}  // namespace aqd
