// The products of orthogonal updates of 32-bit matrices: both parts of each operand.
#include "ortho_gemm_device.h"

namespace evg {

template <>
hipError_t launch_ortho_parts<true>(OrthoOp op, bool tall, bool last, const OrthoArgs& a, hipStream_t s) {
  return launch_ortho_any<true>(op, tall, last, a, s);
}

}  // namespace evg
