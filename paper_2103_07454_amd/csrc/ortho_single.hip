// The products of orthogonal updates of 16-bit matrices: one part of each operand.
#include "ortho_gemm_device.h"

namespace evg {

template <>
hipError_t launch_ortho_parts<false>(OrthoOp op, bool tall, bool last, const OrthoArgs& a, hipStream_t s) {
  return launch_ortho_any<false>(op, tall, last, a, s);
}

}  // namespace evg
