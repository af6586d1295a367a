// The feed-forward block's matrix products, half_t.
#include "ffn_gemm_device.h"

namespace evg {

template <>
hipError_t launch_gemm<half_t>(GemmOp op, GemmTile tile, bool aligned, const GemmArgs& g, hipStream_t s) {
  switch (op) {
    case GEMM_GATED: return launch_op<half_t, GEMM_GATED>(tile, aligned, g, s);
    case GEMM_DOWN: return launch_op<half_t, GEMM_DOWN>(tile, aligned, g, s);
    case GEMM_GATED_BWD: return launch_op<half_t, GEMM_GATED_BWD>(tile, aligned, g, s);
    case GEMM_INPUT: return launch_op<half_t, GEMM_INPUT>(tile, aligned, g, s);
    case GEMM_WEIGHT: return launch_op<half_t, GEMM_WEIGHT>(tile, aligned, g, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace evg
