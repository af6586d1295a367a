// The feed-forward block's matrix products, f16.
#include "ffn_rows_device.h"

namespace evg {

template <>
hipError_t launch_gemm<half_t>(GemmOp op, GemmTile tile, bool aligned, const GemmArgs& g, hipStream_t s) {
  return launch_any<half_t>(op, tile, aligned, g, s);
}

}  // namespace evg
