// The feed-forward block's matrix products, bf16.
#include "ffn_rows_device.h"

namespace evg {

template <>
hipError_t launch_gemm<bf16_t>(GemmOp op, GemmTile tile, bool aligned, const GemmArgs& g, hipStream_t s) {
  return launch_any<bf16_t>(op, tile, aligned, g, s);
}

}  // namespace evg
