// The feed-forward block's matrix products, 32 bits.
#include "ffn_rows_device.h"

namespace evg {

template <>
hipError_t launch_gemm<float>(GemmOp op, GemmTile tile, bool aligned, const GemmArgs& g, hipStream_t s) {
  return launch_any<float>(op, tile, aligned, g, s);
}

}  // namespace evg
