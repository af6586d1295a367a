// Launch descriptions of the feed-forward block's matrix products.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ffn_choose.h"
#include "gemm_operand.h"
#include "launch_pieces.h"

namespace evg {

// a = x s(x): s the logistic function of x (c0 + c1 x^2), the step, or (erf) the normal distribution.
struct Activation {
  float c0, c1;
  uint32_t relu, erf;
};

// C (M x N) from products over K; for each of `workers` and `parts`.
struct GemmArgs {
  GemmOperand a[2], b[2], c[2];   // phases of the product (GEMM_INPUT), gate and up (GEMM_GATED), or parts (GEMM_WEIGHT)
  uint32_t M, N, K, workers, parts;
  uint32_t tiles_m, tiles_n;
  uint32_t first;                  // workgroup of a launch in pieces
  Activation activation;
  // GEMM_GATED, GEMM_GATED_BWD: the projections in 32 bits, in the accumulators' order; the gradients are rows of c[0], gate's at 0, up's at `pitch`
  float* proj;
  uint64_t proj_worker;
  uint32_t pitch;                  // padded hidden width
};

// Copies of operands whose rows are no whole 16-byte units, with rows of `pitch` elements that are: zeros up to the next unit.
struct PackOne {
  GemmOperand from;
  void* to;            // [workers][rows][pitch]
  uint32_t rows, cols, pitch;
  uint64_t first;      // rows of the operands ahead of it
};
struct PackArgs {
  PackOne one[4];
  uint32_t count, first;           // first workgroup of a launch in pieces
  uint64_t lines;
};
hipError_t launch_pack(uint32_t type, PackArgs a, hipStream_t s);

template <typename T> hipError_t launch_gemm(GemmOp op, GemmTile tile, bool aligned, const GemmArgs& g, hipStream_t s);

}  // namespace evg
