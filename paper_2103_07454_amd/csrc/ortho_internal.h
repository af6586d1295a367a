// Launch descriptions of the products of orthogonal updates.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/evg_nn.h"
#include "launch_pieces.h"
#include "nn_device.h"

namespace evg {

enum OrthoOp : uint32_t {
  ORTHO_GRAM = 0,    // S = X X^T, or (tall) X^T X: symmetric
  ORTHO_SQUARE = 1,  // P = b S + c S S: symmetric
  ORTHO_APPLY = 2    // X' = a X + P X, or (tall) a X + X P
};

// A float16 matrix in two parts, hi + lo.  Products of both parts have them side by side: 32 elements of a row's hi, the same 32 of its lo, and so on; products of
// hi alone have a matrix of hi and, `apart` elements behind it, one of lo.
struct Halves {
  uint16_t* p;
  int64_t apart;        // from an element's hi to its lo; 0: there is no lo
  int64_t worker, ld;   // elements between matrices and between rows: whole 128 bytes
  uint32_t paired;
};

__host__ __device__ __forceinline__ uint32_t halves_col(uint32_t paired, uint32_t col) { return paired ? (col & ~31u) * 2 + (col & 31) : col; }

// A float16's nearest value and what that leaves.  The value is settled in 32 bits first: a product or sum that the compiler rounds to 16 bits in one
// instruction in one place, and in two in the other, would leave a remainder of another number than the one that is stored.
__device__ __forceinline__ void halves_of(float v, half_t* hi, half_t* lo) {
  asm("" : "+v"(v));
  *hi = (half_t)v;
  *lo = (half_t)(v - (float)*hi);
}

struct OrthoArgs {
  Halves a, b;           // the product's operands
  Halves own;            // what is added to it, at the same place
  Halves to;
  uint32_t M, N, K;
  float f_acc, f_own;    // result = f_acc * product + f_own * own
  uint32_t matrices, tiles_m, tiles_n, cells, first;
  uint32_t parts, part_steps;   // k is shared out to so many workgroups, so many steps each
  float* partial;        // [matrices][parts][cells][tile], where parts > 1
  uint64_t room;         // floats of it
  evg_mat out;           // the last step's result, of out_type
  uint32_t out_type;
};

// split: products of both parts of the operands; last: the result goes to out.
hipError_t launch_ortho(OrthoOp op, bool tall, bool split, bool last, const OrthoArgs& a, hipStream_t s);
template <bool SPLIT> hipError_t launch_ortho_parts(OrthoOp op, bool tall, bool last, const OrthoArgs& a, hipStream_t s);

}  // namespace evg
