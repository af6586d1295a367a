// The feed-forward block's matrix products and the tiles that they are cut into: which one a product takes.
#pragma once
#include <math.h>
#include <stdint.h>

namespace evg {

enum GemmOp : uint32_t {
  GEMM_GATED = 0,     // h = act(A Bg^T) * (A Bu^T), both K-contiguous; writes h and, for a backward pass, both projections
  GEMM_DOWN = 1,      // C = A B^T, both K-contiguous
  GEMM_GATED_BWD = 2, // dh = A B, B N-contiguous; writes the gradients of both projections
  GEMM_INPUT = 3,     // C = A0 B0 + A1 B1, B N-contiguous
  GEMM_WEIGHT = 4,    // C = A^T B, A M-contiguous, B N-contiguous; two of them at once
  GEMM_OPS = 5
};

// Tiles: 256 x 256 and 128 x 128 (aligned operands of 16 bits), 64 x 128; few tokens (GEMM_GATED and GEMM_DOWN of at most kMostRows); 32 x 64,
// 32 x 32 and 64 x 64 (aligned) with k shared out among the wavefronts.
enum GemmTile : uint32_t { TILE_256 = 0, TILE_128 = 1, TILE_64 = 2, TILE_ROWS = 3, TILE_SMALL = 4, TILE_SMALL_NARROW = 5, TILE_SMALL_SQUARE = 6 };
constexpr uint32_t kMostRows = 64;

// C (M x N) from products over K, for each of `workers` and `parts`; padding columns that are written count.
struct GemmShape { uint32_t M, N, K, workers, parts; };

// The tile with the least time by a model of what was measured (warm, normal values, us; a step is 128 bytes of k of a tile):
//   16 bits  256 x 256  one a CU, 1.29 a step, and 2.1 with all CUs busy, when the chip's power binds
//            128 x 128  two a CU, 0.84 or 1.04 a step; 1.17 times the energy for the same product
//             64 x 128  three a CU, 0.66, 0.72 or 1.0 a step; 1.5 times the energy
//             32 x  64  k shared out to four wavefronts, one a CU: 0.68 for four steps and 2 for their sums, 3.6 where results are many
//             64 x  64  the same with 0.82, and 3.6 or 5.5: half as many of them
//   32 bits  the products bind a CU: 1.06 a step of 64 x 128, 1.3 for four of 32 x 64, 2.26 for four of 64 x 64
// Measured, bf16, 256 / 128 / 64:  8192 tokens 2048 x 8192 in all 2259 / 2657 / 3499;  1024 tokens 2048 x 8192, gated 65 / 71 / 84, down 165 / 95 / 92;
// 2048 tokens 2048 x 2048, gated 51 / 39 / 52;  64 x 128 / 32 x 64 / 64 x 64:  512 tokens 1024 x 2816, down 26 / 11 / 14, input 56 / 17 / 21;  8 x 250 tokens
// 512 x 1344, down 14.0 / 13.4 / 10.8, input 29 / 21 / 16, gated 13 / 41 / 32;  1024 tokens 1024 x 4096, down 36 / 27 / 18, input 81 / 48 / 30; 2048 x 8192, down 96 / 103 / 62, input 161 / 167 / 108;  128 tokens
// 2048 x 5632, gated backward 24 / 19 / 15, weights 18 / 178 / 117;  f32, 8 x 250 tokens 512 x 1344, down 47 / 34 / 31, gated 56 / 84 / 77.
// The gated backward product ends with as much reading and writing as products, which another workgroup's products on the CU overlap: 1024 tokens 2048
// x 8192 76 / 48 / 60, 8192 tokens 433 / 410 / 431; where 128 x 128 are few, 2048 tokens 2048 x 2048, 67 / 35 / 32.
inline GemmTile choose_tile(GemmOp op, const GemmShape& g, bool aligned, bool wide) {
  if ((op == GEMM_GATED || op == GEMM_DOWN) && g.M <= kMostRows) return TILE_ROWS;
  const uint32_t share = op == GEMM_GATED ? 2 : 1;
  auto count = [&](uint64_t bm, uint64_t bn) { return (double)(((g.M + bm - 1) / bm) * ((g.N + bn / share - 1) / (bn / share)) * g.workers * g.parts); };
  const double steps = (double)(((uint64_t)g.K * (wide ? 4 : 2) + 127) / 128 * (op == GEMM_INPUT ? 2 : 1));
  auto rest = [](double c, double slots) { return c - floor(c / slots) * slots; };
  const double c64 = count(64, 128), r64 = rest(c64, 768);
  const double t64 = wide ? steps * 1.06 * ceil(c64 / 256) + 1 : steps * fmax(floor(c64 / 768) + (r64 == 0 ? 0 : r64 <= 256 ? 0.66 : r64 <= 512 ? 0.72 : 1.0), 1.4 * 0.00103 * c64) + 1;
  GemmTile best = TILE_64;
  double t = t64;
  auto offer = [&](GemmTile tile, double time) {
    if (time < t) { best = tile; t = time; }
  };
  if (aligned && !wide) {
    const double c128 = count(128, 128), c256 = count(256, 256), r128 = rest(c128, 512);
    if (op == GEMM_GATED_BWD) {
      if (c128 > 384) return TILE_128;
    } else {
      offer(TILE_128, steps * fmax(floor(c128 / 512) * 1.04 + (r128 == 0 ? 0 : r128 <= 256 ? 0.84 : 1.04), 1.17 * 0.00206 * c128) + 1);
      offer(TILE_256, steps * fmax(ceil(c256 / 256) * 1.29, 0.0082 * c256) + 1);
    }
  }
  if (steps >= 4) {   // one for each wavefront
    const bool many = op == GEMM_GATED_BWD || op == GEMM_WEIGHT;
    const double small = count(32, 64), square = count(64, 64);
    offer(op != GEMM_GATED && small <= 64 ? TILE_SMALL_NARROW : TILE_SMALL, ceil(small / 256) * (steps / 4 * (wide ? 1.3 : 0.68) + (many ? 3.6 : 2.)) + 2);
    if (aligned) offer(TILE_SMALL_SQUARE, ceil(square / 256) * (steps / 4 * (wide ? 2.26 : 0.82) + (many ? 5.5 : 3.6)) + 2);
  }
  return best;
}

}  // namespace evg
