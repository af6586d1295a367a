// The tiles that the products of orthogonal updates are cut into, and into how many parts of k.
#pragma once
#include <math.h>
#include <stdint.h>

namespace evg {

// M x N sums over K for each of `matrices`; floats that partial sums have room in.
struct OrthoShape { uint32_t M, N, K, matrices; uint64_t room; };
struct OrthoChoice { uint32_t tile, parts; };

// Workgroups that a part of a product has; of symmetric ones, whose tiles below the diagonal are left out, some have no tile.
inline uint64_t ortho_cells(bool symmetric, uint64_t tiles_m, uint64_t tiles_n) {
  if (!symmetric) return tiles_m * tiles_n;
  uint64_t cells = 0;
  for (uint64_t first = 0; first < tiles_m; first += 4) cells += (tiles_m - first < 4 ? tiles_m - first : 4) * (tiles_m - first);
  return cells;
}

// Floats of partial sums.
inline uint64_t ortho_partial(const OrthoShape& g, bool symmetric, OrthoChoice c) {
  const uint64_t m = (g.M + c.tile - 1) / c.tile, n = (g.N + c.tile - 1) / c.tile;
  return c.parts > 1 ? ortho_cells(symmetric, m, n) * g.matrices * c.parts * c.tile * c.tile : 0;
}

// The choice with the least time by a model of what was measured (us; a step is 128 bytes of k of a tile, of hi alone or of both parts):
//            a CU has    a step, few workgroups / all CUs busy    both parts      the results' way out
//   256 x 256    1             1.5 / 1.9                            2.4 / 3.2, so never          18, of parts 8, and of X never in parts
//   128 x 128    2             0.72 / 1.05                          0.8 / 1.4                     9          5
//    64 x  64    2             0.42 / 0.5                           0.45 / 0.65                   3.5        3
// and adding up the parts 4 and 0.19 a MB, 0.55 where the caches do not hold them.  Measured, tile and parts: S of 4096 x 11264, hi alone, 256 268, 256 in three parts 211 + 24,
// 128 in two 232 + 17, 64 356; X' of the same 256 386, 128 440, 64 700; both parts, S of 2048 x 5632 256 316, 256 in four 102 + 11, 128 139, 128 in three 89 + 11, 64 151, P 128 59, in three
// 37 + 16, X' 256 158, 128 153, 64 210; S of four 128 x 784 64 12.8, in four parts 5.5 + 4.0.
inline OrthoChoice choose_ortho(const OrthoShape& g, bool symmetric, bool split) {
  struct { uint32_t tile, slots; double few[2], busy[2], out, part_out; } const kinds[] = {
      {256, 256, {1.5, 0}, {1.9, 0}, 18, 8}, {128, 512, {0.72, 0.8}, {1.05, 1.4}, 9, 5}, {64, 512, {0.42, 0.45}, {0.5, 0.65}, 3.5, 3}};
  // More than 192 of 256 workgroups keep the chip as busy as all.
  const uint32_t steps = (uint32_t)(((uint64_t)g.K + (split ? 31 : 63)) / (split ? 32 : 64));
  OrthoChoice best{64, 1};
  double least = 1e300;
  for (const auto& t : kinds) {
    if (t.tile == 256 && split) continue;
    const uint32_t most = t.tile == 256 && !symmetric ? 1 : 8;
    const uint64_t m = ((uint64_t)g.M + t.tile - 1) / t.tile, n = ((uint64_t)g.N + t.tile - 1) / t.tile;
    const double tiles = (double)(symmetric ? m * (m + 1) / 2 : m * n) * g.matrices;
    for (uint32_t parts = 1; parts <= most && parts <= steps; ++parts) {
      const uint64_t partial = ortho_partial(g, symmetric, {t.tile, parts});
      if (partial > g.room) break;
      const double each = (steps + parts - 1) / parts, out = parts > 1 ? t.part_out : t.out, count = tiles * parts;
      const double whole = floor(count / t.slots), rest = count - whole * t.slots;
      const double mb = (double)partial * 4e-6;
      const double time = whole * (each * t.busy[split] + out) + (rest > 0 ? each * (rest <= (t.tile == 256 ? 192 : 256) ? t.few : t.busy)[split] + out : 0) +
                          (parts > 1 ? 4 + mb * (mb > 150 ? 0.55 : 0.19) : 0);
      if (time < least) {
        least = time;
        best = {t.tile, parts};
      }
    }
  }
  return best;
}

}  // namespace evg
