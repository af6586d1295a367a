// The products where there are few tiles: small tiles, and k shared out among a workgroup's wavefronts.
//
// A workgroup has 32 TM rows and 32 TN columns; each of its four or eight wavefronts takes every fourth or eighth step of k through buffers of its
// own, so none waits for another until their sums meet in LDS, in a fixed order.  Then four of them finish a quarter of the columns each.
#pragma once
#include "ffn_gemm_device.h"

namespace evg {

template <typename T, int OP, bool ERF, int TM, int TN, int kSplit, bool ALIGNED>
__global__ __launch_bounds__(kSplit * 64) void k_ffn_small(GemmArgs g) {
  constexpr bool AKC = OP != GEMM_WEIGHT, BKC = OP == GEMM_GATED || OP == GEMM_DOWN;
  static_assert(OP != GEMM_GATED || TN == 2, "gate's columns and up's");
  using LA = Tile<T, 32 * TM, AKC>;
  using LB = Tile<T, 32 * TN, BKC>;
  constexpr int UNITS = LA::kUnits + LB::kUnits, BK = LA::BK;
  __shared__ u32x4 lds0[kSplit][UNITS], lds1[kSplit][UNITS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t tiles = g.tiles_m * g.tiles_n;
  const uint32_t place = place_by_xcd(g.first), cell = place / tiles, part = cell % g.parts, w = cell / g.parts, id = place % tiles;
  const uint32_t m0 = id % g.tiles_m * (32 * TM), n0 = id / g.tiles_m * (OP == GEMM_GATED ? 32 : 32 * TN);

  Loader<T, 32 * TM, AKC, 1, ALIGNED, false> la;
  // Gate's rows of the tile and up's come from two matrices: a loader for each.
  constexpr bool PAIR = OP == GEMM_GATED;
  Loader<T, PAIR ? 32 : 32 * TN, BKC, 1, ALIGNED, false> lb, lb2;
  constexpr int NA = decltype(la)::N, NB = decltype(lb)::N, LOADS = NA + (PAIR ? 2 : 1) * NB;
  u32x4 held[ALIGNED ? 1 : LOADS];
  const uint32_t steps1 = (g.K + BK - 1) / BK, steps = steps1 * (OP == GEMM_INPUT ? 2 : 1);
  uint32_t step = wave, phase = 0;
  auto start = [&]() {
    la.start(g.a[OP == GEMM_WEIGHT ? part : phase], w, m0, g.M, g.K, 0, lane);
    lb.start(g.b[OP == GEMM_INPUT ? phase : 0], w, n0, g.N, g.K, 0, lane);
    if (PAIR) lb2.start(g.b[1], w, n0, g.N, g.K, 0, lane);
    const uint32_t at = step - phase * steps1;
    la.skip(at);
    lb.skip(at);
    if (PAIR) lb2.skip(at);
  };
  auto fetch = [&](u32x4* lds) {   // this wavefront's next step
    if (OP == GEMM_INPUT && !phase && step >= steps1) {
      phase = 1;
      start();
    }
    const int k_left = (int)g.K - (int)((step - phase * steps1) * BK);
    la.fetch(k_left, lds, held, 0, lane);
    lb.fetch(k_left, lds + LA::kUnits, held + (ALIGNED ? 0 : NA), 0, lane);
    if (PAIR) lb2.fetch(k_left, lds + LA::kUnits + 32 * 8, held + (ALIGNED ? 0 : NA + NB), 0, lane);
    la.skip(kSplit - 1);
    lb.skip(kSplit - 1);
    if (PAIR) lb2.skip(kSplit - 1);
    step += kSplit;
  };
  auto put = [&](u32x4* lds) {
    la.put(lds, held, 0, lane);
    lb.put(lds + LA::kUnits, held + (ALIGNED ? 0 : NA), 0, lane);
    if (PAIR) lb2.put(lds + LA::kUnits + 32 * 8, held + (ALIGNED ? 0 : NA + NB), 0, lane);
    __builtin_amdgcn_wave_barrier();
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  auto multiply = [&](const u32x4* lds) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      Frag<T> a[TM];
#pragma unroll
      for (int i = 0; i < TM; ++i) a[i] = read_frag<T, 32 * TM, AKC>(lds, 0, i * 32, ks, lane);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const Frag<T> b = read_frag<T, 32 * TN, BKC>(lds, LA::kUnits, j * 32, ks, lane);
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[i][j] = mfma(b, a[i], acc[i][j]);
      }
    }
  };
  // Loads of two steps are under way; the older ones are waited for, and a buffer is filled again once its reads are done.
  auto wait = [&](auto count) {
    constexpr int N = decltype(count)::value;
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4);   // vmcnt N, lgkmcnt 0
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  const uint32_t mine = steps > (uint32_t)wave ? (steps - wave + kSplit - 1) / kSplit : 0;
  if (mine) {
    start();
    if constexpr (ALIGNED) {
      fetch(lds0[wave]);
      fetch(lds1[wave]);
      for (uint32_t i = 0; i < mine; i += 2) {   // behind the last step come zeros
        wait(std::integral_constant<int, LOADS>{});
        multiply(lds0[wave]);
        wait(std::integral_constant<int, LOADS>{});
        fetch(lds0[wave]);
        wait(std::integral_constant<int, LOADS>{});
        multiply(lds1[wave]);
        wait(std::integral_constant<int, LOADS>{});
        fetch(lds1[wave]);
      }
      wait(std::integral_constant<int, 0>{});
    } else {
      fetch(lds0[wave]);
      for (uint32_t i = 0; i < mine; ++i) {
        put(lds0[wave]);
        if (i + 1 < mine) fetch(lds0[wave]);
        multiply(lds0[wave]);
        __builtin_amdgcn_wave_barrier();
      }
    }
  }

  __syncthreads();
  f32x4* const sums = (f32x4*)&lds0[0][0];   // [wavefront][i][j][q][lane]
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        sums[(((wave * TM + i) * TN + j) * 4 + q) * 64 + lane] = f32x4{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
  __syncthreads();
  if (wave >= 4) return;
  const int q = wave, inner = 8 * q + 4 * (lane >> 5);
  const GemmOperand& co = g.c[OP == GEMM_WEIGHT ? part : 0];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const uint32_t rows0 = m0 + i * 32, m = rows0 + (lane & 31);
    if (m >= g.M) return;
    f32x4 v[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      v[j] = sums[((i * TN + j) * 4 + q) * 64 + lane];
#pragma unroll
      for (int s = 1; s < kSplit; ++s) v[j] += sums[(((s * TM + i) * TN + j) * 4 + q) * 64 + lane];
    }
    T* const c = (T*)co.p + (int64_t)w * co.worker + (int64_t)m * co.ld;
    if constexpr (OP == GEMM_GATED) {
      const uint32_t n = n0 + inner;
      if (n >= g.pitch) return;
      f32x4 gate, up;
      float h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool real = n + e < g.N;   // the columns up to `pitch` are 0
        gate[e] = real ? v[0][e] : 0.f;
        up[e] = real ? v[1][e] : 0.f;
        float a, slope;
        activate<ERF, sizeof(T) == 2>(g.activation, gate[e], a, slope);
        h[e] = real ? a * up[e] : 0.f;
      }
      store_n<4>(c + n, h);
      if (g.proj) {
        float* p = proj_at(g, w, rows0, n0, q, lane);
        *(f32x4*)p = gate;
        *(f32x4*)(p + 1024) = up;
      }
    } else {
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const uint32_t n = n0 + j * 32 + inner;
        if constexpr (OP == GEMM_GATED_BWD) {
          if (n >= g.pitch) continue;
          const float* p = proj_at(g, w, rows0, n0 + j * 32, q, lane);
          const f32x4 gate = *(const f32x4*)p, up = *(const f32x4*)(p + 1024);
          float dg[4], du[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float a, slope;
            activate<ERF, sizeof(T) == 2>(g.activation, gate[e], a, slope);
            const bool real = n + e < g.N;
            dg[e] = real ? v[j][e] * up[e] * slope : 0.f;
            du[e] = real ? v[j][e] * a : 0.f;
          }
          store_n<4>(c + n, dg);
          store_n<4>(c + g.pitch + n, du);
        } else {
          const float y[4] = {v[j][0], v[j][1], v[j][2], v[j][3]};
          if (n < g.N) store_upto<4>(c + n, (int)(g.N - n), y);
        }
      }
    }
  }
}

template <typename T, int OP, bool ERF>
hipError_t launch_small(GemmTile tile, bool aligned, GemmArgs g, hipStream_t s) {
  const bool narrow = tile == TILE_SMALL_NARROW && OP != GEMM_GATED, square = tile == TILE_SMALL_SQUARE;
  if (square && !aligned) return hipErrorInvalidValue;
  const uint32_t n = OP == GEMM_GATED || OP == GEMM_GATED_BWD ? g.pitch : g.N, bm = square ? 64 : 32, bn = OP == GEMM_GATED || narrow ? 32 : 64;
  g.tiles_m = (g.M + bm - 1) / bm;
  g.tiles_n = (n + bn - 1) / bn;
  const uint64_t groups = (uint64_t)g.tiles_m * g.tiles_n * g.workers * g.parts;
  if (!groups) return hipSuccess;
  if (square) return launch_groups(k_ffn_small<T, OP, ERF, 2, 2, 4, true>, groups, 256, g, s);
  if constexpr (OP != GEMM_GATED) {
    if (narrow) return launch_groups(aligned ? k_ffn_small<T, OP, ERF, 1, 1, 8, true> : k_ffn_small<T, OP, ERF, 1, 1, 8, false>, groups, 512, g, s);
  }
  return launch_groups(aligned ? k_ffn_small<T, OP, ERF, 1, 2, 4, true> : k_ffn_small<T, OP, ERF, 1, 2, 4, false>, groups, 256, g, s);
}

}  // namespace evg
