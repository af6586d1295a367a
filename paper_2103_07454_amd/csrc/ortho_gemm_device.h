// The products of orthogonal updates on the matrix cores: float16 operands, sums in 32 bits.
//
// C[m][n] = f_acc sum_k A(m, k) B(n, k) + f_own own[m][n].  Tiles, their ways through LDS and the order of a lane's results are those of
// gemm_tile_device.h.  SPLIT: operands are hi + lo; the product is that of hi and hi, of hi and lo and of lo and hi, one after the other into the same
// accumulators (lo and lo is 2^-22 of it and left out).
//
// S and P are symmetric: tiles below the diagonal are not computed, those above it are written twice, the second time turned round.
#pragma once
#include <type_traits>

#include "gemm_tile_device.h"
#include "ortho_internal.h"

namespace evg {

// Which tile of a symmetric product: bands of four rows of tiles, each from its diagonal on, column by column.
__device__ __forceinline__ void symmetric_tile(uint32_t id, uint32_t tiles, uint32_t* tm, uint32_t* tn) {
  uint32_t first = 0;
  for (;;) {
    const uint32_t rows = min(4u, tiles - first), cells = rows * (tiles - first);
    if (id < cells) {
      *tm = first + id % rows;
      *tn = first + id / rows;
      return;
    }
    id -= cells;
    first += 4;
  }
}

template <int OP, bool TALL, bool SPLIT, bool LAST, int BM, int BN, int WAVES_M, int WAVES_N>
__global__ __launch_bounds__(WAVES_M * WAVES_N * 64, BM == 64 ? 3 : 2) void k_ortho_gemm(OrthoArgs g) {
  typedef half_t T;
  constexpr bool SYMMETRIC = OP != ORTHO_APPLY;
  constexpr bool AKC = !(OP == ORTHO_GRAM && TALL), BKC = OP == ORTHO_SQUARE || (OP == ORTHO_GRAM ? !TALL : TALL);
  constexpr int WAVES = WAVES_M * WAVES_N, WM = BM / WAVES_M, TM = WM / 32, WN = BN / WAVES_N, TN = WN / 32;
  using LA = Tile<T, BM, AKC>;
  using LB = Tile<T, BN, BKC>;
  constexpr int BK = LA::BK;
  constexpr int UNITS = LA::kUnits + LB::kUnits;
  __shared__ u32x4 lds0[UNITS], lds1[UNITS];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t id = place_by_xcd(g.first);
  const uint32_t w = id / g.cells;
  id %= g.cells;
  uint32_t tm, tn;
  if constexpr (SYMMETRIC) {
    symmetric_tile(id, g.tiles_m, &tm, &tn);
    if (tn < tm) return;
  } else {
    constexpr uint32_t BAND = 4;
    const uint32_t band = BAND * g.tiles_n, first = id / band * BAND, rows = min(BAND, g.tiles_m - first);
    tm = first + id % band % rows, tn = id % band / rows;
  }
  const uint32_t m0 = tm * BM, n0 = tn * BN;

  Loader<T, BM, AKC, WAVES, true, false> la;
  Loader<T, BN, BKC, WAVES, true, false> lb;
  const uint32_t steps1 = (g.K + BK - 1) / BK, steps = steps1 * (SPLIT ? 3 : 1);
  constexpr uint32_t PRODUCTS = SPLIT ? 3 : 1;
  uint32_t left = steps1, product = 0;
  int k_left = (int)g.K;
  auto start = [&] {
    la.start({SPLIT && product == 2 ? g.a.lo : g.a.hi, g.a.worker, g.a.ld}, w, m0, g.M, g.K, wave, lane);
    lb.start({SPLIT && product == 1 ? g.b.lo : g.b.hi, g.b.worker, g.b.ld}, w, n0, g.N, g.K, wave, lane);
  };
  auto fetch = [&](u32x4* lds) {
    if constexpr (SPLIT) {
      if (left == 0 && product + 1 < PRODUCTS) {   // the next of the products
        ++product;
        start();
        k_left = (int)g.K;
        left = steps1;
      }
      --left;
    }
    la.fetch(k_left, lds, nullptr, wave, lane);
    lb.fetch(k_left, lds + LA::kUnits, nullptr, wave, lane);
    k_left -= BK;
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  const int wm = wave / WAVES_N * WM, wn = wave % WAVES_N * WN;
  auto multiply = [&](const u32x4* lds) {
    Frag<T> a[2][TM], b[2][TN];
    auto read = [&](int ks) {
#pragma unroll
      for (int j = 0; j < TN; ++j) b[ks & 1][j] = read_frag<T, BN, BKC>(lds, LA::kUnits, wn + j * 32, ks, lane);
#pragma unroll
      for (int i = 0; i < TM; ++i) a[ks & 1][i] = read_frag<T, BM, AKC>(lds, 0, wm + i * 32, ks, lane);
    };
    read(0);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      if (ks < 3) read(ks + 1);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mfma(b[ks & 1][j], a[ks & 1][i], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  start();
  fetch(lds0);
  for (uint32_t step = 0; step < steps; step += 2) {   // an odd last step is followed by one of zeros
    const bool more = step + 2 < steps;
    wait_and_meet();
    fetch(lds1);
    multiply(lds0);
    wait_and_meet();
    if (more) fetch(lds0);
    multiply(lds1);
    if (!more) wait_and_meet();   // LDS is free for the results
  }

  // A lane has, of its row m, four times four neighbouring columns of each accumulator.  32 rows of a wavefront's columns at a time.
  constexpr int PER = WN / 8;   // 16-byte units of a row
  u32x4* const room = lds0 + wave * (32 * PER);
  const uint32_t limit = (g.N + 7) & ~7u;   // columns up to a whole unit are 0
  auto leave = [&](uint16_t* to, uint32_t rows0, auto v) {
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = lane & 31;
        *reinterpret_cast<Pack<T, 4>*>((char*)(room + row * PER + ((j * 4 + q) ^ (row & (PER - 1)))) + (lane >> 5) * 8) = v(j, q);
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int r = 0; r < PER / 2; ++r) {
      const int at = r * 64 + lane, row = at / PER, unit = at % PER;
      const u32x4 x = room[row * PER + (unit ^ (row & (PER - 1)))];
      const uint32_t m = rows0 + row, n = n0 + wn + unit * 8;
      if (m < g.M && n < limit) *(u32x4*)(to + (int64_t)m * g.to.ld + n) = x;
    }
  };
  // The same 32 rows as columns: rows of 64 bytes.
  auto leave_turned = [&](uint16_t* to, uint32_t rows0, auto v) {
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const Pack<T, 4> x = v(j, q);
#pragma unroll
        for (int e = 0; e < 4; ++e) ((T*)room)[(j * 32 + 8 * q + 4 * (lane >> 5) + e) * 32 + (lane & 31)] = x.v[e];
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int r = 0; r < WN / 16; ++r) {
      const int at = r * 64 + lane, row = at / 4, unit = at % 4;
      const u32x4 x = room[at];
      const uint32_t n = n0 + wn + row, m = rows0 + unit * 8;
      // Turned tiles lie below the diagonal: their columns are all real.
      if (n < g.N) *(u32x4*)(to + (int64_t)n * g.to.ld + m) = x;
    }
  };
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const uint32_t rows0 = m0 + wm + i * 32, m = rows0 + (lane & 31);
    if (rows0 >= g.M) break;
    f32x4 v[TN][4];
    Pack<T, 4> hi[TN][4], lo[TN][4];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t n = n0 + wn + j * 32 + 8 * q + 4 * (lane >> 5);
        f32x4 own = {0.f, 0.f, 0.f, 0.f};
        if constexpr (OP != ORTHO_GRAM) {
          if (m < g.M && n < limit) {
            const int64_t at = (int64_t)w * g.own.worker + (int64_t)m * g.own.ld + n;
            const Pack<T, 4> h = *reinterpret_cast<const Pack<T, 4>*>(g.own.hi + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) own[e] = to_f(h.v[e]);
            if (SPLIT || OP == ORTHO_APPLY) {
              const Pack<T, 4> l = *reinterpret_cast<const Pack<T, 4>*>(g.own.lo + at);
#pragma unroll
              for (int e = 0; e < 4; ++e) own[e] += to_f(l.v[e]);
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = acc[i][j][q * 4 + e] * g.f_acc;
          v[j][q][e] = OP == ORTHO_GRAM ? p : fmaf(own[e], g.f_own, p);
          if constexpr (!LAST) halves_of(v[j][q][e], &hi[j][q].v[e], &lo[j][q].v[e]);
        }
      }
    if constexpr (LAST) {
      if (m < g.M) {
        const int64_t row = (int64_t)w * g.out.worker + (int64_t)m * g.out.row;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t n = n0 + wn + j * 32 + 8 * q + 4 * (lane >> 5);
            const float x[4] = {v[j][q][0], v[j][q][1], v[j][q][2], v[j][q][3]};
            const int count = n < g.N ? (int)(g.N - n) : 0;
            if (g.out_type == EVG_F32) store_upto<4>((float*)g.out.p + row + n, count, x);
            else if (g.out_type == EVG_F16) store_upto<4>((half_t*)g.out.p + row + n, count, x);
            else store_upto<4>((bf16_t*)g.out.p + row + n, count, x);
          }
      }
    } else {
      const int64_t to = (int64_t)w * g.to.worker;
      leave(g.to.hi + to, rows0, [&](int j, int q) { return hi[j][q]; });
      if (SPLIT || OP == ORTHO_APPLY) leave(g.to.lo + to, rows0, [&](int j, int q) { return lo[j][q]; });
      if (SYMMETRIC && tm != tn) {
        leave_turned(g.to.hi + to, rows0, [&](int j, int q) { return hi[j][q]; });
        if (SPLIT) leave_turned(g.to.lo + to, rows0, [&](int j, int q) { return lo[j][q]; });
      }
    }
  }
}

template <int OP, bool TALL, bool SPLIT, bool LAST, int BM, int WAVES_M, int WAVES_N>
hipError_t launch_ortho_tile(OrthoArgs a, hipStream_t s) {
  a.tiles_m = (a.M + BM - 1) / BM;
  a.tiles_n = (a.N + BM - 1) / BM;
  uint64_t cells = (uint64_t)a.tiles_m * a.tiles_n;
  if (OP != ORTHO_APPLY) {
    cells = 0;
    for (uint32_t first = 0; first < a.tiles_m; first += 4) cells += (uint64_t)(a.tiles_m - first < 4 ? a.tiles_m - first : 4) * (a.tiles_m - first);
  }
  a.cells = (uint32_t)cells;
  const uint64_t groups = cells * a.matrices;
  if (groups > 0x7FFFFFFFull) return hipErrorInvalidValue;
  launch_pieces(groups, WAVES_M * WAVES_N * 64, [&](uint32_t first, uint32_t grid) {
    a.first = first;
    k_ortho_gemm<OP, TALL, SPLIT, LAST, BM, BM, WAVES_M, WAVES_N><<<grid, WAVES_M * WAVES_N * 64, 0, s>>>(a);
  });
  return hipGetLastError();
}

// The tile with the least time by what a step of 64 of k of a round of workgroups takes.
template <int OP, bool TALL, bool SPLIT, bool LAST>
hipError_t launch_ortho_op(const OrthoArgs& a, hipStream_t s) {
  auto count = [&](uint32_t b) {
    const uint64_t m = (a.M + b - 1) / b, n = (a.N + b - 1) / b;
    return (OP == ORTHO_APPLY ? m * n : m * (m + 1) / 2) * a.matrices;
  };
  auto rounds = [](uint64_t c, uint64_t slots) { return (double)((c + slots - 1) / slots); };
  const double t256 = rounds(count(256), 256) * 1.29, t128 = rounds(count(128), 512) * 1.04, t64 = rounds(count(64), 768) * 0.7;
  if (t64 <= t128 && t64 <= t256) return launch_ortho_tile<OP, TALL, SPLIT, LAST, 64, 2, 2>(a, s);
  if (t128 <= t256) return launch_ortho_tile<OP, TALL, SPLIT, LAST, 128, 2, 2>(a, s);
  return launch_ortho_tile<OP, TALL, SPLIT, LAST, 256, 2, 4>(a, s);
}

template <bool SPLIT>
hipError_t launch_ortho_any(OrthoOp op, bool tall, bool last, const OrthoArgs& a, hipStream_t s) {
  if (op == ORTHO_GRAM) return tall ? launch_ortho_op<ORTHO_GRAM, true, SPLIT, false>(a, s) : launch_ortho_op<ORTHO_GRAM, false, SPLIT, false>(a, s);
  if (op == ORTHO_SQUARE) return launch_ortho_op<ORTHO_SQUARE, false, SPLIT, false>(a, s);
  if (last) return tall ? launch_ortho_op<ORTHO_APPLY, true, SPLIT, true>(a, s) : launch_ortho_op<ORTHO_APPLY, false, SPLIT, true>(a, s);
  return tall ? launch_ortho_op<ORTHO_APPLY, true, SPLIT, false>(a, s) : launch_ortho_op<ORTHO_APPLY, false, SPLIT, false>(a, s);
}

}  // namespace evg
