// The feed-forward block's matrix products on the matrix cores: one kernel for all types, orders of the operands and epilogues.
//
// C[m][n] = sum_k A(m, k) B(n, k).  An operand is K-contiguous (rows of k) or M/N-contiguous (rows of m or n).  A workgroup has a
// tile of BM x BN; each step of 128 bytes of k (64 elements of 16 bits, 32 of 32) is staged through one of two buffers in LDS, while
// the matrix cores work on the other.  A wavefront has WM x WN of the tile in accumulators of 32 x 32.
//
// The operands of the matrix instruction are swapped (B's fragment first), so that a lane holds four neighbouring n of one m, which
// leave as one store.
#pragma once
#include <type_traits>

#include "ffn_internal.h"
#include "gemm_tile_device.h"
#include "nn_device.h"
#include "../../include/evg_nn.h"

namespace evg {

// An activation a = x s(x) and its slope s + x s'(x).  SiLU and the tanh form of GELU are logistic functions of z = x (c0 + c1 x^2),
// 0.5 (1 + tanh y) = 1 / (1 + exp(-2 y)), and ReLU is the step; GELU itself (ERF) has kernels of its own, as the error function is
// long.  For 16-bit tensors exp and the quotient are the hardware's, a few units of 2^-23 off where s is not vanishing.
template <bool ERF, bool FAST>
__device__ __forceinline__ void activate(const Activation& f, float x, float& a, float& slope) {
  if constexpr (ERF) {
    const float cdf = 0.5f * erfcf(-0.70710678118654752f * x);
    a = x * cdf;
    slope = fmaf(x, 0.39894228040143268f * (FAST ? __expf(-0.5f * x * x) : expf(-0.5f * x * x)), cdf);
  } else {
    const float z = x * fmaf(f.c1 * x, x, f.c0), dz = fmaf(3.f * f.c1 * x, x, f.c0);
    const float e = 1.f + (FAST ? __expf(-z) : expf(-z));   // infinite for z below -88: s is 0 then
    const float s = FAST ? __builtin_amdgcn_rcpf(e) : 1.f / e;
    const float t = s * (1.f - s);
    // Selected, not branched to: branches in the midst of an epilogue cost it a hundred registers.
    const bool off = x <= 0.f;
    a = f.relu ? (off ? 0.f : x) : x * s;
    slope = f.relu ? (off ? 0.f : x > 0.f ? 1.f : x) : t > 0.f ? fmaf(x * dz, t, s) : s;   // far out x dz may be infinite
  }
}

// The projections lie as accumulators hold them: 32 x 32 of gate's, then of up's, each as four times 16 bytes of every lane, so that
// whatever the tile, a wavefront writes and reads 1 KB at a time.  (Row by row the forward product of 8192 tokens, 2048 x 8192, that keeps
// them took 830 us, and the backward one that reads them 808.)
__device__ __forceinline__ float* proj_at(const GemmArgs& g, uint32_t w, uint32_t m, uint32_t n, int q, int lane) {
  return g.proj + w * g.proj_worker + ((uint64_t)(m >> 5) * (g.pitch >> 5) + (n >> 5)) * 2048 + q * 256 + lane * 4;
}

// Large tiles, whose products have many, move them past the caches, which keep the operands instead: forward and backward of 2048 tokens,
// 2048 x 8192, in 675 instead of 762 us, of 8192 in 2245 instead of 2294; where 64 rows are a tile it makes no difference.
template <bool ONCE>
__device__ __forceinline__ void put_proj(float* p, f32x4 v) {
  if constexpr (ONCE) __builtin_nontemporal_store(v, (f32x4*)p);
  else *(f32x4*)p = v;
}
template <bool ONCE>
__device__ __forceinline__ f32x4 get_proj(const float* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load((const f32x4*)p);
  else return *(const f32x4*)p;
}

template <typename T, int OP, bool ERF, int BM, int BN, int WAVES_M, int WAVES_N, bool ALIGNED>
__global__ __launch_bounds__(WAVES_M * WAVES_N * 64, BM == 64 ? 3 : 2) void k_ffn_gemm(GemmArgs g) {
  constexpr bool AKC = OP != GEMM_WEIGHT, BKC = OP == GEMM_GATED || OP == GEMM_DOWN;
  constexpr int WAVES = WAVES_M * WAVES_N, WM = BM / WAVES_M, TM = WM / 32, WN = BN / WAVES_N, TN = WN / 32;
  static_assert(WN % 64 == 0 && WM % 32 == 0, "a wavefront has pairs of accumulators side by side");
  using LA = Tile<T, BM, AKC>;
  using LB = Tile<T, BN, BKC>;
  constexpr int BK = LA::BK;
  constexpr int UNITS = LA::kUnits + LB::kUnits;
  __shared__ u32x4 lds0[UNITS], lds1[UNITS];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Tiles in an order in which neighbours share operands: four rows of tiles, column by column, so that the 32 workgroups of an XCD read
  // four rows' and eight columns' operands at a time (up to 7 % less time for the products of 8192 x 2048 x 8192 than bands of eight
  // rows, 20 % less than of sixteen).
  const uint32_t tiles = g.tiles_m * g.tiles_n;
  uint32_t id = place_by_xcd(g.first);
  const uint32_t cell = id / tiles, part = cell % g.parts, w = cell / g.parts;
  id %= tiles;
  constexpr uint32_t BAND = 4;
  const uint32_t band = BAND * g.tiles_n, first = id / band * BAND, rows = min(BAND, g.tiles_m - first);
  const uint32_t tm = first + id % band % rows, tn = id % band / rows;
  const uint32_t m0 = tm * BM, n0 = tn * (OP == GEMM_GATED ? BN / 2 : BN);

  Loader<T, BM, AKC, WAVES, ALIGNED, false> la;
  Loader<T, BN, BKC, WAVES, ALIGNED, OP == GEMM_GATED> lb;
  static_assert(OP != GEMM_GATED || decltype(lb)::N * 8 == 32, "a wavefront loads rows of one matrix only");
  constexpr int LOADS = decltype(la)::N + decltype(lb)::N;
  u32x4 held[2][ALIGNED ? 1 : LOADS];   // what is loaded into registers, two steps ahead
  const uint32_t steps1 = (g.K + BK - 1) / BK, steps = steps1 * (OP == GEMM_INPUT ? 2 : 1);
  uint32_t fetched = 0;
  int k_left = (int)g.K;
  auto fetch = [&](u32x4* lds, int set) {
    if (OP == GEMM_INPUT && fetched == steps1) {   // the second of the two products
      la.start(g.a[1], w, m0, g.M, g.K, wave, lane);
      lb.start(g.b[1], w, n0, g.N, g.K, wave, lane);
      k_left = (int)g.K;
    }
    la.fetch(k_left, lds, held[set], wave, lane);
    lb.fetch(k_left, lds + LA::kUnits, held[set] + (ALIGNED ? 0 : decltype(la)::N), wave, lane);
    k_left -= BK;
    ++fetched;
  };
  auto put = [&](u32x4* lds, int set) {
    la.put(lds, held[set], wave, lane);
    lb.put(lds + LA::kUnits, held[set] + (ALIGNED ? 0 : decltype(la)::N), wave, lane);
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  const int wm = wave / WAVES_N * WM, wn = wave % WAVES_N * WN;
  // A step's products; fragments are read one step of 32 bytes ahead of them.
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

  if (steps) {   // none: the product is 0
    la.start(g.a[OP == GEMM_WEIGHT ? part : 0], w, m0, g.M, g.K, wave, lane);
    lb.start(g.b[OP == GEMM_GATED ? wave & 1 : 0], w, n0, g.N, g.K, wave, lane);
    fetch(lds0, 0);
    if constexpr (!ALIGNED) {
      fetch(lds1, 1);
      put(lds0, 0);
      __syncthreads();
    }
  }
  for (uint32_t step = 0; step < steps; step += 2) {   // an odd last step is followed by one of zeros
    const bool more = step + 2 < steps;
    if constexpr (ALIGNED) {
      wait_and_meet();
      fetch(lds1, 0);
      multiply(lds0);
      wait_and_meet();
      if (more) fetch(lds0, 0);
      multiply(lds1);
      if (!more) wait_and_meet();   // LDS is free for the results
    } else {
      if (more) fetch(lds0, 0);
      multiply(lds0);
      put(lds1, 1);
      __syncthreads();
      if (more) fetch(lds1, 1);
      multiply(lds1);
      if (more) put(lds0, 0);
      __syncthreads();
    }
  }

  // A lane has, of its row m, four times four neighbouring columns of each accumulator.
  const GemmOperand& co = g.c[OP == GEMM_WEIGHT ? part : 0];
  T* const c = (T*)co.p + (int64_t)w * co.worker;
  // 32 rows of a wavefront's columns leave as rows: 16-bit results go through LDS, so that a store has 64 or 128 bytes of a row at a
  // time instead of 16 (the L2 takes a request for each).  COLS: how many; first: the first of them; v(j, q): a lane's four, rounded.
  auto leave = [&](auto cols, T* to, uint32_t rows0, uint32_t first, uint32_t limit, auto v) {
    constexpr int COLS = decltype(cols)::value;
    if constexpr (sizeof(T) == 2) {
      constexpr int PER = COLS / 8;   // units of a row
      u32x4* const own = lds0 + wave * (32 * 8);
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < COLS / 32; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int row = lane & 31;
          *reinterpret_cast<Pack<T, 4>*>((char*)(own + row * PER + ((j * 4 + q) ^ (row & (PER - 1)))) + (lane >> 5) * 8) = v(j, q);
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int r = 0; r < PER / 2; ++r) {
        const int at = r * 64 + lane, row = at / PER, unit = at % PER;
        const u32x4 x = own[row * PER + (unit ^ (row & (PER - 1)))];
        const uint32_t m = rows0 + row, n = first + unit * 8;
        if (m < g.M && n < limit) {
          T* const p = to + (int64_t)m * co.ld + n;
          if (n + 8 <= limit) {
            __builtin_memcpy(__builtin_assume_aligned(p, sizeof(T)), &x, 16);
          } else {
            T e[8];
            __builtin_memcpy(e, &x, 16);
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (n + i < limit) p[i] = e[i];
          }
        }
      }
    } else {
      const uint32_t m = rows0 + (lane & 31);
      if (m < g.M) {
#pragma unroll
        for (int j = 0; j < COLS / 32; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t n = first + j * 32 + 8 * q + 4 * (lane >> 5);
            const Pack<T, 4> x = v(j, q);
            store_upto<4>(to + (int64_t)m * co.ld + n, n < limit ? (int)(limit - n) : 0, x.v);
          }
      }
    }
  };
  using Cols = std::integral_constant<int, OP == GEMM_GATED ? WN / 2 : WN>;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const uint32_t rows0 = m0 + wm + i * 32;
    if (rows0 >= g.M) break;
    if constexpr (OP == GEMM_GATED) {
      const uint32_t first = n0 + (wn >> 1);
      Pack<T, 4> h[TN / 2][4];
#pragma unroll
      for (int j = 0; j < TN / 2; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t n = first + j * 32 + 8 * q + 4 * (lane >> 5);
          f32x4 gate, up;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool real = n + e < g.N;     // the columns up to `pitch` are 0
            gate[e] = real ? acc[i][2 * j][q * 4 + e] : 0.f;
            up[e] = real ? acc[i][2 * j + 1][q * 4 + e] : 0.f;
            float a, slope;
            activate<ERF, sizeof(T) == 2>(g.activation, gate[e], a, slope);
            h[j][q].v[e] = from_f<T>(real ? a * up[e] : 0.f);
          }
          if (g.proj && n < g.pitch) {
            float* p = proj_at(g, w, rows0, n, q, lane);
            put_proj<(BM >= 128)>(p, gate);
            put_proj<(BM >= 128)>(p + 1024, up);
          }
        }
      leave(Cols{}, c, rows0, first, g.pitch, [&](int j, int q) { return h[j][q]; });
    } else if constexpr (OP == GEMM_GATED_BWD) {
      // The projections of 32 x 32 at once, all asked for before the first is used; what lies beyond the tensors reads its last block's.
      const uint32_t first = n0 + wn;
      Pack<T, 4> dg[TN][4], du[TN][4];
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        f32x4 gate[4], up[4];
        const float* p = proj_at(g, w, rows0, min(first + j * 32, g.pitch - 32), 0, lane);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          gate[q] = get_proj<(BM >= 128)>(p + q * 256);
          up[q] = get_proj<(BM >= 128)>(p + 1024 + q * 256);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t n = first + j * 32 + 8 * q + 4 * (lane >> 5);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float a, slope;
            activate<ERF, sizeof(T) == 2>(g.activation, gate[q][e], a, slope);
            const float d = acc[i][j][q * 4 + e];
            const bool real = n + e < g.N;
            dg[j][q].v[e] = from_f<T>(real ? d * up[q][e] * slope : 0.f);
            du[j][q].v[e] = from_f<T>(real ? d * a : 0.f);
          }
          __builtin_amdgcn_sched_barrier(0);   // four at a time: more would take the registers of a second workgroup
        }
      }
      leave(Cols{}, c, rows0, first, g.pitch, [&](int j, int q) { return dg[j][q]; });
      leave(Cols{}, c + g.pitch, rows0, first, g.pitch, [&](int j, int q) { return du[j][q]; });
    } else {
      leave(Cols{}, c, rows0, n0 + wn, g.N, [&](int j, int q) {
        Pack<T, 4> x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x.v[e] = from_f<T>(acc[i][j][q * 4 + e]);
        return x;
      });
    }
  }
}

template <typename Kernel>
hipError_t launch_groups(Kernel kernel, uint64_t groups, uint32_t threads, GemmArgs g, hipStream_t s) {
  if (groups > 0x7FFFFFFFull) return hipErrorInvalidValue;
  launch_pieces(groups, threads, [&](uint32_t first, uint32_t grid) {
    g.first = first;
    kernel<<<grid, threads, 0, s>>>(g);
  });
  return hipGetLastError();
}

template <typename T, int OP, bool ERF>
hipError_t launch_op(GemmTile tile, bool aligned, GemmArgs g, hipStream_t s) {
  constexpr uint32_t share = OP == GEMM_GATED ? 2 : 1;   // a tile's columns are gate's and up's
  const uint32_t bm = tile == TILE_256 ? 256 : tile == TILE_128 ? 128 : 64, bn = (tile == TILE_256 ? 256 : 128) / share;
  g.tiles_m = (g.M + bm - 1) / bm;
  // padding columns are written too where there are any
  const uint32_t n = OP == GEMM_GATED || OP == GEMM_GATED_BWD ? g.pitch : g.N;
  g.tiles_n = (n + bn - 1) / bn;
  const uint64_t groups = (uint64_t)g.tiles_m * g.tiles_n * g.workers * g.parts;
  if (!groups) return hipSuccess;
  if constexpr (sizeof(T) == 2) {
    if constexpr (OP != GEMM_GATED_BWD) {   // which overlaps its reading and writing with a second workgroup's products
      if (aligned && tile == TILE_256) return launch_groups(k_ffn_gemm<T, OP, ERF, 256, 256, 2, 4, true>, groups, 512, g, s);
    }
    if (aligned && tile == TILE_128) return launch_groups(k_ffn_gemm<T, OP, ERF, 128, 128, 2, 2, true>, groups, 256, g, s);
  }
  if (tile != TILE_64) return hipErrorInvalidValue;
  return launch_groups(aligned ? k_ffn_gemm<T, OP, ERF, 64, 128, 2, 2, true> : k_ffn_gemm<T, OP, ERF, 64, 128, 2, 2, false>, groups, 256, g, s);
}

}  // namespace evg
