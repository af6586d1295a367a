// The forward products for few tokens: every weight is read once, straight into the matrix cores' fragments.
//
// A workgroup has 16 columns (of gate and of up) and all tokens, up to 16 G; its wavefronts share out k, 128 bytes of each weight row in
// turn, and their sums meet in LDS in a fixed order.  Nothing goes through LDS on the way in: no weight is used twice, and the tokens come
// from the L2.  Bound by memory: what counts is how many loads are under way, so each wavefront asks for up to four steps at once.
#pragma once
#include "ffn_small_device.h"

namespace evg {

__device__ __forceinline__ f32x4 mfma16(const Frag<half_t>& a, const Frag<half_t>& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.v), __builtin_bit_cast(f16x8, b.v), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.v), __builtin_bit_cast(bf16x8, b.v), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(const Frag<float>& a, const Frag<float>& b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.v[i]), __uint_as_float(b.v[i]), c, 0, 0, 0);
  return c;
}

// EIGHT: at most 8 tokens and 8 columns.  The matrix instruction's other 8 rows and columns take the second half of a step's k for the same
// ones, so each of the two 8 x 8 blocks on the diagonal of its result is half of the sum: twice the workgroups, no weight loaded by two lanes,
// and 128 bytes of a row in one load (one token through 2048 x 5632: 10.2 and 6.0 us instead of 12.2 and 8.1).
template <typename T, int OP, bool ERF, int G, int kRowWaves, bool EIGHT>
__global__ __launch_bounds__(kRowWaves * 64) void k_ffn_rows(GemmArgs g) {
  static_assert(!EIGHT || G == 1, "");
  constexpr int E = 16 / sizeof(T), STEP = 128 / sizeof(T), B = OP == GEMM_GATED ? 2 : 1, HALVES = EIGHT ? 1 : 2, COLS = EIGHT ? 8 : 16;
  constexpr int AHEAD = EIGHT ? (B == 2 ? 4 : 6) : G == 1 ? 4 : 2;
  __shared__ f32x4 sums[kRowWaves][B * G][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t block = g.first + blockIdx.x, groups = g.tiles_n, w = block / groups, n0 = block % groups * COLS;
  const int row = lane & (COLS - 1), quarter = lane >> 4, within = quarter * E + (EIGHT ? (lane >> 3 & 1) * (STEP / 2) : 0);   // of a step's k
  // A fragment's lane has 16 bytes of one row.  Rows that there are not read the last one's, and what comes of them is not stored.
  const T* wp[B];
#pragma unroll
  for (int b = 0; b < B; ++b) wp[b] = (const T*)g.b[b].p + (int64_t)w * g.b[b].worker + (int64_t)min(n0 + row, g.N - 1) * g.b[b].ld + within;
  const T* xp[G];
#pragma unroll
  for (int i = 0; i < G; ++i) xp[i] = (const T*)g.a[0].p + (int64_t)w * g.a[0].worker + (int64_t)min(i * 16u + row, g.M - 1) * g.a[0].ld + within;
  f32x4 acc[B][G];
#pragma unroll
  for (int b = 0; b < B; ++b)
#pragma unroll
    for (int i = 0; i < G; ++i) acc[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto load = [](const T* p) {
    Frag<T> f;
    __builtin_memcpy(&f.v, __builtin_assume_aligned(p, sizeof(T)), 16);
    return f;
  };
  const uint32_t whole = g.K / STEP;   // steps
  auto run = [&](uint32_t step, auto count) {   // `count` steps of this wavefront from `step` on
    constexpr int C = decltype(count)::value;
    Frag<T> fw[C][HALVES][B], fx[C][HALVES][G];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint32_t k = (step + c * kRowWaves) * STEP;
#pragma unroll
      for (int half = 0; half < HALVES; ++half) {
#pragma unroll
        for (int b = 0; b < B; ++b) fw[c][half][b] = load(wp[b] + k + half * (STEP / 2));
#pragma unroll
        for (int i = 0; i < G; ++i) fx[c][half][i] = load(xp[i] + k + half * (STEP / 2));
      }
    }
    __builtin_amdgcn_sched_barrier(0);   // all of them are asked for before the first is used
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int half = 0; half < HALVES; ++half)
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
          for (int i = 0; i < G; ++i) acc[b][i] = mfma16(fw[c][half][b], fx[c][half][i], acc[b][i]);
  };
  uint32_t step = wave;
  for (; step + (AHEAD - 1) * kRowWaves < whole; step += AHEAD * kRowWaves) run(step, std::integral_constant<int, AHEAD>{});
  if (AHEAD > 4 && step + 3 * kRowWaves < whole) {
    run(step, std::integral_constant<int, 4>{});
    step += 4 * kRowWaves;
  }
  if (AHEAD > 2 && step + kRowWaves < whole) {
    run(step, std::integral_constant<int, 2>{});
    step += 2 * kRowWaves;
  }
  if (step < whole) {
    run(step, std::integral_constant<int, 1>{});
    step += kRowWaves;
  }
  if (step == whole && g.K % STEP) {   // what is left of k: 16 bytes that reach beyond it are read element by element
#pragma unroll
    for (int half = 0; half < HALVES; ++half) {
      const uint32_t k = whole * STEP + half * (STEP / 2);
      const int left = (int)(g.K - k) - within;
      auto some = [&](const T* p) {
        Frag<T> f;
        f.v = u32x4{0, 0, 0, 0};
        if (left >= E) return load(p + k);
        if (left > 0) {
          T e[E];
#pragma unroll
          for (int j = 0; j < E; ++j) e[j] = j < left ? p[k + j] : (T)0.f;
          __builtin_memcpy(&f.v, e, 16);
        }
        return f;
      };
      Frag<T> fw[B];
#pragma unroll
      for (int b = 0; b < B; ++b) fw[b] = some(wp[b]);
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const Frag<T> fx = some(xp[i]);
#pragma unroll
        for (int b = 0; b < B; ++b) acc[b][i] = mfma16(fw[b], fx, acc[b][i]);
      }
    }
  }

#pragma unroll
  for (int b = 0; b < B; ++b)
#pragma unroll
    for (int i = 0; i < G; ++i) sums[wave][b * G + i][lane] = acc[b][i];
  __syncthreads();
  if (wave >= G || (EIGHT && (lane & 40))) return;
  f32x4 v[B];
#pragma unroll
  for (int b = 0; b < B; ++b) {
    v[b] = sums[0][b * G + wave][lane];
    if (EIGHT) v[b] += sums[0][b * G + wave][lane + 40];   // the other corner: 8 rows and 8 columns on
#pragma unroll
    for (int s = 1; s < kRowWaves; ++s) {
      v[b] += sums[s][b * G + wave][lane];
      if (EIGHT) v[b] += sums[s][b * G + wave][lane + 40];
    }
  }
  // A lane has four neighbouring columns of one token.
  const uint32_t m = wave * 16 + row, n = n0 + quarter * 4;
  if (m >= g.M) return;
  T* const c = (T*)g.c[0].p + (int64_t)w * g.c[0].worker + (int64_t)m * g.c[0].ld + n;
  if constexpr (OP == GEMM_GATED) {
    float gate[4], up[4], h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool real = n + e < g.N;   // the columns up to `pitch` are 0
      gate[e] = real ? v[0][e] : 0.f;
      up[e] = real ? v[1][e] : 0.f;
      float a, slope;
      activate<ERF, sizeof(T) == 2>(g.activation, gate[e], a, slope);
      h[e] = real ? a * up[e] : 0.f;
    }
    store_n<4>(c, h);
    if (g.proj) {
      float* p = proj_at(g, w, m, n, (int)(n >> 3 & 3), (int)((m & 31) + (n >> 2 & 1) * 32));
      *(f32x4*)p = f32x4{gate[0], gate[1], gate[2], gate[3]};
      *(f32x4*)(p + 1024) = f32x4{up[0], up[1], up[2], up[3]};
    }
  } else {
    const float y[4] = {v[0][0], v[0][1], v[0][2], v[0][3]};
    store_upto<4>(c, (int)g.N - (int)n, y);
  }
}

template <typename T, int OP, bool ERF>
hipError_t launch_rows(GemmArgs g, hipStream_t s) {
  const bool eight = g.M <= 8;
  const uint32_t cols = eight ? 8 : 16;
  g.tiles_n = ((OP == GEMM_GATED ? g.pitch : g.N) + cols - 1) / cols;
  const uint64_t groups = (uint64_t)g.tiles_n * g.workers;
  constexpr int waves = OP == GEMM_GATED ? 8 : 16;   // columns of gate and of up, or of one product: as many loads
  if (eight) return launch_groups(k_ffn_rows<T, OP, ERF, 1, waves, true>, groups, waves * 64, g, s);
  if (g.M <= 16) return launch_groups(k_ffn_rows<T, OP, ERF, 1, waves, false>, groups, waves * 64, g, s);
  if (g.M <= 32) return launch_groups(k_ffn_rows<T, OP, ERF, 2, waves, false>, groups, waves * 64, g, s);
  return launch_groups(k_ffn_rows<T, OP, ERF, 4, waves, false>, groups, waves * 64, g, s);
}

template <typename T>
hipError_t launch_any(GemmOp op, GemmTile tile, bool aligned, const GemmArgs& g, hipStream_t s) {
  const bool erf = g.activation.erf;
  if (tile == TILE_ROWS) {
    if (g.M > kMostRows || !g.M) return hipErrorInvalidValue;
    if (op == GEMM_DOWN) return launch_rows<T, GEMM_DOWN, false>(g, s);
    if (op != GEMM_GATED) return hipErrorInvalidValue;
    return erf ? launch_rows<T, GEMM_GATED, true>(g, s) : launch_rows<T, GEMM_GATED, false>(g, s);
  }
  if (tile == TILE_SMALL || tile == TILE_SMALL_NARROW || tile == TILE_SMALL_SQUARE) {
    switch (op) {
      case GEMM_GATED: return erf ? launch_small<T, GEMM_GATED, true>(tile, aligned, g, s) : launch_small<T, GEMM_GATED, false>(tile, aligned, g, s);
      case GEMM_GATED_BWD: return erf ? launch_small<T, GEMM_GATED_BWD, true>(tile, aligned, g, s) : launch_small<T, GEMM_GATED_BWD, false>(tile, aligned, g, s);
      case GEMM_DOWN: return launch_small<T, GEMM_DOWN, false>(tile, aligned, g, s);
      case GEMM_INPUT: return launch_small<T, GEMM_INPUT, false>(tile, aligned, g, s);
      case GEMM_WEIGHT: return launch_small<T, GEMM_WEIGHT, false>(tile, aligned, g, s);
      default: return hipErrorInvalidValue;
    }
  }
  switch (op) {
    case GEMM_GATED: return erf ? launch_op<T, GEMM_GATED, true>(tile, aligned, g, s) : launch_op<T, GEMM_GATED, false>(tile, aligned, g, s);
    case GEMM_GATED_BWD: return erf ? launch_op<T, GEMM_GATED_BWD, true>(tile, aligned, g, s) : launch_op<T, GEMM_GATED_BWD, false>(tile, aligned, g, s);
    case GEMM_DOWN: return launch_op<T, GEMM_DOWN, false>(tile, aligned, g, s);
    case GEMM_INPUT: return launch_op<T, GEMM_INPUT, false>(tile, aligned, g, s);
    case GEMM_WEIGHT: return launch_op<T, GEMM_WEIGHT, false>(tile, aligned, g, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace evg
