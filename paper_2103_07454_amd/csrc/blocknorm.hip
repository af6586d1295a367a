// Norms before and after a block with its gate and residual scale, and their backward pass (include/evg_nn.h, evg_blocknorm_*).
//
// With the unit rows  ub = (b - mean_b) / s_b  and  ur = (r' - mean_r) / s_r  (RMS: no means),  after = ub * post + post_bias:
//     r' = alpha r + beta gate after,    n = ur * pre + pre_bias
// and, with q = dn * pre and p = da * post:
//     dr = dr' + (q - mean(q) - ur mean(q ur)) / s_r           (RMS: no mean(q))
//     d_residual = alpha dr,   d_gate = beta dr after summed over the rows that share it,   da = beta gate dr
//     d_branch = (p - mean(p) - ub mean(p ub)) / s_b           (da itself without post)
//     d_pre = sum dn ur,  d_pre_bias = sum dn,  d_post = sum da ub,  d_post_bias = sum da     over a worker's rows
// The backward pass makes both norms anew from residual and branch: nothing has to be kept, and r' is not read in rounded form.
// A mean in 32 bits is off by units of where the row lies, which may be more than its spread.  The differences from it are exact where that is so;
// what they still add up to, delta a value, is summed beside their squares and taken back: from the row, from the variance (mean of squares
// - delta^2) and from sums of products with the row.  Rows of 1e4 with a spread of 0.05 were off by 1e-2 without.
//
// Both passes are bound by memory.  A row stays in the registers of 16 to 1024 threads (64 and more in the backward pass), 8 or 16 elements
// of each tensor in a thread, so that each tensor is read once; the sums over a row go through the wavefront and one exchange in LDS.
// Several narrow rows to a wavefront: 11 x 5331 rows of 64 forward in 17 instead of 36 us, 8000 of 256 in 7 instead of 10.
#include <hip/hip_runtime.h>

#include <cmath>
#include <exception>
#include <new>
#include <type_traits>

#include "nn_device.h"
#include "nn_host.h"

namespace evg {
namespace {

constexpr int kV = 8;                    // elements of a thread that lie together

struct NormArgs {
  evg_blocknorm_in in;
  evg_mat out, normed;                   // forward
  evg_mat d_out, d_normed;               // backward
  evg_blocknorm_grads d;
  uint32_t width, workers;
  float eps, alpha, beta, inv_width;
  // backward: stripes of rows
  uint32_t stripes, stripe_rows;         // of a worker
  uint32_t group_stripes;                // stripes of a gate's group; 0: a stripe has whole groups
  float* partials;                       // [workers][stripes][slots][padded width]: pre, pre_bias, post, post_bias, gate; RMS: no biases
  uint32_t slots;
  uint32_t padded;
  uint32_t first;                        // workgroup of a launch in pieces
};

// Rows of sums that a stripe leaves: of both weights, the gate and a layer norm's biases.
__host__ __device__ constexpr uint32_t slots_of(bool layer) { return layer ? 5 : 3; }

template <typename T>
__device__ __forceinline__ T* at(const evg_mat& m, uint32_t w, uint64_t row) {
  return (T*)m.p + (int64_t)w * m.worker + (int64_t)row * m.row;
}

template <int TPR> constexpr int kRowWaves = TPR < 64 ? 1 : TPR / 64;   // that share a row

// The sums of two or three values over the threads that share a row.  `red` alternates between two sets, so one barrier is enough.
constexpr int kSums = 3;
// All sums of many wavefronts are more than a layer norm's kernels have registers for: there each lane takes one wavefront's, and the lanes add them up
// (8192 rows of 4096 bf16, norm after the block, no gate, backward 119 instead of 153 us; two sums of 8 are faster read by every lane, 90 and 97).
template <int TPR, bool LAYER, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*red)[kSums][kRowWaves<TPR>], int& turn) {
  static_assert(N <= kSums, "");
  if constexpr (TPR < 64) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = lanes_sum<16>(v[n]);
    if constexpr (TPR == 32)
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] += __shfl_xor(v[n], 16);
    return;
  }
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = wave_sum_uniform(v[n]);
  if constexpr (TPR > 64) {
    float(&set)[kSums][kRowWaves<TPR>] = red[turn];
    turn ^= 1;
    const int wave = threadIdx.x % TPR / 64;
    if (threadIdx.x % 64 == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) set[n][wave] = v[n];
    __syncthreads();
    constexpr int W = TPR / 64;
    if constexpr (LAYER && W >= (N == 3 ? 4 : 16)) {
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] = lanes_sum<W>(set[n][threadIdx.x % W]);
      return;
    }
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = set[n][0];
#pragma unroll
    for (int i = 1; i < W; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] += set[n][i];
  }
}

template <int NV> struct Row { float v[NV * kV]; };

// Where a lane's 8 elements of a row of at least 8 begin, and how many of them belong to its neighbour: one that has fewer reads the row's
// last 8, one that has none the first.  So every lane loads 16 bytes, without a branch between one tensor's loads and the next one's.
struct Place { int at, skip; bool any; };
__device__ __forceinline__ Place place_of(int c, int width) {
  const bool any = c < width, whole = c + kV <= width;
  return {whole ? c : any ? width - kV : 0, any && !whole ? c + kV - width : 0, any};
}

// Elements beyond the width are 0.
template <int NV, int TPR, typename T>
__device__ __forceinline__ void load_row(const T* p, int width, int lane, Row<NV>& r) {
  if (width >= kV) {
    Place at[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      at[k] = place_of((k * TPR + lane) * kV, width);
      load_n<kV>(p + at[k].at, r.v + k * kV);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float* v = r.v + k * kV;
      if (width % kV) {
#pragma unroll
        for (int s = 1; s < kV; s *= 2)
#pragma unroll
          for (int i = 0; i < kV; ++i) v[i] = at[k].skip & s ? (i + s < kV ? v[i + s] : 0.f) : v[i];
      }
#pragma unroll
      for (int i = 0; i < kV; ++i) v[i] = at[k].any ? v[i] : 0.f;
    }
  } else {
#pragma unroll
    for (int k = 0; k < NV; ++k) load_upto<kV>(p, lane || k ? 0 : width, r.v + k * kV);
  }
}

template <int NV, int TPR, typename T>
__device__ __forceinline__ void store_row(T* p, int width, int lane, const Row<NV>& r) {
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * TPR + lane) * kV;
    store_upto<kV>(p + c, width - c, r.v + k * kV);
  }
}

// The sum over the width, rounded once where the mean has no more bits than fit: the quotient by the rounded reciprocal, and what its product
// leaves of the sum.
__device__ __forceinline__ float mean_of(float sum, const NormArgs& g) {
  const float q = sum * g.inv_width;
  return fmaf(fmaf(-q, (float)g.width, sum), g.inv_width, q);
}

// From the mean of the squares about a mean that is off by delta.  A NaN stays one.
template <bool LAYER>
__device__ __forceinline__ float variance(float squares, float delta) {
  if (!LAYER) return squares;
  const float v = fmaf(-delta, delta, squares);
  return v < 0.f ? 0.f : v;
}

// x becomes its unit row; what is beyond the width is 0 (RMS) or finite where the row is (it meets weights of 0).  Returns 1 / s.
template <int NV, int TPR, bool LAYER, typename R>
__device__ __forceinline__ float make_unit(Row<NV>& x, const NormArgs& g, int lane, R red, int& turn) {
  if constexpr (LAYER) {
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV * kV; ++i) s[0] += x.v[i];
    row_sums<TPR, LAYER>(s, red, turn);
    const float mean = mean_of(s[0], g);
#pragma unroll
    for (int i = 0; i < NV * kV; ++i) x.v[i] = ((i / kV) * TPR + lane) * kV + i % kV < (int)g.width ? x.v[i] - mean : 0.f;
  }
  float s[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NV * kV; ++i) {
    s[0] = fmaf(x.v[i], x.v[i], s[0]);
    if (LAYER) s[1] += x.v[i];
  }
  row_sums<TPR, LAYER>(s, red, turn);
  const float delta = LAYER ? s[1] * g.inv_width : 0.f;
  const float inv = 1.f / sqrtf(variance<LAYER>(s[0] * g.inv_width, delta) + g.eps);
#pragma unroll
  for (int i = 0; i < NV * kV; ++i) x.v[i] = LAYER ? fmaf(x.v[i], inv, -delta * inv) : x.v[i] * inv;
  return inv;
}

template <typename T, int NV, int TPR, bool LAYER>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_blocknorm_forward(NormArgs g) {
  constexpr int ROWS = TPR < 256 ? 256 / TPR : 1;   // rows of a workgroup
  __shared__ float shared[ROWS][2][kSums][kRowWaves<TPR>];
  int turn = 0;
  const int lane = threadIdx.x % TPR;
  float(*red)[kSums][kRowWaves<TPR>] = shared[threadIdx.x / TPR];
  const uint64_t row0 = ((uint64_t)g.first + blockIdx.x) * ROWS + threadIdx.x / TPR, all = (uint64_t)g.workers * g.in.rows;
  const bool real = row0 < all;
  const uint64_t row = real ? row0 : all - 1;       // all threads of a workgroup meet at its barriers
  const uint32_t w = (uint32_t)(row / g.in.rows), t = (uint32_t)(row % g.in.rows);
  const int width = (int)g.width;
  Row<NV> r;
  load_row<NV, TPR>(at<const T>(g.in.residual, w, t), width, lane, r);
  if (g.in.branch.p) {
    Row<NV> b, k;
    load_row<NV, TPR>(at<const T>(g.in.branch, w, t), width, lane, b);
    if (g.in.post.p) {
      make_unit<NV, TPR, LAYER>(b, g, lane, red, turn);
      load_row<NV, TPR>(at<const T>(g.in.post, w, 0), width, lane, k);
#pragma unroll
      for (int i = 0; i < NV * kV; ++i) b.v[i] *= k.v[i];
      if (LAYER && g.in.post_bias.p) {
        load_row<NV, TPR>(at<const T>(g.in.post_bias, w, 0), width, lane, k);
#pragma unroll
        for (int i = 0; i < NV * kV; ++i) b.v[i] += k.v[i];
      }
    }
    if (g.in.gate.p) {
      load_row<NV, TPR>(at<const T>(g.in.gate, w, t / g.in.gate_rows), width, lane, k);
#pragma unroll
      for (int i = 0; i < NV * kV; ++i) b.v[i] *= k.v[i];
    }
#pragma unroll
    for (int i = 0; i < NV * kV; ++i) r.v[i] = fmaf(g.alpha, r.v[i], g.beta * b.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < NV * kV; ++i) r.v[i] *= g.alpha;
  }
  if (g.out.p && real) store_row<NV, TPR>(at<T>(g.out, w, t), width, lane, r);
  if (!g.normed.p) return;
  make_unit<NV, TPR, LAYER>(r, g, lane, red, turn);
  Row<NV> k;
  load_row<NV, TPR>(at<const T>(g.in.pre, w, 0), width, lane, k);
#pragma unroll
  for (int i = 0; i < NV * kV; ++i) r.v[i] *= k.v[i];
  if (LAYER && g.in.pre_bias.p) {
    load_row<NV, TPR>(at<const T>(g.in.pre_bias, w, 0), width, lane, k);
#pragma unroll
    for (int i = 0; i < NV * kV; ++i) r.v[i] += k.v[i];
  }
  if (real) store_row<NV, TPR>(at<T>(g.normed, w, t), width, lane, r);
}

// A thread's part of a row as it lies in memory, in whole registers (two 16-bit elements to each).
template <typename T, int NV> struct Raw { uint32_t w[NV][kV * sizeof(T) / 4]; int skip[NV]; };

template <typename T>
__device__ __forceinline__ float element(const uint32_t* w, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
  else if constexpr (std::is_same_v<T, bf16_t>) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  else return (float)__builtin_bit_cast(half_t, (uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu));
}

// WHOLE: the width is a multiple of 8, so a lane has 8 elements or none.  ONCE: they go past the caches.
template <bool WHOLE, int NV, int TPR, bool ONCE = false, typename T>
__device__ __forceinline__ void load_raw(const T* p, int width, int lane, Raw<T, NV>& r) {
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * TPR + lane) * kV;
    constexpr int N = kV * sizeof(T) / 4;
    if (WHOLE || width >= kV) {
      const Place at = place_of(c, width);
      typedef uint32_t words __attribute__((ext_vector_type(N), aligned(sizeof(T))));
      const words* from = reinterpret_cast<const words*>(p + (WHOLE && !at.any ? 0 : at.at));
      const words x = ONCE ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
      for (int i = 0; i < N; ++i) r.w[k][i] = x[i];
      if (!WHOLE) r.skip[k] = at.skip;
    } else {
      T e[kV];
#pragma unroll
      for (int i = 0; i < kV; ++i) e[i] = c + i < width ? p[c + i] : (T)0.f;
      __builtin_memcpy(r.w[k], e, sizeof e);
      r.skip[k] = 0;
    }
  }
}

// As values; those beyond the width are 0.  The empty statement keeps the compiler from making them long before they are needed, which
// would take twice the registers.
template <bool WHOLE, int NV, int TPR, typename T>
__device__ __forceinline__ void unpack(Raw<T, NV>& r, int width, int lane, Row<NV>& x) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < kV / 2; ++i) asm volatile("" : "+v"(r.w[k][i]));
  }
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < kV; ++i) x.v[k * kV + i] = (k * TPR + lane) * kV < width ? element<T>(r.w[k], i) : 0.f;
  if constexpr (!WHOLE) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float* v = x.v + k * kV;
#pragma unroll
      for (int s = 1; s < kV; s *= 2)
#pragma unroll
        for (int i = 0; i < kV; ++i) v[i] = r.skip[k] & s ? (i + s < kV ? v[i + s] : 0.f) : v[i];
    }
  }
}

template <bool WHOLE, int NV, int TPR, bool ONCE = false, typename T>
__device__ __forceinline__ void put_row(T* p, int width, int lane, const Row<NV>& r) {
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * TPR + lane) * kV;
    if (WHOLE) {
      if (c < width) { if (ONCE) store_n_once<kV>(p + c, r.v + k * kV); else store_n<kV>(p + c, r.v + k * kV); }
    } else {
      store_upto<kV>(p + c, width - c, r.v + k * kV);
    }
  }
}

// A tensor's rows in their order.
template <typename T> struct Lines {
  T* p;
  int64_t row;
  __device__ __forceinline__ Lines(const evg_mat& m, uint32_t w, uint32_t t) : p(m.p ? at<T>(m, w, t) : nullptr), row(m.row) {}
  __device__ __forceinline__ void next() { p += row; }
};

// One stripe of a worker's rows: the rows' gradients, and the stripe's share of the weights' and the gate's.  GATED, POST: whether
// there is a gate and a norm after the block; -1: as the arguments say (widths that are no multiple of 8).
template <typename T, int NV, int TPR, bool LAYER, int GATED, int POST>
__global__ __launch_bounds__(TPR) void k_blocknorm_backward(NormArgs g) {
  constexpr bool WHOLE = GATED >= 0;
  __shared__ float red[2][kSums][TPR / 64];
  int turn = 0;
  const int lane = threadIdx.x;
  const uint32_t block = g.first + blockIdx.x, w = block / g.stripes, stripe = block % g.stripes;
  const int width = (int)g.width;
  uint32_t t0, t1;
  if (g.group_stripes) {
    const uint32_t group = stripe / g.group_stripes, end = min((uint64_t)g.in.rows, (uint64_t)(group + 1) * g.in.gate_rows);
    t0 = min(end, group * g.in.gate_rows + stripe % g.group_stripes * g.stripe_rows);
    t1 = min(end, t0 + g.stripe_rows);
  } else {
    t0 = min(g.in.rows, stripe * g.stripe_rows);
    t1 = min(g.in.rows, t0 + g.stripe_rows);
  }
  constexpr int N = NV * kV;
  const bool branch = g.in.branch.p, pre = g.d_normed.p, direct = g.d_out.p;
  const bool gated = GATED >= 0 ? GATED : g.in.gate.p != nullptr, post = POST >= 0 ? POST : g.in.post.p != nullptr;
  const bool post_bias = LAYER && g.in.post_bias.p;
  Raw<T, NV> w_post, w_postbias, w_pre;
  if (post) load_raw<WHOLE, NV, TPR>(at<const T>(g.in.post, w, 0), width, lane, w_post);
  if (post_bias) load_raw<WHOLE, NV, TPR>(at<const T>(g.in.post_bias, w, 0), width, lane, w_postbias);
  if (pre) load_raw<WHOLE, NV, TPR>(at<const T>(g.in.pre, w, 0), width, lane, w_pre);
  Row<NV> s_pre, s_prebias, s_post, s_postbias, s_gate;
#pragma unroll
  for (int i = 0; i < N; ++i) s_pre.v[i] = s_prebias.v[i] = s_post.v[i] = s_postbias.v[i] = s_gate.v[i] = 0.f;

  Lines<const T> l_r(g.in.residual, w, t0), l_b(g.in.branch, w, t0), l_dn(g.d_normed, w, t0), l_do(g.d_out, w, t0);
  Lines<T> o_r(g.d.residual, w, t0), o_b(g.d.branch, w, t0);
  uint32_t gate_row = gated ? t0 / g.in.gate_rows : 0, until = gated ? (uint32_t)min((uint64_t)g.in.rows, (uint64_t)(gate_row + 1) * g.in.gate_rows) : 0;
  const float alpha = g.alpha, beta = g.beta, inv_width = g.inv_width;
  // The next row's residual and branch, which its first sums need, are on their way while a row is finished, where a thread has 8 elements of it
  // (of 16 there are no registers for them).
  constexpr bool AHEAD = NV == 1;
  Raw<T, NV> n_r, n_b;
  auto ask = [&]() {
    load_raw<WHOLE, NV, TPR, true>(l_r.p, width, lane, n_r);
    if (branch) load_raw<WHOLE, NV, TPR, true>(l_b.p, width, lane, n_b);
    l_r.next(), l_b.next();
  };
  if (AHEAD && t0 < t1) ask();
  for (uint32_t t = t0; t < t1; ++t) {
    Raw<T, NV> c_r, c_b, c_gate, c_dn, c_do;
    if (!AHEAD) ask();
    c_r = n_r, c_b = n_b;
    if (gated) load_raw<WHOLE, NV, TPR>(at<const T>(g.in.gate, w, gate_row), width, lane, c_gate);
    if (pre) load_raw<WHOLE, NV, TPR, true>(l_dn.p, width, lane, c_dn);
    if (direct) load_raw<WHOLE, NV, TPR, true>(l_do.p, width, lane, c_do);
    if (AHEAD && t + 1 < t1) ask();
    l_dn.next(), l_do.next();
    Row<NV> r, b, k, d;
    float inv_b = 1.f;
    // after the block: the unit row stays in b, and is scaled where it is needed
    auto after = [&](Row<NV>& a) {
      a = b;
      if (post) {
        unpack<WHOLE, NV, TPR>(w_post, width, lane, a);
#pragma unroll
        for (int i = 0; i < N; ++i) a.v[i] *= b.v[i];
        if (post_bias) {
          Row<NV> e;
          unpack<WHOLE, NV, TPR>(w_postbias, width, lane, e);
#pragma unroll
          for (int i = 0; i < N; ++i) a.v[i] += e.v[i];
        }
      }
    };
    if (branch) {
      unpack<WHOLE, NV, TPR>(c_b, width, lane, b);
      if (post) inv_b = make_unit<NV, TPR, LAYER>(b, g, lane, red, turn);
      Row<NV> a;
      after(a);
      if (gated) {
        unpack<WHOLE, NV, TPR>(c_gate, width, lane, k);
#pragma unroll
        for (int i = 0; i < N; ++i) a.v[i] *= k.v[i];
      }
      unpack<WHOLE, NV, TPR>(c_r, width, lane, r);
#pragma unroll
      for (int i = 0; i < N; ++i) r.v[i] = fmaf(alpha, r.v[i], beta * a.v[i]);
    } else {
      unpack<WHOLE, NV, TPR>(c_r, width, lane, r);
#pragma unroll
      for (int i = 0; i < N; ++i) r.v[i] *= alpha;
    }
    if (pre) {
      // with q = dn pre:  (q - mean(q) - r mean(q r) / s^2) / s of the centred row r, whose two sums go together
      unpack<WHOLE, NV, TPR>(c_dn, width, lane, d);
      unpack<WHOLE, NV, TPR>(w_pre, width, lane, k);
      float mean_q = 0.f;
      if constexpr (LAYER) {
        float s[2] = {0.f, 0.f};   // r, q
#pragma unroll
        for (int i = 0; i < N; ++i) { s[0] += r.v[i]; s[1] = fmaf(d.v[i], k.v[i], s[1]); }
        row_sums<TPR, LAYER>(s, red, turn);
        const float mean = mean_of(s[0], g);
        mean_q = s[1] * inv_width;
#pragma unroll
        for (int i = 0; i < N; ++i) r.v[i] = ((i / kV) * TPR + lane) * kV + i % kV < width ? r.v[i] - mean : 0.f;
      }
      float s[LAYER ? 3 : 2] = {};   // r^2, q r, r
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s[0] = fmaf(r.v[i], r.v[i], s[0]);
        s[1] = fmaf(d.v[i] * k.v[i], r.v[i], s[1]);
        if constexpr (LAYER) s[2] += r.v[i];
      }
      row_sums<TPR, LAYER>(s, red, turn);
      float delta = 0.f;
      if constexpr (LAYER) delta = s[2] * inv_width;
      const float inv = 1.f / sqrtf(variance<LAYER>(s[0] * inv_width, delta) + g.eps);
      const float c = (LAYER ? fmaf(-delta, mean_q, s[1] * inv_width) : s[1] * inv_width) * inv;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float u = LAYER ? fmaf(r.v[i], inv, -delta * inv) : r.v[i] * inv;   // what lies beyond the width meets a d and a sum that are not used there
        s_pre.v[i] = fmaf(d.v[i], u, s_pre.v[i]);
        if (LAYER) s_prebias.v[i] += d.v[i];
        d.v[i] = (d.v[i] * k.v[i] - mean_q - u * c) * inv;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) d.v[i] = 0.f;
    }
    if (direct) {
      unpack<WHOLE, NV, TPR>(c_do, width, lane, k);
#pragma unroll
      for (int i = 0; i < N; ++i) d.v[i] += k.v[i];
    }
    if (o_r.p) {
#pragma unroll
      for (int i = 0; i < N; ++i) k.v[i] = alpha * d.v[i];
      put_row<WHOLE, NV, TPR, true>(o_r.p, width, lane, k);
      o_r.next();
    }
    if (!branch) continue;
#pragma unroll
    for (int i = 0; i < N; ++i) d.v[i] *= beta;
    if (gated) {
      after(k);
#pragma unroll
      for (int i = 0; i < N; ++i) s_gate.v[i] = fmaf(d.v[i], k.v[i], s_gate.v[i]);
      unpack<WHOLE, NV, TPR>(c_gate, width, lane, k);
#pragma unroll
      for (int i = 0; i < N; ++i) d.v[i] *= k.v[i];
      if (t + 1 == until && !g.group_stripes) {
        if (g.d.gate.p) put_row<WHOLE, NV, TPR>(at<T>(g.d.gate, w, gate_row), width, lane, s_gate);
#pragma unroll
        for (int i = 0; i < N; ++i) s_gate.v[i] = 0.f;
        ++gate_row;
        until = (uint32_t)min((uint64_t)g.in.rows, (uint64_t)until + g.in.gate_rows);
      }
    }
    if (post) {
      unpack<WHOLE, NV, TPR>(w_post, width, lane, k);
      float s[2] = {0.f, 0.f};   // p b, p
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s_post.v[i] = fmaf(d.v[i], b.v[i], s_post.v[i]);
        if (LAYER) s_postbias.v[i] += d.v[i];
        d.v[i] *= k.v[i];
        s[0] = fmaf(d.v[i], b.v[i], s[0]);
        if (LAYER) s[1] += d.v[i];
      }
      row_sums<TPR, LAYER>(s, red, turn);
      const float pb = s[0] * inv_width, sp = s[1] * inv_width;
#pragma unroll
      for (int i = 0; i < N; ++i) d.v[i] = (d.v[i] - sp - b.v[i] * pb) * inv_b;
    }
    if (o_b.p) {
      put_row<WHOLE, NV, TPR, true>(o_b.p, width, lane, d);
      o_b.next();
    }
  }
  constexpr int SLOTS = slots_of(LAYER), P_POST = LAYER ? 2 : 1;
  float* p = g.partials + ((uint64_t)w * g.stripes + stripe) * SLOTS * g.padded;
  const int padded = (int)g.padded;   // a multiple of 64
  if (g.d.pre.p) put_row<true, NV, TPR>(p, padded, lane, s_pre);
  if (LAYER && g.d.pre_bias.p) put_row<true, NV, TPR>(p + padded, padded, lane, s_prebias);
  if (g.d.post.p) put_row<true, NV, TPR>(p + P_POST * padded, padded, lane, s_post);
  if (LAYER && g.d.post_bias.p) put_row<true, NV, TPR>(p + 3 * padded, padded, lane, s_postbias);
  if (g.d.gate.p && g.group_stripes) put_row<true, NV, TPR>(p + (SLOTS - 1) * padded, padded, lane, s_gate);
}

// Adds the stripes' shares, in their order: 64 columns to a workgroup, each of its wavefronts has every 16th stripe.
constexpr int kJoinWaves = 16;
template <typename T>
__global__ __launch_bounds__(kJoinWaves * 64) void k_blocknorm_join(NormArgs g, uint32_t groups) {
  __shared__ float part[kJoinWaves][64];
  const uint32_t block = g.first + blockIdx.x, blocks = (g.width + 63) / 64, cell = block / blocks;   // cells: worker x (four weights, then the gate's groups)
  const uint32_t w = cell / (4 + groups), which = cell % (4 + groups);
  const evg_mat& out = which == 0 ? g.d.pre : which == 1 ? g.d.pre_bias : which == 2 ? g.d.post : which == 3 ? g.d.post_bias : g.d.gate;
  if (!out.p) return;
  const uint32_t s0 = which < 4 ? 0 : (which - 4) * g.group_stripes, s1 = which < 4 ? g.stripes : s0 + g.group_stripes;
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = block % blocks * 64 + lane;
  float sum = 0.f;
  if (c < g.padded) {
    const uint32_t slot = g.slots == slots_of(true) ? min(which, 4u) : min(which, 4u) / 2;
    const float* p = g.partials + ((uint64_t)w * g.stripes * g.slots + slot) * g.padded + c;
#pragma unroll 8
    for (uint32_t s = s0 + wave; s < s1; s += kJoinWaves) sum += p[(uint64_t)s * g.slots * g.padded];
  }
  part[wave][lane] = sum;
  __syncthreads();
  if (wave || c >= g.width) return;
#pragma unroll
  for (int i = 1; i < kJoinWaves; ++i) sum += part[i][lane];
  at<T>(out, w, which < 4 ? 0 : which - 4)[c] = from_f<T>(sum);
}

template <typename T, int NV, int TPR, bool LAYER>
hipError_t forward_sized(NormArgs g, hipStream_t s) {
  constexpr int rows = TPR < 256 ? 256 / TPR : 1;
  const uint64_t all = (uint64_t)g.workers * g.in.rows;
  launch_pieces((all + rows - 1) / rows, TPR * rows, [&](uint32_t first, uint32_t grid) {
    g.first = first;
    k_blocknorm_forward<T, NV, TPR, LAYER><<<grid, TPR * rows, 0, s>>>(g);
  });
  return hipGetLastError();
}

template <typename T, bool LAYER>
hipError_t launch_forward(const NormArgs& g, hipStream_t s) {
  if (g.width <= 128) return forward_sized<T, 1, 16, LAYER>(g, s);
  if (g.width <= 256) return forward_sized<T, 1, 32, LAYER>(g, s);
  if (g.width <= 512) return forward_sized<T, 1, 64, LAYER>(g, s);
  if (g.width <= 1024) return forward_sized<T, 2, 64, LAYER>(g, s);
  if (g.width <= 2048) return forward_sized<T, 2, 128, LAYER>(g, s);
  if (g.width <= 4096) return forward_sized<T, 2, 256, LAYER>(g, s);
  if (g.width <= 8192) return forward_sized<T, 2, 512, LAYER>(g, s);
  return forward_sized<T, 2, 1024, LAYER>(g, s);
}

// 1024 threads leave 128 registers to each, and that is not enough for the sums of every weight: of 4097 to 8192 elements most forms with a norm behind
// the block spill some (up to 52, 157 where the width is no multiple of 8), above 8192 all do (up to 497).  2^25 elements of bf16, layer norms
// and a gate, widths 4096 / 8192 / 8200: 166 / 212 / 910 us, of float32 229 / 447 / 1552.
template <typename T, bool LAYER, int GATED, int POST>
hipError_t backward_sized(NormArgs g, hipStream_t s) {
  auto launch = [&](auto kernel, uint32_t threads) {
    launch_pieces((uint64_t)g.workers * g.stripes, threads, [&](uint32_t first, uint32_t grid) {
      g.first = first;
      kernel<<<grid, threads, 0, s>>>(g);
    });
    return hipGetLastError();
  };
  if (!g.stripes) return hipSuccess;
  if (g.width <= 512) return launch(k_blocknorm_backward<T, 1, 64, LAYER, GATED, POST>, 64);
  if (g.width <= 1024) return launch(k_blocknorm_backward<T, 1, 128, LAYER, GATED, POST>, 128);
  if (g.width <= 2048) return launch(k_blocknorm_backward<T, 1, 256, LAYER, GATED, POST>, 256);
  if (g.width <= 4096) return launch(k_blocknorm_backward<T, 1, 512, LAYER, GATED, POST>, 512);
  if (g.width <= 8192) return launch(k_blocknorm_backward<T, 1, 1024, LAYER, GATED, POST>, 1024);
  return launch(k_blocknorm_backward<T, 2, 1024, LAYER, GATED, POST>, 1024);
}

template <typename T, bool LAYER>
hipError_t launch_backward(const NormArgs& g, hipStream_t s) {
  if (g.width % kV) return backward_sized<T, LAYER, -1, -1>(g, s);
  if (g.in.gate.p) return g.in.post.p ? backward_sized<T, LAYER, 1, 1>(g, s) : backward_sized<T, LAYER, 1, 0>(g, s);
  return g.in.post.p ? backward_sized<T, LAYER, 0, 1>(g, s) : backward_sized<T, LAYER, 0, 0>(g, s);
}

template <typename T>
hipError_t launch_blocknorm(NormArgs g, uint32_t kind, bool backward, hipStream_t s) {
  if (!backward) return kind == EVG_NORM_LAYER ? launch_forward<T, true>(g, s) : launch_forward<T, false>(g, s);
  const hipError_t e = kind == EVG_NORM_LAYER ? launch_backward<T, true>(g, s) : launch_backward<T, false>(g, s);
  if (e != hipSuccess) return e;
  const uint32_t groups = g.d.gate.p && g.group_stripes ? g.stripes / g.group_stripes : 0;
  if (!g.d.pre.p && !g.d.pre_bias.p && !g.d.post.p && !g.d.post_bias.p && !groups) return hipSuccess;
  launch_pieces((uint64_t)((g.width + 63) / 64) * g.workers * (4 + groups), kJoinWaves * 64, [&](uint32_t first, uint32_t grid) {
    g.first = first;
    k_blocknorm_join<T><<<grid, kJoinWaves * 64, 0, s>>>(g, groups);
  });
  return hipGetLastError();
}

hipError_t launch_typed(const NormArgs& g, uint32_t type, uint32_t kind, bool backward, hipStream_t s) {
  if (type == EVG_F32) return launch_blocknorm<float>(g, kind, backward, s);
  if (type == EVG_F16) return launch_blocknorm<half_t>(g, kind, backward, s);
  return launch_blocknorm<bf16_t>(g, kind, backward, s);
}

}  // namespace
}  // namespace evg

using namespace evg;

struct evg_blocknorm {
  evg_blocknorm_config cfg{};
  hipStream_t stream = nullptr;
  float* partials = nullptr;
  uint64_t max_stripes = 0;   // of a worker
  uint32_t padded = 0;
};

namespace {

// Stripes of all workers together, about.  A stripe is a workgroup, and the more wavefronts that has the fewer fill the chip; every one
// leaves a row of sums for the join, which is the slower the more of them one worker has.  Backward and join, 1024 / 2048 / 4096 of them:
// 16384 rows of 4096 179 / 190 / 222 us, of 1024 66 / 55 / 68; 8 x 2000 of 512 48 / 36 / 33; 11 x 5331 of 64 103 / 65 / 50; 1 x 16384 of 64
// 40 / 36 / 43.  One worker's rows of at most 512 with 2048 / 4096: 4000 of 64 18 / 25, 16384 of 256 34 / 40 (float32 37 / 47), 6000 of 512 25 / 28,
// 65536 of 512 96 / 104; only very many narrow ones are the other way, 100 000 of 64 111 / 99, 65536 of 256 85 / 78 (float32 101 / 109).
uint32_t most_stripes(uint32_t workers, uint32_t width) { return width > 1024 ? 1024 : width > 512 || workers == 1 ? 2048 : 4096; }

// Rows of a stripe such that there are about so many.
uint32_t stripe_rows(uint32_t workers, uint32_t width, uint32_t rows) {
  const uint32_t most = most_stripes(workers, width);
  const uint64_t r = ((uint64_t)workers * rows + most - 1) / most;
  return (uint32_t)(r < 1 ? 1 : r > rows ? (rows ? rows : 1) : r);
}

evg_status check_norm_in(const evg_blocknorm* c, const evg_blocknorm_in* in) {
  const evg_blocknorm_config& f = c->cfg;
  const uint32_t W = f.workers, D = f.width, ty = f.type;
  if (in->rows > f.max_rows) return fail(EVG_ERR_INVALID, "rows exceeds the context's max_rows");
  if (!in->branch.p && (in->gate.p || in->post.p || in->post_bias.p)) return fail(EVG_ERR_INVALID, "without a branch there is no gate and no norm after it");
  if (in->gate.p && !in->gate_rows) return fail(EVG_ERR_INVALID, "gate_rows must be at least 1");
  if ((in->post_bias.p && !in->post.p) || (in->pre_bias.p && !in->pre.p)) return fail(EVG_ERR_INVALID, "a bias needs its norm's weight");
  if (f.kind == EVG_NORM_RMS && (in->post_bias.p || in->pre_bias.p)) return fail(EVG_ERR_INVALID, "RMS norms have no bias");
  evg_status st;
  if ((st = check_mat(&in->residual, W, in->rows, D, ty, false, "residual")) != EVG_OK) return st;
  if (in->branch.p && (st = check_mat(&in->branch, W, in->rows, D, ty, false, "branch")) != EVG_OK) return st;
  if (in->gate.p && (st = check_mat(&in->gate, W, ((uint64_t)in->rows + in->gate_rows - 1) / in->gate_rows, D, ty, false, "gate")) != EVG_OK) return st;
  const struct { const evg_mat* m; const char* what; } vectors[] = {{&in->post, "post"}, {&in->post_bias, "post_bias"}, {&in->pre, "pre"}, {&in->pre_bias, "pre_bias"}};
  for (const auto& v : vectors)
    if (v.m->p && (st = check_mat(v.m, W, 1, D, ty, false, v.what)) != EVG_OK) return st;
  return EVG_OK;
}

NormArgs norm_args(const evg_blocknorm* c, const evg_blocknorm_in* in) {
  NormArgs g{};
  g.in = *in;
  g.width = c->cfg.width;
  g.workers = c->cfg.workers;
  g.eps = c->cfg.eps;
  g.alpha = c->cfg.residual_scale;
  g.beta = c->cfg.branch_scale;
  g.inv_width = (float)(1.0 / c->cfg.width);
  g.partials = c->partials;
  g.slots = slots_of(c->cfg.kind == EVG_NORM_LAYER);
  g.padded = c->padded;
  return g;
}

}  // namespace

extern "C" {

evg_status evg_blocknorm_init(evg_blocknorm** out, const evg_blocknorm_config* cfg, void* hip_stream) {
  if (!out || !cfg) return fail(EVG_ERR_INVALID, "out and cfg must be non-NULL");
  *out = nullptr;
  if (cfg->workers < 1 || cfg->width < 1 || cfg->width > EVG_BLOCKNORM_MAX_WIDTH)
    return fail(EVG_ERR_INVALID, "workers must be at least 1, width 1 .. %u", EVG_BLOCKNORM_MAX_WIDTH);
  if ((uint64_t)cfg->workers * cfg->max_rows > 0x7FFFFFFFull || (uint64_t)cfg->workers * cfg->width > 0x7FFFFFFFull)
    return fail(EVG_ERR_INVALID, "workers, max_rows: more than 2^31 rows or weights");
  evg_status st;
  if ((st = check_type(cfg->type, "type")) != EVG_OK) return st;
  if (cfg->kind > EVG_NORM_LAYER) return fail(EVG_ERR_INVALID, "kind must be EVG_NORM_RMS or EVG_NORM_LAYER");
  if (!(cfg->eps >= 0.f) || std::isinf(cfg->eps)) return fail(EVG_ERR_INVALID, "eps must be finite and not negative");
  if (!std::isfinite(cfg->residual_scale) || !std::isfinite(cfg->branch_scale)) return fail(EVG_ERR_INVALID, "the scales must be finite");
  evg_blocknorm* c = new (std::nothrow) evg_blocknorm();
  if (!c) return fail(EVG_ERR_OOM, "host allocation failed");
  c->cfg = *cfg;
  c->stream = static_cast<hipStream_t>(hip_stream);
  c->padded = (cfg->width + 63) / 64 * 64;
  // Stripes that fit the gate's groups (backward) are at most twice as many as those asked for, s = ceil(rows / n) of n rows.  Whole groups to a
  // stripe: more than n / 2 rows.  a groups of g > n rows in b stripes each: s >= (a - 1)(b - 1) + 1, and a b is at most twice that where a and b
  // are 2 or more; a = 1 is b = s.
  const uint64_t per = ((uint64_t)most_stripes(cfg->workers, cfg->width) + cfg->workers - 1) / cfg->workers;
  c->max_stripes = 2 * (per < cfg->max_rows ? per : cfg->max_rows);
  const uint64_t bytes = cfg->workers * c->max_stripes * slots_of(cfg->kind == EVG_NORM_LAYER) * c->padded * sizeof(float);
  const hipError_t e = cfg->forward_only || !bytes ? hipSuccess : hipMalloc((void**)&c->partials, bytes);
  if (e != hipSuccess) {
    delete c;
    return fail(e == hipErrorOutOfMemory ? EVG_ERR_OOM : EVG_ERR_HIP, "workspace: %s", hipGetErrorString(e));
  }
  *out = c;
  return EVG_OK;
}

evg_status evg_blocknorm_forward(evg_blocknorm* c, const evg_blocknorm_in* in, const evg_mat* residual_out, const evg_mat* normed) {
  if (!c || !in) return fail(EVG_ERR_INVALID, "context and in must be non-NULL");
  evg_status st = check_norm_in(c, in);
  if (st != EVG_OK) return st;
  const uint32_t W = c->cfg.workers, D = c->cfg.width, ty = c->cfg.type;
  const bool has_out = residual_out && residual_out->p, has_normed = normed && normed->p;
  if (has_normed != (in->pre.p != nullptr)) return fail(EVG_ERR_INVALID, "normed is given exactly if pre is");
  if (!has_out && !has_normed) return fail(EVG_ERR_INVALID, "there is nothing to compute");
  if (has_out && (st = check_mat(residual_out, W, in->rows, D, ty, true, "residual_out")) != EVG_OK) return st;
  if (has_normed && (st = check_mat(normed, W, in->rows, D, ty, true, "normed")) != EVG_OK) return st;
  const uint64_t gates = in->gate.p ? ((uint64_t)in->rows + in->gate_rows - 1) / in->gate_rows : 0;
  const Span outs[] = {mat_span(residual_out, W, in->rows, D, ty, "residual_out"), mat_span(normed, W, in->rows, D, ty, "normed")};
  const Span ins[] = {mat_span(&in->residual, W, in->rows, D, ty, "residual"), mat_span(&in->branch, W, in->rows, D, ty, "branch"),
                      mat_span(&in->gate, W, gates, D, ty, "gate"), mat_span(&in->post, W, 1, D, ty, "post"),
                      mat_span(&in->post_bias, W, 1, D, ty, "post_bias"), mat_span(&in->pre, W, 1, D, ty, "pre"),
                      mat_span(&in->pre_bias, W, 1, D, ty, "pre_bias")};
  if ((st = check_apart(outs, 2, ins, 7, 0, 0)) != EVG_OK) return st;
  if (!in->rows) return EVG_OK;
  NormArgs g = norm_args(c, in);
  if (has_out) g.out = *residual_out;
  if (has_normed) g.normed = *normed;
  HIP_TRY(launch_typed(g, ty, c->cfg.kind, false, c->stream));
  return EVG_OK;
}

evg_status evg_blocknorm_backward(evg_blocknorm* c, const evg_blocknorm_in* in, const evg_mat* d_residual, const evg_mat* d_normed,
                                  const evg_blocknorm_grads* out) {
  if (!c || !in || !out) return fail(EVG_ERR_INVALID, "context, in and out must be non-NULL");
  if (c->cfg.forward_only) return fail(EVG_ERR_STATE, "the context was made forward_only");
  evg_status st = check_norm_in(c, in);
  if (st != EVG_OK) return st;
  const uint32_t W = c->cfg.workers, D = c->cfg.width, ty = c->cfg.type;
  const bool has_res = d_residual && d_residual->p, has_normed = d_normed && d_normed->p;
  if (has_normed && !in->pre.p) return fail(EVG_ERR_INVALID, "d_normed is given without pre");
  if (has_res && (st = check_mat(d_residual, W, in->rows, D, ty, false, "d_residual")) != EVG_OK) return st;
  if (has_normed && (st = check_mat(d_normed, W, in->rows, D, ty, false, "d_normed")) != EVG_OK) return st;
  const uint64_t gates = in->gate.p ? ((uint64_t)in->rows + in->gate_rows - 1) / in->gate_rows : 0;
  const struct { const evg_mat *m, *of; uint64_t rows; const char* what; } grads[] = {
      {&out->residual, &in->residual, in->rows, "the gradient of residual"}, {&out->branch, &in->branch, in->rows, "the gradient of branch"},
      {&out->gate, &in->gate, gates, "the gradient of gate"}, {&out->post, &in->post, 1, "the gradient of post"},
      {&out->post_bias, &in->post_bias, 1, "the gradient of post_bias"}, {&out->pre, &in->pre, 1, "the gradient of pre"},
      {&out->pre_bias, &in->pre_bias, 1, "the gradient of pre_bias"}};
  Span outs[7], ins[9];
  int n = 0;
  for (int i = 0; i < 7; ++i) {
    ins[i] = mat_span(grads[i].of, W, grads[i].rows, D, ty, "an input");
    if (!grads[i].m->p) continue;
    if (!grads[i].of->p) return fail(EVG_ERR_INVALID, "%s is asked for, which is absent", grads[i].what);
    if ((st = check_mat(grads[i].m, W, grads[i].rows, D, ty, true, grads[i].what)) != EVG_OK) return st;
    outs[n++] = mat_span(grads[i].m, W, grads[i].rows, D, ty, grads[i].what);
  }
  ins[7] = mat_span(has_res ? d_residual : nullptr, W, in->rows, D, ty, "d_residual");
  ins[8] = mat_span(has_normed ? d_normed : nullptr, W, in->rows, D, ty, "d_normed");
  if ((st = check_apart(outs, n, ins, 9, out->residual.p ? 0 : -1, 7)) != EVG_OK) return st;
  NormArgs g = norm_args(c, in);
  if (has_res) g.d_out = *d_residual;
  if (has_normed) g.d_normed = *d_normed;
  g.d = *out;
  if (in->rows) {
    g.stripe_rows = stripe_rows(W, D, in->rows);
    g.stripes = (in->rows + g.stripe_rows - 1) / g.stripe_rows;
    if (out->gate.p && in->gate_rows <= g.stripe_rows) {
      g.stripe_rows = g.stripe_rows / in->gate_rows * in->gate_rows;
      g.stripes = (in->rows + g.stripe_rows - 1) / g.stripe_rows;
    } else if (out->gate.p) {
      const uint32_t group = in->gate_rows < in->rows ? in->gate_rows : in->rows;
      g.group_stripes = (group + g.stripe_rows - 1) / g.stripe_rows;
      g.stripe_rows = (group + g.group_stripes - 1) / g.group_stripes;
      g.stripes = (uint32_t)gates * g.group_stripes;
    }
    if (g.stripes > c->max_stripes) return fail(EVG_ERR_STATE, "%u stripes of rows, room for %llu", g.stripes, (unsigned long long)c->max_stripes);
  }
  HIP_TRY(launch_typed(g, ty, c->cfg.kind, true, c->stream));
  return EVG_OK;
}

evg_status evg_blocknorm_destroy(evg_blocknorm* c) {
  if (!c) return EVG_OK;
  hipError_t e = hipStreamSynchronize(c->stream);
  if (c->partials) { const hipError_t f = hipFree(c->partials); if (e == hipSuccess) e = f; }
  delete c;
  HIP_TRY(e);
  return EVG_OK;
}

}  // extern "C"
