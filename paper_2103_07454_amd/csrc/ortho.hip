// Host side and the elementwise passes of orthogonal updates (include/evg_nn.h, evg_ortho_*).
//
//     m' = mu m + G,  u = G + mu m' or m',  X = u / (|u| + eps);  steps times  S = X X^T,  P = b S + c S S,  X <- a X + P X
//
// With n the smaller side and k the larger, a step is n^2 k (S, half of it), n^3 (S S, half of it) and 2 n^2 k operations, all on the matrix cores,
// three launches.  What the steps cost in precision was looked at with each value rounded by itself (gradients of few directions, of few strong and many weak ones, and of all alike;
// sides 4 to 2816, five usual steps).  Rounding X to float16 between steps leaves an error of 1e-3 to 1e-2 of the result, as the small singular values grow up to 485-fold and what is
// rounded off the large ones' part grows with them. So X is kept in two parts, 22 bits, of which products read the first; the second costs a read and a write a
// step.  Rounding S, P and the products' operands then leaves 1e-4 to 3e-3, most where all singular values are alike and the smaller side is short (2.5e-3 at 16, 2.1e-3 at 64, 1.8e-3 at
// 256, 1.4e-3 at 1024).  Multiplying both parts of all operands, three products for one, leaves 3e-7 to 4e-5 beside the sums' own.
//   bfloat16 rounds 1.7e-3 off a result.  Above a smaller side of 256 products are of one part, which leaves about as much at most (1.8e-3 of 512 x 4000; time: 8 of 1024 x 2816: 731 us, 1498 with both parts); up to there of
//   both, which costs little (128 x 128: 76 us with one part, 82 with both; four of 128 x 784 97 and 103; 256 x 1024 100 and 115, eight of them 110 and 154).
//   float16 rounds off 2e-4.  Where only the last two steps multiplied both parts, the first three left up to 2e-3 (16 x 16; 6e-4 at 512 x 512, 4e-4 of 64 equal directions of 1024 x 2816): all do.
//
// The elementwise passes are bound by memory: 4096 x 11264 with its momentum 93 and 86 us, 460 MB each, 4.9 and 5.3 TB/s.  The norm is known only behind the first, so the
// second reads gradient and momentum again.
//
// X, S and P are kept times powers of two, so that the largest elements that they can have come near float16's 65504 and the small ones
// stay clear of its subnormals: an element is at most the largest singular value, which p(s) = a s + b s^3 + c s^5 bounds.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "nn_device.h"
#include "nn_host.h"
#include "ortho_choose.h"
#include "ortho_internal.h"

namespace evg {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kBlocks = 2048;  // of a matrix, at most: each of the second pass adds up what those of the first left
constexpr int kVector = 8;          // elements of a lane
constexpr uint32_t kBothSide = 256;   // largest smaller side of bfloat16 matrices whose products are of both parts

struct UpdateArgs {
  evg_mat grad, momentum, momentum_out;
  uint32_t rows, cols, nesterov, blocks, first;
  float mu, eps, scale_x;
  double* partials;     // [matrices][blocks]
  Halves x;
};

// The update's elements at (row, col .. col + 7) from the gradient and, where it is there, the new momentum.
__device__ __forceinline__ void update_of(const UpdateArgs& a, const float* g, const float* m, float* u) {
#pragma unroll
  for (int i = 0; i < kVector; ++i) u[i] = a.momentum.p ? (a.nesterov ? fmaf(a.mu, m[i], g[i]) : m[i]) : g[i];
}

__device__ __forceinline__ double group_sum(double v, double* part) {
  v = wave_sum(v);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) v += part[i];
  return v;
}

// The new momentum, and each workgroup's sum of the update's squares.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_ortho_momentum(UpdateArgs a) {
  __shared__ double part[kWaves];
  const uint32_t group = a.first + blockIdx.x, w = group / a.blocks, b = group % a.blocks;
  const uint32_t across = (a.cols + 64 * kVector - 1) / (64 * kVector);
  const uint64_t jobs = (uint64_t)a.rows * across;
  const int lane = threadIdx.x & 63;
  double sum = 0.0;
  for (uint64_t job = b * kWaves + threadIdx.x / 64; job < jobs; job += (uint64_t)a.blocks * kWaves) {
    const uint32_t row = (uint32_t)(job / across), col = ((uint32_t)(job % across) * 64 + lane) * kVector;
    const int n = (int)a.cols - (int)col;
    float g[kVector], m[kVector] = {}, u[kVector];
    load_upto<kVector>((const T*)a.grad.p + (int64_t)w * a.grad.worker + (int64_t)row * a.grad.row + col, n, g);
    if (a.momentum.p) {
      load_upto<kVector>((const float*)a.momentum.p + (int64_t)w * a.momentum.worker + (int64_t)row * a.momentum.row + col, n, m);
#pragma unroll
      for (int i = 0; i < kVector; ++i) m[i] = fmaf(a.mu, m[i], g[i]);
      store_upto<kVector>((float*)a.momentum_out.p + (int64_t)w * a.momentum_out.worker + (int64_t)row * a.momentum_out.row + col, n, m);
    }
    update_of(a, g, m, u);
#pragma unroll
    for (int i = 0; i < kVector; ++i) sum = fma((double)u[i], (double)u[i], sum);
  }
  sum = group_sum(sum, part);
  if (threadIdx.x == 0) a.partials[(uint64_t)w * a.blocks + b] = sum;
}

// X in two parts, and zeros up to whole units behind its rows.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_ortho_start(UpdateArgs a) {
  __shared__ double part[kWaves];
  const uint32_t group = a.first + blockIdx.x, w = group / a.blocks, b = group % a.blocks;
  double sum = 0.0;
  for (uint32_t i = threadIdx.x; i < a.blocks; i += kThreads) sum += a.partials[(uint64_t)w * a.blocks + i];
  const double norm = sqrt(group_sum(sum, part));
  // The factor as a fraction and a power of two: that of a tiny norm is beyond 32 bits, what it makes of the update's elements is not.
  int power = 0;
  const float f = norm == 0.0 ? 0.f : (float)frexp((double)a.scale_x / (norm + (double)a.eps), &power);
  const uint32_t across = (a.cols + 64 * kVector - 1) / (64 * kVector);
  const uint64_t jobs = (uint64_t)a.rows * across;
  const int lane = threadIdx.x & 63;
  for (uint64_t job = b * kWaves + threadIdx.x / 64; job < jobs; job += (uint64_t)a.blocks * kWaves) {
    const uint32_t row = (uint32_t)(job / across), col = ((uint32_t)(job % across) * 64 + lane) * kVector;
    const int n = (int)a.cols - (int)col;
    if (n <= 0) continue;
    float g[kVector], m[kVector] = {}, u[kVector];
    load_upto<kVector>((const T*)a.grad.p + (int64_t)w * a.grad.worker + (int64_t)row * a.grad.row + col, n, g);
    if (a.momentum.p) load_upto<kVector>((const float*)a.momentum_out.p + (int64_t)w * a.momentum_out.worker + (int64_t)row * a.momentum_out.row + col, n, m);
    update_of(a, g, m, u);
    Pack<half_t, kVector> hi, lo;
#pragma unroll
    for (int i = 0; i < kVector; ++i) {
      halves_of(i < n ? ldexpf(u[i], power) * f : 0.f, &hi.v[i], &lo.v[i]);
    }
    uint16_t* const p = a.x.p + (int64_t)w * a.x.worker + (int64_t)row * a.x.ld + halves_col(a.x.paired, col);
    *reinterpret_cast<Pack<half_t, kVector>*>(p) = hi;
    *reinterpret_cast<Pack<half_t, kVector>*>(p + a.x.apart) = lo;
  }
}

template <typename T>
hipError_t launch_start(UpdateArgs a, uint32_t matrices, hipStream_t s) {
  const uint64_t groups = (uint64_t)matrices * a.blocks;
  if (groups > 0x7FFFFFFFull) return hipErrorInvalidValue;
  launch_pieces(groups, kThreads, [&](uint32_t first, uint32_t grid) {
    a.first = first;
    k_ortho_momentum<T><<<grid, kThreads, 0, s>>>(a);
  });
  launch_pieces(groups, kThreads, [&](uint32_t first, uint32_t grid) {
    a.first = first;
    k_ortho_start<T><<<grid, kThreads, 0, s>>>(a);
  });
  return hipGetLastError();
}

}  // namespace

hipError_t launch_ortho(OrthoOp op, bool tall, bool split, bool last, const OrthoArgs& a, hipStream_t s) {
  return split ? launch_ortho_parts<true>(op, tall, last, a, s) : launch_ortho_parts<false>(op, tall, last, a, s);
}

}  // namespace evg

using namespace evg;

struct evg_ortho {
  evg_ortho_config cfg{};
  hipStream_t stream = nullptr;
  void* owned = nullptr;
  double* partials = nullptr;
  uint16_t *x[2]{}, *s = nullptr, *p = nullptr;   // each with room for both parts
  float* sums = nullptr;   // partial sums of products
  uint64_t room = 0;       // how many
  uint32_t blocks = 1;
  bool split = false;      // products of both parts
  float scale_x = 1.f, scale_s = 1.f, scale_p = 1.f;
};

namespace {

// The largest |b t + c t^2| for t in 0 .. end.
double most_quadratic(double b, double c, double end) {
  double most = std::fabs(b * end + c * end * end);
  const double top = c != 0.0 ? -b / (2.0 * c) : 0.0;
  if (top > 0.0 && top < end) most = std::fmax(most, std::fabs(b * top + c * top * top));
  return most;
}

// The largest |a s + b s^3 + c s^5| for s in 0 .. end: at the end or where the derivative a + 3 b t + 5 c t^2, t = s^2, is 0.
double most_quintic(double a, double b, double c, double end) {
  auto p = [&](double s) { return std::fabs(s * (a + s * s * (b + s * s * c))); };
  double most = p(end);
  auto offer = [&](double t) {
    if (t > 0.0 && t < end * end) most = std::fmax(most, p(std::sqrt(t)));
  };
  if (c != 0.0) {
    const double d = 9.0 * b * b - 20.0 * a * c;
    if (d >= 0.0) {
      offer((-3.0 * b + std::sqrt(d)) / (10.0 * c));
      offer((-3.0 * b - std::sqrt(d)) / (10.0 * c));
    }
  } else if (b != 0.0) {
    offer(-a / (3.0 * b));
  }
  return most;
}

// The power of two that takes `most` to between 2^14 and 2^15.
float scale_for(double most) {
  int e = 0;
  (void)std::frexp(std::fmax(most, 1e-3), &e);
  return std::ldexp(1.f, 15 - e);
}

// Rows of a matrix's parts are whole 128 bytes apart.
uint64_t pitch_of(uint32_t cols) { return ((uint64_t)cols + 63) / 64 * 64; }

// A matrix for products of both parts, or of hi alone; with or without a lo.
Halves halves(uint16_t* p, uint32_t matrices, uint32_t rows, uint32_t cols, bool split, bool lo) {
  const int64_t pitch = (int64_t)pitch_of(cols), plane = (int64_t)rows * pitch;
  if (split) return {p, 32, 2 * plane, 2 * pitch, 1};
  return {p, lo ? (int64_t)matrices * plane : 0, plane, pitch, 0};
}

// Floats that partial sums may take at most; no product that is better in parts has been seen to need half of it.
constexpr uint64_t kMostSums = 1ull << 26;

}  // namespace

extern "C" {

evg_status evg_ortho_init(evg_ortho** out, const evg_ortho_config* cfg, void* hip_stream) {
  if (!out || !cfg) return fail(EVG_ERR_INVALID, "out and cfg must be non-NULL");
  *out = nullptr;
  if (cfg->matrices < 1 || cfg->matrices > 65535) return fail(EVG_ERR_INVALID, "matrices must be 1 .. 65535");
  if (cfg->rows < 1 || cfg->rows > 65536 || cfg->cols < 1 || cfg->cols > 65536) return fail(EVG_ERR_INVALID, "rows and cols must be 1 .. 65536");
  const uint32_t n = cfg->rows < cfg->cols ? cfg->rows : cfg->cols;
  if (n > 16384) return fail(EVG_ERR_INVALID, "the smaller of rows and cols must be at most 16384");
  evg_status st;
  if ((st = check_type(cfg->type, "type")) != EVG_OK || (st = check_type(cfg->out_type, "out_type")) != EVG_OK) return st;
  if (cfg->out_type != cfg->type && cfg->out_type != EVG_F32) return fail(EVG_ERR_INVALID, "out_type must be type or EVG_F32");
  if (cfg->steps < 1 || cfg->steps > 64) return fail(EVG_ERR_INVALID, "steps must be 1 .. 64");
  for (float v : {cfg->a, cfg->b, cfg->c, cfg->momentum, cfg->scale})
    if (!std::isfinite(v)) return fail(EVG_ERR_INVALID, "a, b, c, momentum and scale must be finite");
  if (!(cfg->eps >= 0.f) || std::isinf(cfg->eps)) return fail(EVG_ERR_INVALID, "eps must be finite and not negative");
  // It is multiplied with the powers of two that X and P are kept times, at most 2^38, taken back.
  if (cfg->scale != 0.f && std::fabs(cfg->scale) < 0x1p-80f) return fail(EVG_ERR_INVALID, "scale must be 0 or at least 2^-80 in magnitude");
  // Singular values begin at no more than the norm, 1; what rounding adds is less than the hundredth that is allowed for.
  double bound = 1.01;
  for (uint32_t i = 0; i < cfg->steps && bound <= 3.0; ++i) bound = std::fmax(bound, 1.01 * most_quintic(cfg->a, cfg->b, cfg->c, bound));
  if (!(bound <= 3.0)) return fail(EVG_ERR_INVALID, "a, b and c let a singular value pass 3");
  evg_ortho* c = new (std::nothrow) evg_ortho();
  if (!c) return fail(EVG_ERR_OOM, "host allocation failed");
  c->cfg = *cfg;
  c->stream = static_cast<hipStream_t>(hip_stream);
  c->scale_x = scale_for(bound);
  c->scale_s = scale_for(bound * bound);
  c->scale_p = scale_for(1.01 * most_quadratic(cfg->b, cfg->c, bound * bound));
  c->split = cfg->type != EVG_BF16 || n <= kBothSide;
  const uint64_t across = ((uint64_t)cfg->cols + 64 * kVector - 1) / (64 * kVector), jobs = (cfg->rows * across + kWaves - 1) / kWaves;
  c->blocks = (uint32_t)(jobs < kBlocks ? jobs : kBlocks);
  const uint64_t W = cfg->matrices, x = W * cfg->rows * pitch_of(cfg->cols) * 2 * sizeof(uint16_t), s = W * n * pitch_of(n) * 2 * sizeof(uint16_t);
  const uint32_t k = cfg->rows < cfg->cols ? cfg->cols : cfg->rows;
  const OrthoShape gram{n, n, k, cfg->matrices, kMostSums}, square{n, n, n, cfg->matrices, kMostSums}, apply{cfg->rows, cfg->cols, n, cfg->matrices, kMostSums};
  for (const uint64_t need : {ortho_partial(gram, true, choose_ortho(gram, true, c->split)), ortho_partial(square, true, choose_ortho(square, true, c->split)),
                              ortho_partial(apply, false, choose_ortho(apply, false, c->split))})
    if (need > c->room) c->room = need;
  auto whole = [](uint64_t bytes) { return (bytes + 255) / 256 * 256; };
  struct { void** to; uint64_t bytes; } parts[] = {{(void**)&c->partials, W * c->blocks * sizeof(double)}, {(void**)&c->x[0], x}, {(void**)&c->x[1], x},
                                                   {(void**)&c->s, s}, {(void**)&c->p, s}, {(void**)&c->sums, c->room * sizeof(float)}};
  uint64_t total = 0;
  for (auto& q : parts) total += whole(q.bytes);
  const hipError_t e = total >> 46 ? hipErrorOutOfMemory : hipMalloc(&c->owned, total);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    delete c;
    return fail(e == hipErrorOutOfMemory ? EVG_ERR_OOM : EVG_ERR_HIP, "workspace: %s", hipGetErrorString(e));
  }
  char* at = (char*)c->owned;
  for (auto& q : parts) {
    *q.to = at;
    at += whole(q.bytes);
  }
  *out = c;
  return EVG_OK;
}

evg_status evg_ortho_update(evg_ortho* c, const evg_mat* grad, const evg_mat* momentum, const evg_mat* momentum_out, const evg_mat* out) {
  if (!c) return fail(EVG_ERR_INVALID, "context must be non-NULL");
  const evg_ortho_config& g = c->cfg;
  const uint32_t W = g.matrices, R = g.rows, C = g.cols;
  const bool has = momentum && momentum->p;
  if (has != (momentum_out && momentum_out->p)) return fail(EVG_ERR_INVALID, "momentum and momentum_out are given together or not at all");
  evg_status st;
  if ((st = check_mat(grad, W, R, C, g.type, false, "grad")) != EVG_OK) return st;
  if (has && (st = check_mat(momentum, W, R, C, EVG_F32, false, "momentum")) != EVG_OK) return st;
  if (has && (st = check_mat(momentum_out, W, R, C, EVG_F32, true, "momentum_out")) != EVG_OK) return st;
  if ((st = check_mat(out, W, R, C, g.out_type, true, "out")) != EVG_OK) return st;
  // out is written when all else has been read: it may be the gradient, but not the momentum.
  const Span grads = mat_span(grad, W, R, C, g.type, "grad"), old = mat_span(momentum, W, R, C, EVG_F32, "momentum");
  const Span next = mat_span(momentum_out, W, R, C, EVG_F32, "momentum_out"), result = mat_span(out, W, R, C, g.out_type, "out");
  const Span first[] = {grads, old}, rest[] = {old, next, grads};
  if ((st = check_apart(&next, 1, first, 2, 0, 1)) != EVG_OK) return st;
  if ((st = check_apart(&result, 1, rest, 3, g.type == g.out_type ? 0 : -1, 2)) != EVG_OK) return st;

  UpdateArgs u{};
  u.grad = *grad;
  if (has) u.momentum = *momentum, u.momentum_out = *momentum_out;
  for (evg_mat* m : {&u.grad, &u.momentum, &u.momentum_out}) {
    if (W <= 1) m->worker = 0;
    if (R <= 1) m->row = 0;
  }
  u.rows = R, u.cols = C, u.nesterov = g.nesterov, u.blocks = c->blocks;
  u.mu = g.momentum, u.eps = g.eps, u.scale_x = c->scale_x;
  u.partials = c->partials;
  const bool tall = R > C;
  const uint32_t n = tall ? C : R, k = tall ? R : C;
  const bool split = c->split;
  auto x_at = [&](uint32_t step) { return halves(c->x[step & 1], W, R, C, split, true); };
  u.x = x_at(0);
  HIP_TRY(g.type == EVG_F32   ? launch_start<float>(u, W, c->stream)
          : g.type == EVG_F16 ? launch_start<half_t>(u, W, c->stream)
                              : launch_start<bf16_t>(u, W, c->stream));

  const float sx = c->scale_x, ss = c->scale_s, sp = c->scale_p;
  for (uint32_t i = 0; i < g.steps; ++i) {
    const bool last = i + 1 == g.steps;
    const Halves x = x_at(i), S = halves(c->s, W, n, n, split, false), P = halves(c->p, W, n, n, split, false);
    OrthoArgs a{};
    a.matrices = W;
    a.partial = c->sums, a.room = c->room;
    a.a = a.b = x;
    a.to = S;
    a.M = a.N = n, a.K = k;
    a.f_acc = ss / (sx * sx);
    HIP_TRY(launch_ortho(ORTHO_GRAM, tall, split, false, a, c->stream));

    a.a = a.b = a.own = S;
    a.to = P;
    a.K = n;
    a.f_acc = g.c * sp / (ss * ss), a.f_own = g.b * sp / ss;
    HIP_TRY(launch_ortho(ORTHO_SQUARE, tall, split, false, a, c->stream));

    a.a = tall ? x : P;
    a.b = tall ? P : x;
    a.own = x;
    a.to = x_at(i + 1);
    a.M = R, a.N = C;
    a.f_acc = 1.f / sp, a.f_own = g.a;
    if (last) {
      a.f_acc *= g.scale / sx, a.f_own *= g.scale / sx;
      a.out = *out;
      a.out_type = g.out_type;
      if (W <= 1) a.out.worker = 0;
      if (R <= 1) a.out.row = 0;
    }
    HIP_TRY(launch_ortho(ORTHO_APPLY, tall, split, last, a, c->stream));
  }
  return EVG_OK;
}

evg_status evg_ortho_destroy(evg_ortho* c) {
  if (!c) return EVG_OK;
  hipError_t e = hipStreamSynchronize(c->stream);
  if (c->owned) { const hipError_t f = hipFree(c->owned); if (e == hipSuccess) e = f; }
  delete c;
  HIP_TRY(e);
  return EVG_OK;
}

}  // extern "C"
