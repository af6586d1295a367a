// Clipping of each worker's gradient by its global norm (include/evg_nn.h, evg_clip_*).
//
// With s the scale, for worker r:  norm = |s| sqrt(sum_j g_j^2) over all its tensors,  out_j = g_j * (s * min(1, max / (norm + eps))).
// No product can be written before the last square is summed, so the gradient is read twice.  Both passes are bound by memory: 12 bytes an
// element in 32 bits, 64 workers of 11 million elements in 1390 to 1407 us, 6.1 TB/s.  What the second pass reads and writes of whole chunks of 8192 is
// not read again and goes past the caches (1521 us without): results of 32 bits in arenas of more than 8 M elements.  Shorter chunks, which the
// caches hold, and results of 16 bits go through them, a load at a time; so do the squares of 16 bits.  Squaring and scaling by groups of workers, so that the second pass finds a group in the 256 MB
// last-level cache, is no faster: 1404 us in launches that square one group and scale the one before, 1564 in launches of their own.
#include <hip/hip_runtime.h>

#include <cmath>
#include <exception>
#include <new>
#include <vector>

#include "nn_device.h"
#include "nn_host.h"

namespace evg {
namespace {

constexpr int kClipThreads = 256;
// Up to so many sums, each workgroup that writes adds up its worker's for itself (a load or two for each thread); more are added by a launch between.
constexpr uint32_t kOwnSums = 512;

constexpr int kMostChunk = 8192;

// A run of at most kMostChunk elements of a worker's slice without padding in it.
struct ClipChunk { uint32_t off, len; };   // off: a multiple of 4

struct ClipTables {
  const ClipChunk* chunks;
  uint32_t nchunks, P;
  uint64_t pitch;        // elements of a worker's slice
  double* partials;      // [P][nchunks]
  float* factor;         // [P], where a launch of its own finds them
  uint32_t first;        // workgroup of a launch in pieces
};

struct ClipCall {
  float max_norm, scale, eps;
  uint32_t zero_nonfinite;
  float* norm;           // [P] or null
};

// The sum of a workgroup's values, in every thread; the order is fixed.
__device__ __forceinline__ double group_sum(double v, double* part) {
  v = wave_sum(v);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int i = 1; i < kClipThreads / 64; ++i) v += part[i];
  return v;
}

// One workgroup sums the squares of a chunk.  Squares of 32 bits are exact in 64.
template <typename T>
__global__ __launch_bounds__(kClipThreads) void k_clip_squares(ClipTables t, const T* __restrict__ grad) {
  constexpr int E = 16 / sizeof(T), U = 8;
  __shared__ double part[kClipThreads / 64];
  const uint32_t block = t.first + blockIdx.x, r = block / t.nchunks, c = block % t.nchunks;
  const ClipChunk d = t.chunks[c];
  const T* g = grad + (uint64_t)r * t.pitch + d.off;
  double sum[2] = {0.0, 0.0};
  uint32_t j = threadIdx.x * E;
  if constexpr (U * kClipThreads * E <= kMostChunk) {   // 32 bits: a whole chunk's loads are under way at once
    for (; j + (U - 1) * kClipThreads * E + E <= d.len; j += U * kClipThreads * E) {
      float v[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u) load_n<E>(g + j + u * kClipThreads * E, v[u]);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < E; ++i) sum[i & 1] = fma((double)v[u][i], (double)v[u][i], sum[i & 1]);
    }
  }
  for (; j < d.len; j += kClipThreads * E) {
    float v[E];
    load_upto<E>(g + j, (int)(d.len - j), v);
#pragma unroll
    for (int i = 0; i < E; ++i) sum[i & 1] = fma((double)v[i], (double)v[i], sum[i & 1]);
  }
  const double all = group_sum(sum[0] + sum[1], part);
  if (threadIdx.x == 0) t.partials[(uint64_t)r * t.nchunks + c] = all;
}

// Worker r's norm and factor from its chunks' sums, in their order.
__device__ __forceinline__ float clip_factor(const ClipTables& t, const ClipCall& call, uint32_t r, double* part, float* norm_out) {
  double sum = 0.0;
#pragma unroll 4
  for (uint32_t i = threadIdx.x; i < t.nchunks; i += kClipThreads) sum += t.partials[(uint64_t)r * t.nchunks + i];
  sum = group_sum(sum, part);
  const float norm = (float)(sqrt(sum) * fabs((double)call.scale));
  // Compared, not only divided: infinity / infinity and 0 / 0 keep the gradient too.  A NaN stays one.
  const float bound = norm + call.eps;
  float factor = call.scale * (bound <= call.max_norm ? 1.f : call.max_norm / bound);
  if (call.zero_nonfinite && !(norm <= 3.402823466e38f)) factor = 0.f;
  if (norm_out && threadIdx.x == 0) norm_out[r] = norm;
  return factor;
}

__global__ __launch_bounds__(kClipThreads) void k_clip_factor(ClipTables t, ClipCall call) {
  __shared__ double part[kClipThreads / 64];
  const uint32_t r = t.first + blockIdx.x;
  const float f = clip_factor(t, call, r, part, call.norm);
  if (threadIdx.x == 0) t.factor[r] = f;
}

template <typename T, typename U, bool OWN>
__global__ __launch_bounds__(kClipThreads) void k_clip_scale(ClipTables t, ClipCall call, const T* __restrict__ grad, U* __restrict__ out, bool in_place) {
  constexpr int E = 16 / sizeof(U), N = 8;
  __shared__ double part[OWN ? kClipThreads / 64 : 1];
  const uint32_t block = t.first + blockIdx.x, r = block / t.nchunks, c = block % t.nchunks;
  const float f = OWN ? clip_factor(t, call, r, part, c == 0 ? call.norm : nullptr) : t.factor[r];
  if (in_place && f == 1.f) return;
  const bool zero = call.zero_nonfinite && f == 0.f;   // also where an element is not finite
  const ClipChunk d = t.chunks[c];
  const T* g = grad + (uint64_t)r * t.pitch + d.off;
  U* o = out + (uint64_t)r * t.pitch + d.off;
  uint32_t j = threadIdx.x * E;
  if constexpr (N * kClipThreads * E <= kMostChunk) {   // results of 32 bits
    for (; j + (N - 1) * kClipThreads * E + E <= d.len; j += N * kClipThreads * E) {
      float v[N][E];
#pragma unroll
      for (int u = 0; u < N; ++u) load_n_once<E>(g + j + u * kClipThreads * E, v[u]);
#pragma unroll
      for (int u = 0; u < N; ++u) {
#pragma unroll
        for (int i = 0; i < E; ++i) v[u][i] = zero ? 0.f : v[u][i] * f;
        store_n_once<E>(o + j + u * kClipThreads * E, v[u]);
      }
    }
  }
  for (; j < d.len; j += kClipThreads * E) {
    float v[E];
    load_upto<E>(g + j, (int)(d.len - j), v);
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = zero ? 0.f : v[i] * f;
    store_upto<E>(o + j, (int)(d.len - j), v);
  }
}

template <typename T, typename U>
hipError_t launch_clip(ClipTables t, const ClipCall& call, const void* grad, void* out, hipStream_t s) {
  auto launch = [&](uint64_t groups, auto kernel, auto... args) {
    launch_pieces(groups, kClipThreads, [&](uint32_t first, uint32_t grid) {
      t.first = first;
      kernel<<<grid, kClipThreads, 0, s>>>(t, args...);
    });
  };
  const uint64_t groups = (uint64_t)t.P * t.nchunks;
  launch(groups, k_clip_squares<T>, (const T*)grad);
  if (t.nchunks <= kOwnSums) {
    launch(groups, k_clip_scale<T, U, true>, call, (const T*)grad, (U*)out, grad == out);
  } else {
    launch(t.P, k_clip_factor, call);
    launch(groups, k_clip_scale<T, U, false>, call, (const T*)grad, (U*)out, grad == out);
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace evg

using namespace evg;

struct evg_clip {
  evg_clip_config cfg{};
  hipStream_t stream = nullptr;
  ClipTables t{};
  void* owned = nullptr;
};

extern "C" {

evg_status evg_clip_init(evg_clip** out, const evg_clip_config* cfg, void* hip_stream) {
  if (!out || !cfg) return fail(EVG_ERR_INVALID, "out and cfg must be non-NULL");
  *out = nullptr;
  if (cfg->P < 1 || cfg->L < 1) return fail(EVG_ERR_INVALID, "P and L must be at least 1");
  if (!cfg->layer_numel) return fail(EVG_ERR_INVALID, "layer_numel must be non-NULL");
  evg_status st;
  if ((st = check_type(cfg->grad_type, "grad_type")) != EVG_OK || (st = check_type(cfg->out_type, "out_type")) != EVG_OK) return st;
  if (cfg->out_type != cfg->grad_type && cfg->out_type != EVG_F32) return fail(EVG_ERR_INVALID, "out_type must be grad_type or EVG_F32");
  if (!(cfg->eps >= 0.f) || std::isinf(cfg->eps)) return fail(EVG_ERR_INVALID, "eps must be finite and not negative");
  if (cfg->nonfinite > EVG_NONFINITE_ZERO) return fail(EVG_ERR_INVALID, "nonfinite must be EVG_NONFINITE_PASS or EVG_NONFINITE_ZERO");
  const uint64_t pitch = evg_padded_numel(cfg->L, cfg->layer_numel);
  if (!pitch) return fail(EVG_ERR_INVALID, "layer_numel: each must be 1 .. 2^31-8, a worker's slice at most 2^32 elements");
  if ((unsigned __int128)cfg->P * pitch >> 60) return fail(EVG_ERR_INVALID, "P is out of range");
  try {
    std::vector<ClipChunk> chunks;
    // Tensors whose length is a multiple of 4 run into the next one without padding.
    const uint64_t most = (uint64_t)cfg->P * pitch <= (8u << 20) ? 2048 : kMostChunk;
    uint64_t at = 0, begin = 0;
    for (uint32_t l = 0; l < cfg->L; ++l) {
      at += cfg->layer_numel[l];
      if (at % 4 == 0 && l + 1 < cfg->L) continue;
      for (; begin < at; begin += most) chunks.push_back({(uint32_t)begin, (uint32_t)(at - begin < most ? at - begin : most)});
      at = begin = (at + 3) / 4 * 4;
    }
    if ((uint64_t)chunks.size() * cfg->P > 0x7FFFFFFFull) return fail(EVG_ERR_INVALID, "P is out of range");
    evg_clip* c = new evg_clip();
    c->cfg = *cfg;
    c->cfg.layer_numel = nullptr;
    c->stream = static_cast<hipStream_t>(hip_stream);
    c->t.nchunks = (uint32_t)chunks.size();
    c->t.P = cfg->P;
    c->t.pitch = pitch;
    const size_t partials = (size_t)cfg->P * chunks.size() * 8, descs = chunks.size() * sizeof(ClipChunk);
    hipError_t e = hipMalloc(&c->owned, partials + descs + (size_t)cfg->P * 4);
    char* p = (char*)c->owned;
    if (e == hipSuccess) e = hipMemcpyAsync(p + partials, chunks.data(), descs, hipMemcpyHostToDevice, c->stream);
    if (e == hipSuccess) e = hipStreamSynchronize(c->stream);
    if (e != hipSuccess) {
      if (c->owned) (void)hipFree(c->owned);
      delete c;
      return fail(e == hipErrorOutOfMemory ? EVG_ERR_OOM : EVG_ERR_HIP, "tables: %s", hipGetErrorString(e));
    }
    c->t.partials = (double*)p;
    c->t.chunks = (const ClipChunk*)(p + partials);
    c->t.factor = (float*)(p + partials + descs);
    *out = c;
  } catch (const std::exception&) {
    return fail(EVG_ERR_OOM, "host allocation failed");
  }
  return EVG_OK;
}

evg_status evg_clip_run(evg_clip* c, const void* grad, void* out, float max_norm, float scale, float* norm) {
  if (!c || !grad || !out) return fail(EVG_ERR_INVALID, "context, grad and out must be non-NULL");
  if (!(max_norm >= 0.f)) return fail(EVG_ERR_INVALID, "max_norm must not be negative or NaN");
  if (!std::isfinite(scale)) return fail(EVG_ERR_INVALID, "scale must be finite");
  const uint32_t ge = type_bytes(c->cfg.grad_type), oe = type_bytes(c->cfg.out_type);
  if ((uintptr_t)grad % (4 * ge) || (uintptr_t)out % (4 * oe)) return fail(EVG_ERR_ALIGN, "grad and out must be aligned to four elements");
  if ((uintptr_t)norm % 4) return fail(EVG_ERR_ALIGN, "norm is not aligned to its elements");
  const uint64_t n = (uint64_t)c->t.P * c->t.pitch;
  evg_status st;
  if ((st = check_device_array(grad, n * ge, "grad")) != EVG_OK || (st = check_device_array(out, n * oe, "out")) != EVG_OK) return st;
  if (norm && (st = check_device_array(norm, (uint64_t)c->t.P * 4, "norm")) != EVG_OK) return st;
  const uintptr_t g = (uintptr_t)grad, o = (uintptr_t)out, m = (uintptr_t)norm;
  if (g < o + n * oe && o < g + n * ge && !(g == o && ge == oe)) return fail(EVG_ERR_INVALID, "out overlaps grad and is not grad itself");
  if (m && ((m < o + n * oe && o < m + c->t.P * 4ull) || (m < g + n * ge && g < m + c->t.P * 4ull))) return fail(EVG_ERR_INVALID, "norm overlaps an arena");
  const ClipCall call{max_norm, scale, c->cfg.eps, c->cfg.nonfinite == EVG_NONFINITE_ZERO, norm};
  hipError_t e;
  const bool wide = c->cfg.out_type == EVG_F32;
  if (c->cfg.grad_type == EVG_F32) e = launch_clip<float, float>(c->t, call, grad, out, c->stream);
  else if (c->cfg.grad_type == EVG_F16) e = wide ? launch_clip<half_t, float>(c->t, call, grad, out, c->stream) : launch_clip<half_t, half_t>(c->t, call, grad, out, c->stream);
  else e = wide ? launch_clip<bf16_t, float>(c->t, call, grad, out, c->stream) : launch_clip<bf16_t, bf16_t>(c->t, call, grad, out, c->stream);
  HIP_TRY(e);
  return EVG_OK;
}

evg_status evg_clip_destroy(evg_clip* c) {
  if (!c) return EVG_OK;
  hipError_t e = hipStreamSynchronize(c->stream);
  if (c->owned) { const hipError_t f = hipFree(c->owned); if (e == hipSuccess) e = f; }
  delete c;
  HIP_TRY(e);
  return EVG_OK;
}

}  // extern "C"
