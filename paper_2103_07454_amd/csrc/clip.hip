// Clipping of each worker's gradient by its global norm (include/evg_nn.h, evg_clip_*).
//
// With s the scale, for worker r:  norm = |s| sqrt(sum_j g_j^2) over all its tensors,  out_j = g_j * (s * min(1, max / (norm + eps))).
// No product can be written before the last square is summed, so the gradient is read twice.  Both passes are bound by memory.
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

// A run of elements of a worker's slice without padding in it.
struct ClipChunk { uint32_t off, len; };   // off: a multiple of 4

struct ClipTables {
  const ClipChunk* chunks;
  uint32_t nchunks, P;
  uint64_t pitch;        // elements of a worker's slice
  double* partials;      // [P][nchunks]
  uint32_t* arrived;     // [P], 0 between launches
  float* factor;         // [P]
};

struct ClipCall {
  float max_norm, scale, eps;
  uint32_t zero_nonfinite;
  float* norm;           // [P] or null
};

// One workgroup sums the squares of a chunk; a worker's last one to arrive adds the chunks' sums, in their order, and leaves the factor.
template <typename T>
__global__ __launch_bounds__(kClipThreads) void k_clip_norm(ClipTables t, ClipCall call, const T* __restrict__ grad) {
  constexpr int E = 16 / sizeof(T);
  __shared__ double part[kClipThreads / 64];
  __shared__ bool last;
  const uint32_t r = blockIdx.x / t.nchunks, c = blockIdx.x % t.nchunks;
  const ClipChunk d = t.chunks[c];
  const T* g = grad + (uint64_t)r * t.pitch + d.off;
  double sum = 0.0;
#pragma unroll 4
  for (uint32_t j = threadIdx.x * E; j < d.len; j += kClipThreads * E) {
    float v[E];
    load_upto<E>(g + j, (int)(d.len - j), v);
#pragma unroll
    for (int i = 0; i < E; ++i) sum = fma((double)v[i], (double)v[i], sum);
  }
  const int wave = threadIdx.x / 64;
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) part[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = part[0];
    for (int i = 1; i < kClipThreads / 64; ++i) sum += part[i];
    __hip_atomic_store(&t.partials[(uint64_t)r * t.nchunks + c], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = __hip_atomic_fetch_add(&t.arrived[r], 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == t.nchunks - 1;
  }
  __syncthreads();
  if (!last) return;
  sum = 0.0;
  for (uint32_t i = threadIdx.x; i < t.nchunks; i += kClipThreads)
    sum += __hip_atomic_load(&t.partials[(uint64_t)r * t.nchunks + i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) part[wave] = sum;
  __syncthreads();
  if (threadIdx.x) return;
  sum = part[0];
  for (int i = 1; i < kClipThreads / 64; ++i) sum += part[i];
  const float norm = (float)(sqrt(sum) * fabs((double)call.scale));
  const float keep = call.max_norm / (norm + call.eps);
  float factor = call.scale * (keep > 1.f ? 1.f : keep);   // a NaN stays one
  if (call.zero_nonfinite && !(norm <= 3.402823466e38f)) factor = 0.f;
  t.factor[r] = factor;
  if (call.norm) call.norm[r] = norm;
  t.arrived[r] = 0;
}

template <typename T, typename U>
__global__ __launch_bounds__(kClipThreads) void k_clip_scale(ClipTables t, ClipCall call, const T* __restrict__ grad, U* __restrict__ out, bool in_place) {
  constexpr int E = 16 / sizeof(U);
  const uint32_t r = blockIdx.x / t.nchunks, c = blockIdx.x % t.nchunks;
  const float f = t.factor[r];
  if (in_place && f == 1.f) return;
  const bool zero = call.zero_nonfinite && f == 0.f;   // also where an element is not finite
  const ClipChunk d = t.chunks[c];
  const T* g = grad + (uint64_t)r * t.pitch + d.off;
  U* o = out + (uint64_t)r * t.pitch + d.off;
#pragma unroll 4
  for (uint32_t j = threadIdx.x * E; j < d.len; j += kClipThreads * E) {
    float v[E];
    load_upto<E>(g + j, (int)(d.len - j), v);
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = zero ? 0.f : v[i] * f;
    store_upto<E>(o + j, (int)(d.len - j), v);
  }
}

template <typename T, typename U>
hipError_t launch_clip(const ClipTables& t, const ClipCall& call, const void* grad, void* out, hipStream_t s) {
  const uint32_t grid = t.P * t.nchunks;
  k_clip_norm<T><<<grid, kClipThreads, 0, s>>>(t, call, (const T*)grad);
  k_clip_scale<T, U><<<grid, kClipThreads, 0, s>>>(t, call, (const T*)grad, (U*)out, grad == out);
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
    const uint64_t most = (uint64_t)cfg->P * pitch <= (8u << 20) ? 2048 : 8192;
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
    const size_t partials = (size_t)cfg->P * chunks.size() * 8, descs = chunks.size() * sizeof(ClipChunk), words = ((size_t)cfg->P * 4 + 7) / 8 * 8;
    hipError_t e = hipMalloc(&c->owned, partials + descs + 2 * words);
    if (e == hipSuccess) e = hipMemsetAsync(c->owned, 0, partials + descs + 2 * words, c->stream);
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
    c->t.arrived = (uint32_t*)(p + partials + descs);
    c->t.factor = (float*)(p + partials + descs + words);
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
