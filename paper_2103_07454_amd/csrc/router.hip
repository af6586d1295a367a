// Which experts a token goes to, and the gradient of their weights (include/evg_nn.h, evg_router_*).
//
// A token's logits lie in the registers of 1 to 64 lanes, eight to a lane (sixteen above 512 experts).  K times the lanes find the largest
// among those not chosen yet: a lane its own, then the group by exchanges, of one word that has the logit's rank above and
// the expert's number, turned round, below.  So equal logits go to the lowest number, and the order of the lanes is of no matter.
// A logit of 16 bits and its number fit a word of 32 bits, one of 32 needs 64.
//
// Bound by the choices' instructions, some thirty each, and by latency: 128 experts of 32768 tokens in bfloat16, top 8, 9.9 us (8 MB in, 2 MB out), of which a wavefront
// keeps what was chosen in LDS (13.2 with each lane noting the places of its own experts; 22 with words of 64 bits); the gradient 8.2, with three
// reductions over a row's lanes by exchanges through LDS, each waiting for the last.
#include <hip/hip_runtime.h>

#include <new>

#include "nn_device.h"
#include "nn_host.h"

namespace evg {
namespace {

constexpr int kThreads = 256;

struct RouterArgs {
  evg_mat logits, d_logits;
  int32_t* chosen;
  float* weights;             // d_weights in the backward pass
  uint64_t lines;             // workers * tokens
  uint32_t tokens, experts, top, over_chosen, first;
};

// A logit and its expert as a whole number, ordered as they are chosen: a NaN highest, then by value, both zeros one, then the lowest number.  0 for minus
// infinity, which is never chosen.
template <typename T> struct Word {
  typedef uint32_t type;
  static __device__ __forceinline__ type of(float v, int e) {   // exact in T
    const uint32_t b = __builtin_bit_cast(uint16_t, from_f<T>(v + 0.f));
    const uint32_t r = v != v ? 0xFFFFu : b & 0x8000u ? ~b & 0xFFFFu : b | 0x8000u;
    return v == -INFINITY ? 0 : r << 16 | (0xFFFFu - e);
  }
  static __device__ __forceinline__ int expert(type w) { return (int)(0xFFFFu - (w & 0xFFFFu)); }
  static __device__ __forceinline__ float value(type w) {
    const uint32_t r = w >> 16;
    return r == 0xFFFFu ? NAN : to_f(__builtin_bit_cast(T, (uint16_t)(r & 0x8000u ? r & 0x7FFFu : ~r)));
  }
};
template <> struct Word<float> {
  typedef uint64_t type;
  static __device__ __forceinline__ type of(float v, int e) {
    const uint32_t b = __float_as_uint(v + 0.f);
    const uint32_t r = v != v ? 0xFFFFFFFFu : b & 0x80000000u ? ~b : b | 0x80000000u;
    return v == -INFINITY ? 0 : (uint64_t)r << 32 | (0xFFFFFFFFu - (uint32_t)e);
  }
  static __device__ __forceinline__ int expert(type w) { return (int)(0xFFFFFFFFu - (uint32_t)w); }
  static __device__ __forceinline__ float value(type w) {
    const uint32_t r = (uint32_t)(w >> 32);
    return r == 0xFFFFFFFFu ? NAN : __uint_as_float(r & 0x80000000u ? r & 0x7FFFFFFFu : ~r);
  }
};

// The same of another lane, by data-parallel moves within 16 lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t moved_word(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false); }
template <int CTRL>
__device__ __forceinline__ uint64_t moved_word(uint64_t v) { return (uint64_t)moved_word<CTRL>((uint32_t)(v >> 32)) << 32 | moved_word<CTRL>((uint32_t)v); }

// The largest of a group's words, in all of its lanes.
template <int LANES, typename W>
__device__ __forceinline__ W lanes_largest(W v) {
  if constexpr (LANES >= 2) v = max(v, moved_word<0xB1>(v));    // lanes 1 0 3 2
  if constexpr (LANES >= 4) v = max(v, moved_word<0x4E>(v));    // lanes 2 3 0 1
  if constexpr (LANES >= 8) v = max(v, moved_word<0x141>(v));   // mirrored within 8
  if constexpr (LANES >= 16) v = max(v, moved_word<0x140>(v));  // mirrored within 16
  if constexpr (LANES >= 32) v = max(v, (W)__shfl_xor(v, 16, 64));
  if constexpr (LANES >= 64) v = max(v, (W)__shfl_xor(v, 32, 64));
  return v;
}

template <int LANES>
__device__ __forceinline__ float lanes_total(float v) {
#pragma unroll
  for (int d = 1; d < LANES; d <<= 1) v += __shfl_xor(v, d, LANES);
  return v;
}

template <int LANES>
__device__ __forceinline__ float lanes_most(float v) {
#pragma unroll
  for (int d = 1; d < LANES; d <<= 1) v = fmaxf(v, __shfl_xor(v, d, LANES));
  return v;
}

// This lane's logits; minus infinity behind the last one.
template <int PER, typename T>
__device__ __forceinline__ void load_logits(const T* p, int n, float* v) {
#pragma unroll
  for (int i = 0; i < PER; i += 8) {
    if (n >= i + 8) {
      load_n<8>(p + i, v + i);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i + j] = i + j < n ? to_f(p[i + j]) : -INFINITY;
    }
  }
}

template <typename T, int LANES, int PER>
__global__ __launch_bounds__(kThreads) void k_router(RouterArgs a) {
  const uint32_t row = (a.first + blockIdx.x) * (kThreads / LANES) + threadIdx.x / LANES;
  if (row >= a.lines) return;   // all of a group's lanes at once
  const uint32_t w = row / a.tokens, t = row % a.tokens;
  const uint64_t line = row;
  const int lane = threadIdx.x % LANES, first = lane * PER;
  float v[PER];
  load_logits<PER>((const T*)a.logits.p + (int64_t)w * a.logits.worker + (int64_t)t * a.logits.row + first, (int)a.experts - first, v);
  typedef typename Word<T>::type W;
  __shared__ W words[kThreads * PER];   // each group's choices, in their order
  W* const picked = words + threadIdx.x / LANES * (LANES * PER);
  W word[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) word[i] = Word<T>::of(v[i], first + i);
  float most = 0.f;
  uint32_t count = 0;
  for (; count < a.top; ++count) {
    W best = word[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) best = max(best, word[i]);
    best = lanes_largest<LANES>(best);
    if (!best) break;   // none is left
    if (count == 0) most = Word<T>::value(best);
    if (lane == 0) picked[count] = best;
#pragma unroll
    for (int i = 0; i < PER; ++i) word[i] = word[i] == best ? 0 : word[i];   // words differ
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  float total = 0.f;
  if (a.over_chosen) {
    for (uint32_t k = lane; k < count; k += LANES) total += expf(Word<T>::value(picked[k]) - most);
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) total += expf(v[i] - most);
  }
  total = lanes_total<LANES>(total);
  int32_t* const chosen = a.chosen + line * a.top;
  float* const weights = a.weights + line * a.top;
  for (uint32_t k = lane; k < a.top; k += LANES) {
    const bool there = k < count;
    const W w_k = there ? picked[k] : 0;
    chosen[k] = there ? Word<T>::expert(w_k) : -1;
    weights[k] = there ? expf(Word<T>::value(w_k) - most) / total : 0.f;
  }
}

template <typename T, int LANES, int PER>
__global__ __launch_bounds__(kThreads) void k_router_backward(RouterArgs a) {
  const uint32_t row = (a.first + blockIdx.x) * (kThreads / LANES) + threadIdx.x / LANES;
  if (row >= a.lines) return;
  const uint32_t w = row / a.tokens, t = row % a.tokens;
  const uint64_t line = row;
  const int lane = threadIdx.x % LANES, first = lane * PER;
  const T* const logits = (const T*)a.logits.p + (int64_t)w * a.logits.worker + (int64_t)t * a.logits.row;
  const int32_t* const chosen = a.chosen + line * a.top;
  const float* const dw = a.weights + line * a.top;
  float v[PER], d[PER];
  bool mine[PER];   // is it chosen?
  load_logits<PER>(logits + first, (int)a.experts - first, v);
  // The chosen find their experts' lanes through LDS, each expert its last place among them; a group's lanes are of one wavefront.
  __shared__ int places[kThreads * PER];
  __shared__ float found[kThreads * PER];
  int* const place = places + threadIdx.x / LANES * (LANES * PER);
  float* const given = found + threadIdx.x / LANES * (LANES * PER);
#pragma unroll
  for (int i = 0; i < PER; ++i) place[first + i] = -1;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  for (uint32_t k = lane; k < a.top; k += LANES) {
    const int e = chosen[k];
    given[k] = dw[k];
    if ((uint32_t)e < a.experts) atomicMax(&place[e], (int)k);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = place[first + i];
    mine[i] = k >= 0;
    d[i] = k >= 0 ? given[k] : 0.f;
  }
  // The softmax over what counts; all that is chosen, or all.
  float most = -INFINITY, total = 0.f, inner = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (a.over_chosen && !mine[i]) v[i] = -INFINITY;
    most = fmaxf(most, v[i]);
  }
  most = lanes_most<LANES>(most);
  if (most == -INFINITY) most = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    v[i] = sizeof(T) == 2 ? __expf(v[i] - most) : expf(v[i] - most);   // results of 16 bits: the hardware's, off by some 2^-23 for each unit of the exponent
    total += v[i];
  }
  total = lanes_total<LANES>(total);
  const float part = total > 0.f || total != total ? 1.f / total : 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    v[i] *= part;
    inner += mine[i] ? v[i] * d[i] : 0.f;
  }
  inner = lanes_total<LANES>(inner);
#pragma unroll
  for (int i = 0; i < PER; ++i) d[i] = a.over_chosen && !mine[i] ? 0.f : v[i] * (d[i] - inner);
  T* const out = (T*)a.d_logits.p + (int64_t)w * a.d_logits.worker + (int64_t)t * a.d_logits.row + first;
#pragma unroll
  for (int i = 0; i < PER; i += 8) store_upto<8>(out + i, (int)a.experts - first - i, d + i);
}

template <typename T, int LANES, int PER>
hipError_t launch_lanes(RouterArgs a, bool backward, hipStream_t s) {
  const uint64_t per = kThreads / LANES, groups = (a.lines + per - 1) / per;
  if (groups > 0x7FFFFFFFull) return hipErrorInvalidValue;
  launch_pieces(groups, kThreads, [&](uint32_t first, uint32_t grid) {
    a.first = first;
    if (backward) k_router_backward<T, LANES, PER><<<grid, kThreads, 0, s>>>(a);
    else k_router<T, LANES, PER><<<grid, kThreads, 0, s>>>(a);
  });
  return hipGetLastError();
}

template <typename T>
hipError_t launch_router(const RouterArgs& a, bool backward, hipStream_t s) {
  if (a.experts <= 8) return launch_lanes<T, 1, 8>(a, backward, s);
  if (a.experts <= 16) return launch_lanes<T, 2, 8>(a, backward, s);
  if (a.experts <= 32) return launch_lanes<T, 4, 8>(a, backward, s);
  if (a.experts <= 64) return launch_lanes<T, 8, 8>(a, backward, s);
  if (a.experts <= 128) return launch_lanes<T, 16, 8>(a, backward, s);
  if (a.experts <= 256) return launch_lanes<T, 32, 8>(a, backward, s);
  if (a.experts <= 512) return launch_lanes<T, 64, 8>(a, backward, s);
  return launch_lanes<T, 64, 16>(a, backward, s);
}

}  // namespace
}  // namespace evg

using namespace evg;

struct evg_router {
  evg_router_config cfg{};
  hipStream_t stream = nullptr;
};

namespace {

hipError_t launch_any(const evg_router* c, RouterArgs& a, uint32_t tokens, bool backward) {
  const evg_router_config& g = c->cfg;
  a.lines = (uint64_t)g.workers * tokens;
  a.tokens = tokens, a.experts = g.experts, a.top = g.top, a.over_chosen = g.over_chosen;
  for (evg_mat* m : {&a.logits, &a.d_logits}) {
    if (g.workers <= 1) m->worker = 0;
    if (tokens <= 1) m->row = 0;
  }
  if (g.type == EVG_F32) return launch_router<float>(a, backward, c->stream);
  if (g.type == EVG_F16) return launch_router<half_t>(a, backward, c->stream);
  return launch_router<bf16_t>(a, backward, c->stream);
}

}  // namespace

extern "C" {

evg_status evg_router_init(evg_router** out, const evg_router_config* cfg, void* hip_stream) {
  if (!out || !cfg) return fail(EVG_ERR_INVALID, "out and cfg must be non-NULL");
  *out = nullptr;
  if (cfg->workers < 1) return fail(EVG_ERR_INVALID, "workers must be at least 1");
  if (cfg->experts < 1 || cfg->experts > EVG_ROUTER_MAX_EXPERTS) return fail(EVG_ERR_INVALID, "experts must be 1 .. %u", EVG_ROUTER_MAX_EXPERTS);
  if (cfg->top < 1 || cfg->top > cfg->experts) return fail(EVG_ERR_INVALID, "top must be 1 .. experts");
  if ((uint64_t)cfg->workers * cfg->max_tokens > 0x7FFFFFFFull) return fail(EVG_ERR_INVALID, "workers and max_tokens together are out of range");
  evg_status st;
  if ((st = check_type(cfg->type, "type")) != EVG_OK) return st;
  evg_router* c = new (std::nothrow) evg_router();
  if (!c) return fail(EVG_ERR_OOM, "host allocation failed");
  c->cfg = *cfg;
  c->stream = static_cast<hipStream_t>(hip_stream);
  *out = c;
  return EVG_OK;
}

evg_status evg_router_forward(evg_router* c, uint32_t tokens, const evg_mat* logits, int32_t* chosen, float* weights) {
  if (!c) return fail(EVG_ERR_INVALID, "context must be non-NULL");
  const evg_router_config& g = c->cfg;
  if (tokens > g.max_tokens) return fail(EVG_ERR_INVALID, "tokens exceeds the context's max_tokens");
  const uint64_t n = (uint64_t)g.workers * tokens * g.top;
  evg_status st;
  if ((st = check_mat(logits, g.workers, tokens, g.experts, g.type, false, "logits")) != EVG_OK) return st;
  if ((st = check_array(chosen, n, "chosen")) != EVG_OK || (st = check_array(weights, n, "weights")) != EVG_OK) return st;
  const Span ins[] = {mat_span(logits, g.workers, tokens, g.experts, g.type, "logits")};
  const Span outs[] = {array_span(chosen, n, "chosen"), array_span(weights, n, "weights")};
  if ((st = check_apart(outs, 2, ins, 1)) != EVG_OK) return st;
  if (!n) return EVG_OK;
  RouterArgs a{};
  a.logits = *logits;
  a.chosen = chosen;
  a.weights = weights;
  HIP_TRY(launch_any(c, a, tokens, false));
  return EVG_OK;
}

evg_status evg_router_backward(evg_router* c, uint32_t tokens, const float* d_weights, const evg_mat* logits, const int32_t* chosen,
                               const evg_mat* d_logits) {
  if (!c) return fail(EVG_ERR_INVALID, "context must be non-NULL");
  const evg_router_config& g = c->cfg;
  if (tokens > g.max_tokens) return fail(EVG_ERR_INVALID, "tokens exceeds the context's max_tokens");
  const uint64_t n = (uint64_t)g.workers * tokens * g.top;
  evg_status st;
  if ((st = check_array(d_weights, n, "d_weights")) != EVG_OK || (st = check_array(chosen, n, "chosen")) != EVG_OK) return st;
  if ((st = check_mat(logits, g.workers, tokens, g.experts, g.type, false, "logits")) != EVG_OK) return st;
  if ((st = check_mat(d_logits, g.workers, tokens, g.experts, g.type, true, "d_logits")) != EVG_OK) return st;
  const Span ins[] = {mat_span(logits, g.workers, tokens, g.experts, g.type, "logits"), array_span(d_weights, n, "d_weights"), array_span(chosen, n, "chosen")};
  const Span outs[] = {mat_span(d_logits, g.workers, tokens, g.experts, g.type, "d_logits")};
  if ((st = check_apart(outs, 1, ins, 3, 0, 0)) != EVG_OK) return st;
  if (!n) return EVG_OK;
  RouterArgs a{};
  a.logits = *logits;
  a.d_logits = *d_logits;
  a.chosen = const_cast<int32_t*>(chosen);
  a.weights = const_cast<float*>(d_weights);
  HIP_TRY(launch_any(c, a, tokens, true));
  return EVG_OK;
}

evg_status evg_router_destroy(evg_router* c) {
  delete c;
  return EVG_OK;
}

}  // extern "C"
