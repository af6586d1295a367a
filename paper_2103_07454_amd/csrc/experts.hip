// Tokens by expert and back (include/evg_nn.h, evg_experts_*).
//
// The plan: entries i = t K + k sorted by expert, stable.  Runs of entries are counted by a workgroup each; then each workgroup adds up the counts of the runs
// ahead of its own and places its entries.  Few entries are placed by one workgroup a worker, in one launch.
//
// Rows move token by token: a token's row is read once and written to its K slots, or its K rows are read and added.  What
// leaves the chip is x once and the slots' rows once, whatever order the experts are in.  Slots that stay empty are zeroed by workgroups of
// the same launch that look through the plan's sources.  All are bound by memory.
#include <hip/hip_runtime.h>

#include <new>

#include "key_sort_device.h"
#include "nn_device.h"
#include "nn_host.h"

namespace evg {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kOneWaves = 16;
constexpr uint32_t kOneSort = 8192;     // most entries of a worker that one workgroup places
constexpr uint32_t kEmptySlots = 64;    // slots that a wavefront looks through

struct ExpertsArgs {
  evg_mat x, rows, d_rows;     // tokens' rows (x, y, dy) and slots' rows
  const int32_t* chosen;
  const float* weights;
  float* d_weights;
  int32_t *slot, *source, *counts;
  uint32_t workers, tokens, experts, top, width, capacity, slots, first;
  uint32_t run, runs, bits;
  uint32_t* run_counts;        // [workers][runs][experts]
  uint32_t blocks;             // column blocks of a token's row
  uint64_t token_groups;       // workgroups ahead of those that look for empty slots
};

// ---- the plan ------------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t expert_of(const ExpertsArgs& a, uint32_t w, uint32_t i) {
  const uint32_t e = (uint32_t)a.chosen[(uint64_t)w * a.tokens * a.top + i];
  return e < a.experts ? e : a.experts;
}

__global__ __launch_bounds__(kThreads) void k_experts_count(ExpertsArgs a) {
  __shared__ uint32_t counts[kMostBins];
  const uint32_t block = a.first + blockIdx.x, w = block / a.runs, r = block % a.runs, n = a.tokens * a.top, begin = r * a.run;
  for (uint32_t i = threadIdx.x; i < a.experts; i += kThreads) counts[i] = 0;
  __syncthreads();
  count_keys<kWaves>(counts, a.experts, min(a.run, n - begin), [&](uint32_t i) { return expert_of(a, w, begin + i); });
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < a.experts; i += kThreads) a.run_counts[((uint64_t)w * a.runs + r) * a.experts + i] = counts[i];
}

// ALONE: the workgroup has all of a worker's entries.
template <bool ALONE, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_experts_place(ExpertsArgs a) {
  constexpr uint32_t THREADS = WAVES * 64, EACH = (kMostBins + THREADS - 1) / THREADS;
  __shared__ uint32_t counts[WAVES * kMostBins], first[kMostBins], ahead[kMostBins], part[WAVES];
  const uint32_t block = a.first + blockIdx.x, w = ALONE ? block : block / a.runs, r = ALONE ? 0 : block % a.runs;
  const uint32_t n = a.tokens * a.top, begin = ALONE ? 0 : r * a.run, here = ALONE ? n : min(a.run, n - begin), E = a.experts;
  int32_t* const slot = a.slot + (uint64_t)w * n;
  int32_t* const source = a.source + (uint64_t)w * a.slots;
  for (uint32_t i = threadIdx.x; i < WAVES * E; i += THREADS) counts[i] = 0;
  __syncthreads();
  auto key = [&](uint32_t i) { return expert_of(a, w, begin + i); };
  count_keys<WAVES>(counts + threadIdx.x / 64 * E, E, here, key);
  __syncthreads();
#pragma unroll
  for (uint32_t j = 0; j < EACH; ++j) {
    const uint32_t e = j * THREADS + threadIdx.x;
    if (e < E) {
      uint32_t sum = 0, before = 0;
      if constexpr (ALONE) {
        for (int v = 0; v < WAVES; ++v) sum += counts[v * E + e];
      } else {
        const uint32_t* c = a.run_counts + (uint64_t)w * a.runs * E + e;
        for (uint32_t q = 0; q < a.runs; ++q, c += E) {
          if (q == r) before = sum;
          sum += *c;
        }
      }
      first[e] = sum;
      ahead[e] = before;
      if (r == 0) a.counts[(uint64_t)w * E + e] = (int32_t)sum;
    }
  }
  __syncthreads();
  if (!a.capacity) scan_bins<WAVES>(first, E, part);
  places_of_waves<WAVES>(counts, ahead, E);   // ranks among the expert's entries
  __syncthreads();
  place_keys<WAVES>(counts + threadIdx.x / 64 * E, E, (int)a.bits, here, key, [&](uint32_t i, uint32_t e, uint32_t rank) {
    const bool fits = !a.capacity || rank < a.capacity;
    const uint32_t at = a.capacity ? e * a.capacity + rank : first[e] + rank;
    slot[begin + i] = fits ? (int32_t)at : -1;
    if (fits) source[at] = (int32_t)(begin + i);
  });
  for (uint32_t i = threadIdx.x; i < here; i += THREADS)
    if (key(i) >= E) slot[begin + i] = -1;
}

// ---- rows ----------------------------------------------------------------------------------------------------------------------

// A slot that the tensors have, whatever the plan holds.
__device__ __forceinline__ bool real_slot(const ExpertsArgs& a, int32_t s) { return (uint32_t)s < a.slots; }

// Zeroes the rows of the empty ones among 64 slots.  PLANNED: the plan's sources tell which they are; else the counts do, and the sources are written.
template <typename T, bool PLANNED>
__device__ __forceinline__ void zero_empty(const ExpertsArgs& a, const evg_mat& rows, uint64_t job, int lane) {
  constexpr int E = 16 / sizeof(T);
  const uint32_t sets = (a.slots + kEmptySlots - 1) / kEmptySlots, w = (uint32_t)(job / sets), s0 = (uint32_t)(job % sets) * kEmptySlots;
  if (w >= a.workers) return;
  const uint32_t mine = s0 + lane;
  int32_t* const source = a.source + (uint64_t)w * a.slots;
  bool empty = mine < a.slots;
  if constexpr (PLANNED) {
    empty = empty && source[mine] < 0;
  } else {
    const int32_t* const counts = a.counts + (uint64_t)w * a.experts;
    if (a.capacity) {
      empty = empty && mine % a.capacity >= (uint32_t)counts[mine / a.capacity];
    } else {
      uint32_t sum = 0;
      for (uint32_t e = lane; e < a.experts; e += 64) sum += (uint32_t)counts[e];
      sum = wave_sum(sum);   // all lanes take part
      empty = empty && mine >= sum;
    }
    if (empty) source[mine] = -1;
  }
  const float zero[E] = {};
  for (uint64_t left = __ballot(empty); left; left &= left - 1) {
    const uint32_t s = s0 + (uint32_t)__ffsll((unsigned long long)left) - 1;
    T* const p = (T*)rows.p + (int64_t)w * rows.worker + (int64_t)s * rows.row;
    for (uint32_t col = lane * E; col < a.width; col += 64 * E) store_upto<E>(p + col, (int)(a.width - col), zero);
  }
}

// rows[slot] = x[t].  A wavefront has 64 vectors of a token's row.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_experts_dispatch(ExpertsArgs a) {
  constexpr int E = 16 / sizeof(T);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t group = (uint64_t)a.first + blockIdx.x;
  if (group >= a.token_groups) {
    zero_empty<T, false>(a, a.rows, (group - a.token_groups) * kWaves + wave, lane);
    return;
  }
  const uint64_t job = group * kWaves + wave, line = job / a.blocks;
  if (line >= (uint64_t)a.workers * a.tokens) return;
  const uint32_t w = (uint32_t)(line / a.tokens), t = (uint32_t)(line % a.tokens), col = (uint32_t)(job % a.blocks) * 64 * E + lane * E;
  const int n = (int)a.width - (int)col;
  if (n <= 0) return;
  const T* const p = (const T*)a.x.p + (int64_t)w * a.x.worker + (int64_t)t * a.x.row + col;
  T* const out = (T*)a.rows.p + (int64_t)w * a.rows.worker + col;
  const int32_t* const slot = a.slot + line * a.top;
  float v[E];
  load_upto<E>(p, n, v);
  for (uint32_t k = 0; k < a.top; ++k) {
    const int32_t s = slot[k];
    if (real_slot(a, s)) store_upto<E>(out + (int64_t)s * a.rows.row, n, v);
  }
}

// y[t] = sum over k of weights[i] rows[slot[i]].
template <typename T>
__global__ __launch_bounds__(kThreads) void k_experts_combine(ExpertsArgs a) {
  constexpr int E = 16 / sizeof(T);
  constexpr uint32_t AHEAD = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t job = ((uint64_t)a.first + blockIdx.x) * kWaves + wave, line = job / a.blocks;
  if (line >= (uint64_t)a.workers * a.tokens) return;
  const uint32_t w = (uint32_t)(line / a.tokens), t = (uint32_t)(line % a.tokens), col = (uint32_t)(job % a.blocks) * 64 * E + lane * E;
  const int n = (int)a.width - (int)col;
  if (n <= 0) return;
  const T* const p = (const T*)a.rows.p + (int64_t)w * a.rows.worker + col;
  const int32_t* const slot = a.slot + line * a.top;
  const float* const weights = a.weights + line * a.top;
  float acc[E] = {};
  for (uint32_t k = 0; k < a.top; k += AHEAD) {
    float v[AHEAD][E], f[AHEAD];
#pragma unroll
    for (uint32_t j = 0; j < AHEAD; ++j) {
      const int32_t s = k + j < a.top ? slot[k + j] : -1;
      const bool real = real_slot(a, s);
      f[j] = real ? (a.weights ? weights[k + j] : 1.f) : 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) v[j][e] = 0.f;
      if (real) load_upto<E>(p + (int64_t)s * a.rows.row, n, v[j]);
    }
#pragma unroll
    for (uint32_t j = 0; j < AHEAD; ++j)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(f[j], v[j][e], acc[e]);
  }
  store_upto<E>((T*)a.x.p + (int64_t)w * a.x.worker + (int64_t)t * a.x.row + col, n, acc);
}

// d_rows[slot] = weights[i] dy[t], d_weights[i] = <dy[t], rows[slot]>.  A wavefront has a token's whole row, four experts at a time.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_experts_combine_backward(ExpertsArgs a) {
  constexpr int E = 16 / sizeof(T);
  constexpr uint32_t AT_ONCE = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t group = (uint64_t)a.first + blockIdx.x;
  if (group >= a.token_groups) {
    zero_empty<T, true>(a, a.d_rows, (group - a.token_groups) * kWaves + wave, lane);
    return;
  }
  const uint64_t line = group * kWaves + wave;
  if (line >= (uint64_t)a.workers * a.tokens) return;
  const uint32_t w = (uint32_t)(line / a.tokens), t = (uint32_t)(line % a.tokens);
  const T* const dy = (const T*)a.x.p + (int64_t)w * a.x.worker + (int64_t)t * a.x.row;
  const T* const rows = (const T*)a.rows.p + (int64_t)w * a.rows.worker;
  T* const d_rows = (T*)a.d_rows.p + (int64_t)w * a.d_rows.worker;
  for (uint32_t k = 0; k < a.top; k += AT_ONCE) {
    int32_t s[AT_ONCE];
    float f[AT_ONCE], sum[AT_ONCE];
    bool real[AT_ONCE];
#pragma unroll
    for (uint32_t j = 0; j < AT_ONCE; ++j) {
      s[j] = k + j < a.top ? a.slot[line * a.top + k + j] : -1;
      real[j] = real_slot(a, s[j]);
      f[j] = real[j] ? a.weights[line * a.top + k + j] : 0.f;
      sum[j] = 0.f;
    }
    for (uint32_t col = lane * E; col < a.width; col += 64 * E) {
      const int n = (int)(a.width - col);
      float g[E];
      load_upto<E>(dy + col, n, g);
#pragma unroll
      for (uint32_t j = 0; j < AT_ONCE; ++j) {
        if (!real[j]) continue;
        float v[E];
        if (a.d_weights) {
          load_upto<E>(rows + (int64_t)s[j] * a.rows.row + col, n, v);
#pragma unroll
          for (int e = 0; e < E; ++e) sum[j] = fmaf(g[e], v[e], sum[j]);
        }
        if (a.d_rows.p) {
#pragma unroll
          for (int e = 0; e < E; ++e) v[e] = f[j] * g[e];
          store_upto<E>(d_rows + (int64_t)s[j] * a.d_rows.row + col, n, v);
        }
      }
    }
    if (a.d_weights) {
#pragma unroll
      for (uint32_t j = 0; j < AT_ONCE; ++j) {
        const float all = wave_sum_uniform(sum[j]);
        if (k + j < a.top && lane == 0) a.d_weights[line * a.top + k + j] = all;
      }
    }
  }
}

}  // namespace
}  // namespace evg

using namespace evg;

struct evg_experts {
  evg_experts_config cfg{};
  hipStream_t stream = nullptr;
  uint32_t* run_counts = nullptr;
};

namespace {

template <typename Kernel>
hipError_t launch(uint64_t groups, uint32_t threads, hipStream_t s, ExpertsArgs& a, Kernel kernel) {
  if (groups > 0x7FFFFFFFull) return hipErrorInvalidValue;
  launch_pieces(groups, threads, [&](uint32_t first, uint32_t grid) {
    a.first = first;
    kernel<<<grid, threads, 0, s>>>(a);
  });
  return hipGetLastError();
}

struct Sizes { uint64_t entries, slots; };   // of all workers

Sizes sizes_of(const evg_experts* c, uint32_t tokens) {
  return {(uint64_t)c->cfg.workers * tokens * c->cfg.top, c->cfg.workers * evg_experts_slots(c, tokens)};
}

ExpertsArgs experts_args(const evg_experts* c, uint32_t tokens, const evg_mat* x, const evg_mat* rows, const evg_mat* d_rows) {
  const evg_experts_config& g = c->cfg;
  ExpertsArgs a{};
  a.workers = g.workers, a.tokens = tokens, a.experts = g.experts, a.top = g.top, a.width = g.width, a.capacity = g.capacity;
  a.slots = (uint32_t)evg_experts_slots(c, tokens);
  const evg_mat none{};
  a.x = *x;
  a.rows = rows ? *rows : none;
  a.d_rows = d_rows ? *d_rows : none;
  if (g.workers <= 1) a.x.worker = a.rows.worker = a.d_rows.worker = 0;
  if (tokens <= 1) a.x.row = 0;
  if (a.slots <= 1) a.rows.row = a.d_rows.row = 0;
  const uint32_t across = 64 * 16 / type_bytes(g.type);
  a.blocks = (g.width + across - 1) / across;
  return a;
}

uint64_t empty_groups(const ExpertsArgs& a) {
  return ((uint64_t)a.workers * ((a.slots + kEmptySlots - 1) / kEmptySlots) + kWaves - 1) / kWaves;
}

template <typename T>
hipError_t dispatch(const evg_experts* c, ExpertsArgs& a) {
  const uint32_t n = a.tokens * a.top;
  hipError_t e;
  while ((1u << a.bits) < a.experts) ++a.bits;
  if (n <= kOneSort) {
    if ((e = launch(a.workers, kOneWaves * 64, c->stream, a, k_experts_place<true, kOneWaves>)) != hipSuccess) return e;
  } else {
    const Runs runs = cut_runs(n);
    a.run = runs.each, a.runs = runs.count;
    const uint64_t groups = (uint64_t)a.workers * a.runs;
    if ((e = launch(groups, kThreads, c->stream, a, k_experts_count)) != hipSuccess) return e;
    if ((e = launch(groups, kThreads, c->stream, a, k_experts_place<false, kWaves>)) != hipSuccess) return e;
  }
  a.token_groups = ((uint64_t)a.workers * a.tokens * a.blocks + kWaves - 1) / kWaves;
  return launch(a.token_groups + empty_groups(a), kThreads, c->stream, a, k_experts_dispatch<T>);
}

template <typename T>
hipError_t combine(const evg_experts* c, ExpertsArgs& a) {
  return launch(((uint64_t)a.workers * a.tokens * a.blocks + kWaves - 1) / kWaves, kThreads, c->stream, a, k_experts_combine<T>);
}

template <typename T>
hipError_t combine_backward(const evg_experts* c, ExpertsArgs& a) {
  a.token_groups = ((uint64_t)a.workers * a.tokens + kWaves - 1) / kWaves;
  return launch(a.token_groups + (a.d_rows.p ? empty_groups(a) : 0), kThreads, c->stream, a, k_experts_combine_backward<T>);
}

evg_status check_plan(const evg_experts* c, uint32_t tokens, const evg_experts_plan* plan, bool source, bool counts) {
  if (!plan) return fail(EVG_ERR_INVALID, "plan must be given");
  const Sizes n = sizes_of(c, tokens);
  evg_status st;
  if ((st = check_array(plan->slot, n.entries, "slot")) != EVG_OK) return st;
  if (source && (st = check_array(plan->source, n.slots, "source")) != EVG_OK) return st;
  if (counts && (st = check_array(plan->counts, (uint64_t)c->cfg.workers * c->cfg.experts, "counts")) != EVG_OK) return st;
  return EVG_OK;
}

}  // namespace

extern "C" {

evg_status evg_experts_init(evg_experts** out, const evg_experts_config* cfg, void* hip_stream) {
  if (!out || !cfg) return fail(EVG_ERR_INVALID, "out and cfg must be non-NULL");
  *out = nullptr;
  if (cfg->workers < 1 || cfg->workers > 65535) return fail(EVG_ERR_INVALID, "workers must be 1 .. 65535");
  if (cfg->experts < 1 || cfg->experts > EVG_ROUTER_MAX_EXPERTS) return fail(EVG_ERR_INVALID, "experts must be 1 .. %u", EVG_ROUTER_MAX_EXPERTS);
  if (cfg->top < 1 || cfg->top > cfg->experts) return fail(EVG_ERR_INVALID, "top must be 1 .. experts");
  if (cfg->width < 1 || cfg->width > (1u << 20)) return fail(EVG_ERR_INVALID, "width must be 1 .. 2^20");
  if ((uint64_t)cfg->max_tokens * cfg->top >> 28) return fail(EVG_ERR_INVALID, "max_tokens and top together must be below 2^28");
  if ((uint64_t)cfg->experts * cfg->capacity >> 31) return fail(EVG_ERR_INVALID, "experts and capacity together must be below 2^31");
  const uint64_t slots = cfg->capacity ? (uint64_t)cfg->experts * cfg->capacity : (uint64_t)cfg->max_tokens * cfg->top;
  const uint64_t blocks = ((uint64_t)cfg->width * 4 + 1023) / 1024;
  if (cfg->workers * ((uint64_t)cfg->max_tokens * blocks + slots / kEmptySlots + 1) / kWaves > 0x7FFF0000ull)
    return fail(EVG_ERR_INVALID, "workers, max_tokens, width and capacity together are out of range");
  evg_status st;
  if ((st = check_type(cfg->type, "type")) != EVG_OK) return st;
  evg_experts* c = new (std::nothrow) evg_experts();
  if (!c) return fail(EVG_ERR_OOM, "host allocation failed");
  c->cfg = *cfg;
  c->stream = static_cast<hipStream_t>(hip_stream);
  if ((uint64_t)cfg->max_tokens * cfg->top > kOneSort) {
    const hipError_t e = hipMalloc((void**)&c->run_counts, (uint64_t)cfg->workers * 128 * cfg->experts * 4);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      delete c;
      return fail(e == hipErrorOutOfMemory ? EVG_ERR_OOM : EVG_ERR_HIP, "workspace: %s", hipGetErrorString(e));
    }
  }
  *out = c;
  return EVG_OK;
}

uint64_t evg_experts_slots(const evg_experts* c, uint32_t tokens) {
  if (!c) return 0;
  return c->cfg.capacity ? (uint64_t)c->cfg.experts * c->cfg.capacity : (uint64_t)tokens * c->cfg.top;
}

evg_status evg_experts_dispatch(evg_experts* c, uint32_t tokens, const evg_mat* x, const int32_t* chosen, const evg_mat* rows,
                                const evg_experts_plan* plan) {
  if (!c) return fail(EVG_ERR_INVALID, "context must be non-NULL");
  const evg_experts_config& g = c->cfg;
  if (tokens > g.max_tokens) return fail(EVG_ERR_INVALID, "tokens exceeds the context's max_tokens");
  const uint64_t slots = evg_experts_slots(c, tokens);
  const Sizes n = sizes_of(c, tokens);
  evg_status st;
  if ((st = check_plan(c, tokens, plan, true, true)) != EVG_OK) return st;
  if ((st = check_array(chosen, n.entries, "chosen")) != EVG_OK) return st;
  if ((st = check_mat(x, g.workers, tokens, g.width, g.type, false, "x")) != EVG_OK) return st;
  if ((st = check_mat(rows, g.workers, slots, g.width, g.type, true, "rows")) != EVG_OK) return st;
  const Span ins[] = {mat_span(x, g.workers, tokens, g.width, g.type, "x"), array_span(chosen, n.entries, "chosen")};
  const Span outs[] = {mat_span(rows, g.workers, slots, g.width, g.type, "rows"), array_span(plan->slot, n.entries, "slot"),
                       array_span(plan->source, n.slots, "source"), array_span(plan->counts, (uint64_t)g.workers * g.experts, "counts")};
  if ((st = check_apart(outs, 4, ins, 2)) != EVG_OK) return st;
  ExpertsArgs a = experts_args(c, tokens, x, rows, nullptr);
  a.chosen = chosen;
  a.slot = plan->slot, a.source = plan->source, a.counts = plan->counts;
  a.run_counts = c->run_counts;
  HIP_TRY(g.type == EVG_F32 ? dispatch<float>(c, a) : g.type == EVG_F16 ? dispatch<half_t>(c, a) : dispatch<bf16_t>(c, a));
  return EVG_OK;
}

evg_status evg_experts_combine(evg_experts* c, uint32_t tokens, const evg_mat* rows, const float* weights, const evg_experts_plan* plan,
                               const evg_mat* y) {
  if (!c) return fail(EVG_ERR_INVALID, "context must be non-NULL");
  const evg_experts_config& g = c->cfg;
  if (tokens > g.max_tokens) return fail(EVG_ERR_INVALID, "tokens exceeds the context's max_tokens");
  const uint64_t slots = evg_experts_slots(c, tokens);
  const Sizes n = sizes_of(c, tokens);
  evg_status st;
  if ((st = check_plan(c, tokens, plan, false, false)) != EVG_OK) return st;
  if (weights && (st = check_array(weights, n.entries, "weights")) != EVG_OK) return st;
  if ((st = check_mat(rows, g.workers, slots, g.width, g.type, false, "rows")) != EVG_OK) return st;
  if ((st = check_mat(y, g.workers, tokens, g.width, g.type, true, "y")) != EVG_OK) return st;
  const Span ins[] = {mat_span(rows, g.workers, slots, g.width, g.type, "rows"), array_span(weights, n.entries, "weights"), array_span(plan->slot, n.entries, "slot")};
  const Span outs[] = {mat_span(y, g.workers, tokens, g.width, g.type, "y")};
  if ((st = check_apart(outs, 1, ins, 3)) != EVG_OK) return st;
  if (!tokens) return EVG_OK;
  ExpertsArgs a = experts_args(c, tokens, y, rows, nullptr);
  a.weights = weights;
  a.slot = plan->slot;
  HIP_TRY(g.type == EVG_F32 ? combine<float>(c, a) : g.type == EVG_F16 ? combine<half_t>(c, a) : combine<bf16_t>(c, a));
  return EVG_OK;
}

evg_status evg_experts_combine_backward(evg_experts* c, uint32_t tokens, const evg_mat* dy, const evg_mat* rows, const float* weights,
                                        const evg_experts_plan* plan, const evg_mat* d_rows, float* d_weights) {
  if (!c) return fail(EVG_ERR_INVALID, "context must be non-NULL");
  const evg_experts_config& g = c->cfg;
  if (tokens > g.max_tokens) return fail(EVG_ERR_INVALID, "tokens exceeds the context's max_tokens");
  const uint64_t slots = evg_experts_slots(c, tokens);
  const Sizes n = sizes_of(c, tokens);
  const bool has_rows = d_rows && d_rows->p;
  evg_status st;
  if ((st = check_plan(c, tokens, plan, has_rows, false)) != EVG_OK) return st;
  if ((st = check_array(weights, n.entries, "weights")) != EVG_OK) return st;
  if ((st = check_mat(dy, g.workers, tokens, g.width, g.type, false, "dy")) != EVG_OK) return st;
  if (d_weights && (st = check_mat(rows, g.workers, slots, g.width, g.type, false, "rows")) != EVG_OK) return st;
  if (d_weights && (st = check_array(d_weights, n.entries, "d_weights")) != EVG_OK) return st;
  if (has_rows && (st = check_mat(d_rows, g.workers, slots, g.width, g.type, true, "d_rows")) != EVG_OK) return st;
  const Span ins[] = {mat_span(dy, g.workers, tokens, g.width, g.type, "dy"), mat_span(d_weights ? rows : nullptr, g.workers, slots, g.width, g.type, "rows"),
                      array_span(weights, n.entries, "weights"), array_span(plan->slot, n.entries, "slot"),
                      array_span(has_rows ? plan->source : nullptr, n.slots, "source")};
  const Span outs[] = {mat_span(d_rows, g.workers, slots, g.width, g.type, "d_rows"), array_span(d_weights, n.entries, "d_weights")};
  if ((st = check_apart(outs, 2, ins, 5)) != EVG_OK) return st;
  if (!has_rows && !d_weights) return EVG_OK;
  ExpertsArgs a = experts_args(c, tokens, dy, d_weights ? rows : nullptr, d_rows);
  a.weights = weights;
  a.d_weights = d_weights;
  a.slot = plan->slot, a.source = plan->source;
  HIP_TRY(g.type == EVG_F32 ? combine_backward<float>(c, a) : g.type == EVG_F16 ? combine_backward<half_t>(c, a) : combine_backward<bf16_t>(c, a));
  return EVG_OK;
}

evg_status evg_experts_destroy(evg_experts* c) {
  if (!c) return EVG_OK;
  hipError_t e = hipStreamSynchronize(c->stream);
  if (c->run_counts) { const hipError_t f = hipFree(c->run_counts); if (e == hipSuccess) e = f; }
  delete c;
  HIP_TRY(e);
  return EVG_OK;
}

}  // extern "C"
