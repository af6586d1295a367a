// Tokens by expert and back (include/evg_nn.h, evg_experts_*).
//
// The plan: entries i = t K + k sorted by expert, stable.  Runs of entries are counted by a workgroup each; then each workgroup adds up the counts of the runs
// ahead of its own and places its entries.  Few entries are placed by one workgroup a worker, in one launch.
//
// Rows move token by token: a token's row is read once and written to its K slots, or its K rows are read and added.  What
// leaves the chip is x once and the slots' rows once, whatever order the experts are in.  Slots that stay empty are zeroed by workgroups of
// the same launch that look through the plan's sources.  All are bound by memory: 16384 tokens at 8 of 64 experts, 2048 wide in bfloat16, the plan 19 us, dispatch 122 (604 MB,
// 5.0 TB/s), combine 103 (5.9), its backward pass 230 (1141 MB, 5.0); with rows through the caches and a unit at a time 159, 160 and 266.
#include <hip/hip_runtime.h>

#include <new>

#include "key_sort_device.h"
#include "nn_device.h"
#include "nn_host.h"

namespace evg {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kOneWaves = 16;
constexpr int kOnePer = 8, kPer = 4;    // entries of a thread in a round
constexpr uint32_t kOneSort = kOneWaves * 64 * kOnePer;   // most entries of a worker that one workgroup places
constexpr uint32_t kFew = kThreads;     // most entries of a worker that every workgroup places for itself
constexpr uint32_t kEmptySlots = 8;     // slots that a wavefront looks through

struct ExpertsArgs {
  evg_mat x, rows, d_rows;     // tokens' rows (x, y, dy) and slots' rows
  const int32_t* chosen;
  const float* weights;
  float* d_weights;
  int32_t *slot, *source, *counts;
  uint32_t workers, tokens, experts, top, width, capacity, slots, first;
  uint32_t run, runs, bits;
  uint32_t* run_counts;        // [workers][runs][experts]
  uint32_t blocks, lines;      // blocks: of 64 vectors across a row; lines: workers * tokens
  uint32_t empty_groups;       // of each worker, where every workgroup makes the plan
  uint32_t token_groups;       // workgroups ahead of those that look for empty slots
};

// ---- the plan ------------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t expert_of(const ExpertsArgs& a, uint32_t w, uint32_t i) {
  const uint32_t e = (uint32_t)a.chosen[(uint64_t)w * a.tokens * a.top + i];
  return e < a.experts ? e : a.experts;
}

__global__ __launch_bounds__(kThreads) void k_experts_count(ExpertsArgs a) {
  __shared__ uint32_t counts[kMostBins];
  const uint32_t block = a.first + blockIdx.x, w = block / a.runs, r = block % a.runs, end = min(a.tokens * a.top, (r + 1) * a.run);
  for (uint32_t i = threadIdx.x; i < a.experts; i += kThreads) counts[i] = 0;
  __syncthreads();
  for (uint32_t begin = r * a.run; begin < end; begin += kThreads * kPer) {
    uint32_t key[kPer], rank[kPer];
    each_key<kPer>(end - begin, [&](int j, uint32_t i, bool real) { key[j] = real ? expert_of(a, w, begin + i) : a.experts; });
    rank_keys<kPer>([&](int j) { return key[j]; }, rank, counts, a.experts, (int)a.bits);
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < a.experts; i += kThreads) a.run_counts[((uint64_t)w * a.runs + r) * a.experts + i] = counts[i];
}

// ALONE: the workgroup has all of a worker's entries, one round of them.
template <bool ALONE, int WAVES, int PER>
__global__ __launch_bounds__(WAVES * 64) void k_experts_place(ExpertsArgs a) {
  constexpr uint32_t THREADS = WAVES * 64;
  __shared__ uint32_t counts[WAVES * kMostBins], first[kMostBins], ahead[kMostBins], part[WAVES];
  const uint32_t block = a.first + blockIdx.x, w = ALONE ? block : block / a.runs, r = ALONE ? 0 : block % a.runs;
  const uint32_t n = a.tokens * a.top, E = a.experts, end = ALONE ? n : min(n, (r + 1) * a.run);
  int32_t* const slot = a.slot + (uint64_t)w * n;
  int32_t* const source = a.source + (uint64_t)w * a.slots;
  uint32_t* const mine = counts + threadIdx.x / 64 * E;
  if constexpr (!ALONE) {
    sum_runs<WAVES>(a.run_counts + (uint64_t)w * a.runs * E, a.runs, r, E, first, ahead);
    if (r == 0)
      for (uint32_t e = threadIdx.x; e < E; e += THREADS) a.counts[(uint64_t)w * E + e] = (int32_t)first[e];
    if (!a.capacity) scan_bins<WAVES>(first, E, part);
  }
  uint32_t begin = ALONE ? 0 : r * a.run;
  do {
    uint32_t key[PER], rank[PER];
    each_key<PER>(end - begin, [&](int j, uint32_t i, bool real) { key[j] = real ? expert_of(a, w, begin + i) : E; });
    for (uint32_t i = threadIdx.x; i < WAVES * E; i += THREADS) counts[i] = 0;
    __syncthreads();
    rank_keys<PER>([&](int j) { return key[j]; }, rank, mine, E, (int)a.bits);
    __syncthreads();
    if constexpr (ALONE) {
      for (uint32_t e = threadIdx.x; e < E; e += THREADS) {
        uint32_t sum = 0;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) sum += counts[v * E + e];
        first[e] = sum;
        ahead[e] = 0;
        a.counts[(uint64_t)w * E + e] = (int32_t)sum;
      }
      __syncthreads();
      if (!a.capacity) scan_bins<WAVES>(first, E, part);
    }
    places_of_waves<WAVES>(counts, ahead, E);   // ranks among the expert's entries
    __syncthreads();
    each_key<PER>(end - begin, [&](int j, uint32_t i, bool real) {
      if (!real) return;
      const uint32_t e = key[j], at_expert = e < E ? mine[e] + rank[j] : 0;
      const bool fits = e < E && (!a.capacity || at_expert < a.capacity);
      const uint32_t at = !fits ? 0 : a.capacity ? e * a.capacity + at_expert : first[e] + at_expert;
      slot[begin + i] = fits ? (int32_t)at : -1;
      if (fits) source[at] = (int32_t)(begin + i);
    });
    begin += THREADS * PER;
    if constexpr (!ALONE) __syncthreads();
  } while (begin < end);
}

// ---- rows ----------------------------------------------------------------------------------------------------------------------

// A slot that the tensors have, whatever the plan holds.
__device__ __forceinline__ bool real_slot(const ExpertsArgs& a, int32_t s) { return (uint32_t)s < a.slots; }

// Zeroes the rows of the slots s0 + lane that are empty.
template <typename T>
__device__ __forceinline__ void zero_rows(const ExpertsArgs& a, const evg_mat& rows, uint32_t w, uint32_t s0, bool empty, int lane) {
  constexpr int E = 16 / sizeof(T);
  const Pack<T, E> zero = {};
  for (uint64_t left = __ballot(empty); left; left &= left - 1) {
    const uint32_t s = s0 + (uint32_t)__ffsll((unsigned long long)left) - 1;
    T* const p = (T*)rows.p + (int64_t)w * rows.worker + (int64_t)s * rows.row;
    for (uint32_t col = lane * E; col < a.width; col += 64 * E) store_pack<E>(p + col, (int)(a.width - col), zero);
  }
}

// Zeroes the rows of the empty ones among a few slots.  PLANNED: the plan's sources tell which they are; else the counts do, and the sources are written.
template <typename T, bool PLANNED>
__device__ __forceinline__ void zero_empty(const ExpertsArgs& a, const evg_mat& rows, uint32_t job, int lane) {
  const uint32_t sets = (a.slots + kEmptySlots - 1) / kEmptySlots, w = job / sets, s0 = job % sets * kEmptySlots;
  if (w >= a.workers) return;
  const uint32_t mine = s0 + lane;
  int32_t* const source = a.source + (uint64_t)w * a.slots;
  bool empty = lane < (int)kEmptySlots && mine < a.slots;
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
  zero_rows<T>(a, rows, w, s0, empty, lane);
}

// A unit is 64 vectors of a token's row; a wavefront has U neighbouring ones.
struct Unit { uint32_t line, block; };

__device__ __forceinline__ void next_unit(const ExpertsArgs& a, Unit& u) {
  if (++u.block == a.blocks) u.block = 0, ++u.line;
}

// rows[slot] = x[t].
template <typename T, int U, bool ONCE>
__global__ __launch_bounds__(kThreads) void k_experts_dispatch(ExpertsArgs a) {
  constexpr int E = 16 / sizeof(T);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t group = a.first + blockIdx.x;
  if (group >= a.token_groups) {
    zero_empty<T, false>(a, a.rows, (group - a.token_groups) * kWaves + wave, lane);
    return;
  }
  const uint32_t first = (group * kWaves + wave) * U;
  const Unit start{first / a.blocks, first % a.blocks};
  Pack<T, E> v[U];
  Unit at = start;
#pragma unroll
  for (int u = 0; u < U; ++u, next_unit(a, at)) {
    const uint32_t w = at.line / a.tokens, t = at.line % a.tokens, col = (at.block * 64 + lane) * E;
    if (at.line < a.lines) v[u] = load_pack<E>((const T*)a.x.p + (int64_t)w * a.x.worker + (int64_t)t * a.x.row + col, (int)a.width - (int)col);
  }
  // A slot's units one after the other: whole rows where a wavefront has them.
  for (uint32_t k = 0; k < a.top; ++k) {
    at = start;
#pragma unroll
    for (int u = 0; u < U; ++u, next_unit(a, at)) {
      if (at.line >= a.lines) break;
      const uint32_t w = at.line / a.tokens, col = (at.block * 64 + lane) * E;
      const int32_t s = a.slot[(uint64_t)at.line * a.top + k];
      T* const out = (T*)a.rows.p + (int64_t)w * a.rows.worker + col;
      if (real_slot(a, s)) store_pack<E, ONCE>(out + (int64_t)s * a.rows.row, (int)a.width - (int)col, v[u]);
    }
  }
}

// Few entries: each workgroup makes the plan for itself and sends its units, in one launch (one token to 8 experts of 64, 2048 wide: 6.7 us instead
// of 3.4 and 3.9, and a launch of the host's less: with combine 25.4 instead of 28.9).
// A worker has token_groups workgroups for its tokens and empty_groups behind them.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_experts_dispatch_few(ExpertsArgs a) {
  constexpr int E = 16 / sizeof(T);
  __shared__ uint32_t counts[kMostBins], first[kMostBins], part[kWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t block = a.first + blockIdx.x, per = a.token_groups + a.empty_groups, w = block / per, group = block % per, n = a.tokens * a.top;
  int32_t* const source = a.source + (uint64_t)w * a.slots;
  for (uint32_t e = threadIdx.x; e < a.experts; e += kThreads) counts[e] = 0;
  __syncthreads();
  const uint32_t key = threadIdx.x < n ? expert_of(a, w, threadIdx.x) : a.experts;
  if (key < a.experts) atomicAdd(&counts[key], 1u);
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < a.experts; e += kThreads) {
    first[e] = counts[e];
    if (group == 0) a.counts[(uint64_t)w * a.experts + e] = (int32_t)counts[e];
  }
  __syncthreads();
  const uint32_t total = a.capacity ? 0 : scan_bins<kWaves>(first, a.experts, part);
  if (group >= a.token_groups) {
    const uint32_t s0 = ((group - a.token_groups) * kWaves + wave) * kEmptySlots, mine = s0 + lane;
    const bool empty = lane < (int)kEmptySlots && mine < a.slots && (a.capacity ? mine % a.capacity >= counts[mine / a.capacity] : mine >= total);
    if (empty) source[mine] = -1;
    zero_rows<T>(a, a.rows, w, s0, empty, lane);
    return;
  }
  const uint32_t unit = group * kWaves + wave, t = unit / a.blocks, col = (unit % a.blocks * 64 + lane) * E;
  if (t >= a.tokens) return;
  uint32_t keys[kFew / 64];
#pragma unroll
  for (uint32_t c = 0; c < kFew / 64; ++c) keys[c] = c * 64 + lane < n ? expert_of(a, w, c * 64 + lane) : a.experts;
  const Pack<T, E> v = load_pack<E>((const T*)a.x.p + (int64_t)w * a.x.worker + (int64_t)t * a.x.row + col, (int)a.width - (int)col);
  T* const out = (T*)a.rows.p + (int64_t)w * a.rows.worker + col;
  for (uint32_t k = 0; k < a.top; ++k) {
    const uint32_t i = t * a.top + k, e = expert_of(a, w, i);
    uint32_t rank = 0;
#pragma unroll
    for (uint32_t c = 0; c < kFew / 64; ++c) rank += (uint32_t)__popcll(__ballot(keys[c] == e && c * 64 + lane < i));
    const bool fits = e < a.experts && (!a.capacity || rank < a.capacity);
    const uint32_t at = !fits ? 0 : a.capacity ? e * a.capacity + rank : first[e] + rank;
    if (unit % a.blocks == 0 && lane == 0) {
      a.slot[(uint64_t)w * n + i] = fits ? (int32_t)at : -1;
      if (fits) source[at] = (int32_t)i;
    }
    if (fits) store_pack<E>(out + (int64_t)at * a.rows.row, (int)a.width - (int)col, v);
  }
}

// y[t] = sum over k of weights[i] rows[slot[i]], KS rows under way at once.
template <typename T, uint32_t KS, bool ONCE>
__global__ __launch_bounds__(kThreads) void k_experts_combine(ExpertsArgs a) {
  constexpr int E = 16 / sizeof(T);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t job = (a.first + blockIdx.x) * kWaves + wave, line = job / a.blocks;
  if (line >= a.lines) return;
  const uint32_t w = line / a.tokens, t = line % a.tokens, col = (job % a.blocks * 64 + lane) * E;
  const int n = (int)a.width - (int)col;
  const T* const p = (const T*)a.rows.p + (int64_t)w * a.rows.worker + col;
  const int32_t* const slot = a.slot + (uint64_t)line * a.top;
  const float* const weights = a.weights + (uint64_t)line * a.top;
  float acc[E] = {};
  for (uint32_t k = 0; k < a.top; k += KS) {
    Pack<T, E> v[KS];
    float f[KS];
#pragma unroll
    for (uint32_t j = 0; j < KS; ++j) {
      const int32_t s = k + j < a.top ? slot[k + j] : -1;
      const bool real = real_slot(a, s);
      f[j] = real ? (a.weights ? weights[k + j] : 1.f) : 0.f;
      v[j] = load_pack<E, ONCE>(p + (real ? (int64_t)s * a.rows.row : 0), real ? n : 0);
    }
#pragma unroll
    for (uint32_t j = 0; j < KS; ++j)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(f[j], to_f(v[j].v[e]), acc[e]);
  }
  store_upto<E>((T*)a.x.p + (int64_t)w * a.x.worker + (int64_t)t * a.x.row + col, n, acc);
}

// d_rows[slot] = weights[i] dy[t], d_weights[i] = <dy[t], rows[slot]>.  A wavefront has a token, BLOCKS units of its row at a time: those of dy stay, the
// experts' go by, the next one's asked for ahead.
template <typename T, int BLOCKS, bool ONCE>
__global__ __launch_bounds__(kThreads) void k_experts_combine_backward(ExpertsArgs a) {
  constexpr int E = 16 / sizeof(T);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t group = a.first + blockIdx.x;
  if (group >= a.token_groups) {
    zero_empty<T, true>(a, a.d_rows, (group - a.token_groups) * kWaves + wave, lane);
    return;
  }
  const uint32_t line = group * kWaves + wave;
  if (line >= a.lines) return;
  const uint32_t w = line / a.tokens, t = line % a.tokens;
  const T* const dy = (const T*)a.x.p + (int64_t)w * a.x.worker + (int64_t)t * a.x.row;
  const T* const rows = (const T*)a.rows.p + (int64_t)w * a.rows.worker;
  T* const d_rows = (T*)a.d_rows.p + (int64_t)w * a.d_rows.worker;
  const int32_t* const slot = a.slot + (uint64_t)line * a.top;
  const float* const weights = a.weights + (uint64_t)line * a.top;
  for (uint32_t first = 0; first < a.width; first += BLOCKS * 64 * E) {
    Pack<T, E> g[BLOCKS], v[2][BLOCKS];
    int n[BLOCKS];
    uint32_t col[BLOCKS];
#pragma unroll
    for (int u = 0; u < BLOCKS; ++u) {
      col[u] = first + (u * 64 + lane) * E;
      n[u] = (int)a.width - (int)col[u];
      g[u] = load_pack<E>(dy + col[u], n[u]);
    }
    auto ask = [&](uint32_t k, int to) {
      const int32_t s = k < a.top ? slot[k] : -1;
      if (!a.d_weights || !real_slot(a, s)) return;
#pragma unroll
      for (int u = 0; u < BLOCKS; ++u) v[to][u] = load_pack<E, ONCE>(rows + (int64_t)s * a.rows.row + col[u], n[u]);
    };
    ask(0, 0);
    for (uint32_t k0 = 0; k0 < a.top; k0 += 2) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t k = k0 + half;
        if (k >= a.top) break;
        ask(k + 1, half ^ 1);
        const int32_t s = slot[k];
        const bool real = real_slot(a, s);
        if (real && a.d_rows.p) {
          const float f = weights[k];
#pragma unroll
          for (int u = 0; u < BLOCKS; ++u) {
            Pack<T, E> d;
#pragma unroll
            for (int e = 0; e < E; ++e) d.v[e] = from_f<T>(f * to_f(g[u].v[e]));
            store_pack<E, ONCE>(d_rows + (int64_t)s * a.d_rows.row + col[u], n[u], d);
          }
        }
        if (a.d_weights) {
          float sum = 0.f;
          if (real) {
#pragma unroll
            for (int u = 0; u < BLOCKS; ++u)
#pragma unroll
              for (int e = 0; e < E; ++e) sum = fmaf(to_f(g[u].v[e]), to_f(v[half][u].v[e]), sum);
            sum = wave_sum_uniform(sum);
          }
          float* const out = a.d_weights + (uint64_t)line * a.top + k;
          if (lane == 0) *out = first ? *out + sum : sum;
        }
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
  a.workers = g.workers, a.lines = g.workers * tokens, a.tokens = tokens, a.experts = g.experts, a.top = g.top, a.width = g.width, a.capacity = g.capacity;
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

// Do the slots' rows go past the caches, as they do not fit them?
template <typename T>
bool past_caches(const ExpertsArgs& a) { return (uint64_t)a.workers * a.slots * a.width * sizeof(T) > (128u << 20); }

template <typename T>
hipError_t dispatch(const evg_experts* c, ExpertsArgs& a) {
  const uint32_t n = a.tokens * a.top;
  hipError_t e;
  if (n <= kFew) {
    a.token_groups = (a.tokens * a.blocks + kWaves - 1) / kWaves;
    a.empty_groups = (a.slots + kEmptySlots * kWaves - 1) / (kEmptySlots * kWaves);
    if (!(a.token_groups + a.empty_groups)) a.empty_groups = 1;   // the counts are written all the same
    return launch((uint64_t)a.workers * (a.token_groups + a.empty_groups), kThreads, c->stream, a, k_experts_dispatch_few<T>);
  }
  while ((1u << a.bits) < a.experts) ++a.bits;
  if (n <= kOneSort) {
    if ((e = launch(a.workers, kOneWaves * 64, c->stream, a, n <= kOneWaves * 64 ? k_experts_place<true, kOneWaves, 1> : k_experts_place<true, kOneWaves, kOnePer>)) != hipSuccess) return e;
  } else {
    const Runs runs = cut_runs(n, kThreads * kPer);
    a.run = runs.each, a.runs = runs.count;
    const uint64_t groups = (uint64_t)a.workers * a.runs;
    if ((e = launch(groups, kThreads, c->stream, a, k_experts_count)) != hipSuccess) return e;
    if ((e = launch(groups, kThreads, c->stream, a, k_experts_place<false, kWaves, kPer>)) != hipSuccess) return e;
  }
  // Few units go to a wavefront each: the chip has room for 8192 of them.
  const uint32_t units = a.lines * a.blocks, each = units <= 8192 ? 1 : 4;
  a.token_groups = (units + each * kWaves - 1) / (each * kWaves);
  const uint64_t groups = a.token_groups + empty_groups(a);
  if (each == 1) return launch(groups, kThreads, c->stream, a, k_experts_dispatch<T, 1, false>);
  return launch(groups, kThreads, c->stream, a, past_caches<T>(a) ? k_experts_dispatch<T, 4, true> : k_experts_dispatch<T, 4, false>);
}

template <typename T, bool ONCE>
hipError_t combine_by(const evg_experts* c, ExpertsArgs& a) {
  const uint64_t groups = ((uint64_t)a.lines * a.blocks + kWaves - 1) / kWaves;
  return launch(groups, kThreads, c->stream, a,
                a.top <= 2 ? k_experts_combine<T, 2, ONCE> : a.top <= 4 ? k_experts_combine<T, 4, ONCE> : k_experts_combine<T, 8, ONCE>);
}

template <typename T>
hipError_t combine(const evg_experts* c, ExpertsArgs& a) {
  return past_caches<T>(a) ? combine_by<T, true>(c, a) : combine_by<T, false>(c, a);
}

template <typename T, bool ONCE>
hipError_t combine_backward_by(const evg_experts* c, ExpertsArgs& a) {
  a.token_groups = (a.lines + kWaves - 1) / kWaves;
  const uint64_t groups = a.token_groups + (a.d_rows.p ? empty_groups(a) : 0);
  return launch(groups, kThreads, c->stream, a, a.blocks <= 1 ? k_experts_combine_backward<T, 1, ONCE> : a.blocks <= 2 ? k_experts_combine_backward<T, 2, ONCE> : k_experts_combine_backward<T, 4, ONCE>);
}

template <typename T>
hipError_t combine_backward(const evg_experts* c, ExpertsArgs& a) {
  return past_caches<T>(a) ? combine_backward_by<T, true>(c, a) : combine_backward_by<T, false>(c, a);
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
  const uint64_t blocks = ((uint64_t)cfg->width * type_bytes(cfg->type) + 1023) / 1024;
  // Kernels count units of 64 vectors, and slots, in 32 bits.
  if (cfg->workers * (uint64_t)cfg->max_tokens * blocks > 0x7FFFFFFFull || cfg->workers * (slots + kEmptySlots) > 0x7FFFFFFFull)
    return fail(EVG_ERR_INVALID, "workers, max_tokens, width and capacity together are out of range");
  evg_status st;
  if ((st = check_type(cfg->type, "type")) != EVG_OK) return st;
  evg_experts* c = new (std::nothrow) evg_experts();
  if (!c) return fail(EVG_ERR_OOM, "host allocation failed");
  c->cfg = *cfg;
  c->stream = static_cast<hipStream_t>(hip_stream);
  if ((uint64_t)cfg->max_tokens * cfg->top > kOneSort) {
    const hipError_t e = hipMalloc((void**)&c->run_counts, (uint64_t)cfg->workers * kMostRuns * cfg->experts * 4);
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
