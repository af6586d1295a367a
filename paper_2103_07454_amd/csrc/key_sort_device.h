// Stable counting sort of small whole numbers, as tokens and experts have.
//
// A workgroup takes a run of keys; each of its wavefronts a contiguous part of the run.  The wavefronts count their keys, a scan over the bins
// gives each wavefront the place of its first key of each bin, and 64 keys at a time find their places from there: the lanes
// with the same key are found by one ballot for each bit, the first of them moves the bin's place on.  No result depends on the
// order in which wavefronts run.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace evg {

constexpr uint32_t kMostBins = 1024;

// Keys of a wavefront's part of n: whole groups of 64.
template <int WAVES>
__device__ __forceinline__ uint32_t part_keys(uint32_t n) { return (n + WAVES * 64 - 1) / (WAVES * 64) * 64; }

// Adds the keys of this wavefront's part to counts[bin]; keys of `bins` and above do not count.  key(i): that of the run's i-th.
template <int WAVES, typename Key>
__device__ __forceinline__ void count_keys(uint32_t* counts, uint32_t bins, uint32_t n, Key key) {
  const uint32_t part = part_keys<WAVES>(n), begin = threadIdx.x / 64 * part, end = min(n, begin + part);
  for (uint32_t i = begin + threadIdx.x % 64; i < end; i += 64) {
    const uint32_t k = key(i);
    if (k < bins) atomicAdd(&counts[k], 1u);
  }
}

// The places of this wavefront's keys: next[bin] is that of its first, and is moved on.  emit(i, key, place) for each key below `bins` < 2^bits.
template <int WAVES, typename Key, typename Emit>
__device__ __forceinline__ void place_keys(uint32_t* next, uint32_t bins, int bits, uint32_t n, Key key, Emit emit) {
  const uint32_t part = part_keys<WAVES>(n), begin = threadIdx.x / 64 * part, end = min(n, begin + part);
  const int lane = threadIdx.x % 64;
  for (uint32_t base = begin; base < end; base += 64) {
    const uint32_t i = base + lane, k = i < end ? key(i) : bins;
    uint64_t same = __ballot(k < bins);
    for (int b = 0; b < bits; ++b) {
      const uint64_t set = __ballot(k >> b & 1);
      same &= k >> b & 1 ? set : ~set;
    }
    uint32_t at = 0;
    const int leader = same ? __ffsll((unsigned long long)same) - 1 : lane;
    if (k < bins && lane == leader) at = atomicAdd(&next[k], (uint32_t)__popcll(same));
    at = __shfl(at, leader, 64) + (uint32_t)__popcll(same & ((1ull << lane) - 1));
    if (k < bins) emit(i, k, at);
  }
}

// The sum of the values of the threads ahead of this one.  `part`: a word for each wavefront.  All threads of the workgroup take part.
template <int WAVES>
__device__ __forceinline__ uint32_t sum_ahead(uint32_t v, uint32_t* part, uint32_t* total) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint32_t sum = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(sum, d, 64);
    if (lane >= d) sum += o;
  }
  if (lane == 63) part[wave] = sum;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    before += w < wave ? part[w] : 0;
    all += part[w];
  }
  __syncthreads();
  *total = all;
  return before + sum - v;
}

// counts[wave][bin] of a workgroup, on top of first[bin]: the place of each wavefront's first key of each bin.
template <int WAVES>
__device__ __forceinline__ void places_of_waves(uint32_t* counts, const uint32_t* first, uint32_t bins) {
  for (uint32_t b = threadIdx.x; b < bins; b += WAVES * 64) {
    uint32_t at = first[b];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const uint32_t c = counts[w * bins + b];
      counts[w * bins + b] = at;
      at += c;
    }
  }
}

// Exclusive prefix sums of values[bin] in LDS, in place; returns their total.
template <int WAVES>
__device__ __forceinline__ uint32_t scan_bins(uint32_t* values, uint32_t bins, uint32_t* part) {
  constexpr uint32_t EACH = (kMostBins + WAVES * 64 - 1) / (WAVES * 64);
  uint32_t v[EACH], sum = 0, total;
#pragma unroll
  for (uint32_t i = 0; i < EACH; ++i) {
    const uint32_t b = threadIdx.x * EACH + i;
    v[i] = b < bins ? values[b] : 0;
    sum += v[i];
  }
  uint32_t at = sum_ahead<WAVES>(sum, part, &total);
#pragma unroll
  for (uint32_t i = 0; i < EACH; ++i) {
    const uint32_t b = threadIdx.x * EACH + i;
    if (b < bins) values[b] = at;
    at += v[i];
  }
  __syncthreads();
  return total;
}

// How a worker's n keys are cut into runs of a workgroup each: few enough that every workgroup can add up what the runs ahead of its own counted.
struct Runs { uint32_t each, count; };
inline Runs cut_runs(uint32_t n) {
  const uint64_t least = 2048, by = ((uint64_t)n + 127) / 128;
  const uint32_t each = (uint32_t)(by <= least ? least : (by + 1023) / 1024 * 1024);
  return {each, n ? (n + each - 1) / each : 0};
}

}  // namespace evg
