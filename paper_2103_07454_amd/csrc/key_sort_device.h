// Stable counting sort of small whole numbers, as tokens and experts have.
//
// A workgroup takes a run of keys, WAVES * 64 * PER at a time in registers; each of its wavefronts has a contiguous part, all of whose loads are under way at once.
// The wavefronts rank and count their keys, 64 at a time: the lanes with the same key are found by one ballot for each bit, the first of them moves the bin's count
// on.  A scan over the bins then gives each wavefront the place of its first key of each bin.
// No result depends on the order in which wavefronts run.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace evg {

constexpr uint32_t kMostBins = 1024;

// Calls f(j, i) for this thread's keys of a run of n: the i-th of the run is its j-th.
template <int PER, typename F>
__device__ __forceinline__ void each_key(uint32_t n, F f) {
  const uint32_t begin = threadIdx.x / 64 * (64 * PER) + threadIdx.x % 64;
#pragma unroll
  for (int j = 0; j < PER; ++j) f(j, begin + j * 64, begin + j * 64 < n);
}

// Counts this wavefront's keys, key(j), in counts[bin]; what was there before each key is its rank.  Keys of `bins` <= 2^bits and above do not count.  (Counting by an
// LDS operation of each lane costs one of a lane after the other where many keys are the same: 60 us for 16384 tokens of which half had the same upper byte.)
template <int PER, typename Key>
__device__ __forceinline__ void rank_keys(Key key, uint32_t* rank, uint32_t* counts, uint32_t bins, int bits) {
  const int lane = threadIdx.x % 64;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const uint32_t k = key(j);
    uint64_t same = __ballot(k < bins);
    rank[j] = 0;
    if (!same) continue;
    for (int b = 0; b < bits; ++b) {
      const uint64_t set = __ballot(k >> b & 1);
      same &= k >> b & 1 ? set : ~set;
    }
    uint32_t at = 0;
    const int leader = same ? __ffsll((unsigned long long)same) - 1 : lane;
    if (k < bins && lane == leader) at = atomicAdd(&counts[k], (uint32_t)__popcll(same));
    rank[j] = __shfl(at, leader, 64) + (uint32_t)__popcll(same & ((1ull << lane) - 1));
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

// counts[wave][bin] of a workgroup, on top of first[bin]: the place of each wavefront's first key of each bin; first[bin] goes on behind the last one's.
template <int WAVES>
__device__ __forceinline__ void places_of_waves(uint32_t* counts, uint32_t* first, uint32_t bins) {
  for (uint32_t b = threadIdx.x; b < bins; b += WAVES * 64) {
    uint32_t at = first[b];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const uint32_t c = counts[w * bins + b];
      counts[w * bins + b] = at;
      at += c;
    }
    first[b] = at;
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

// What all runs counted, all[run][bin], added up: total[bin] over all of them, ahead[bin] over those ahead of run r.  Both in LDS.  Threads beyond the bins
// take runs of their own.
template <int WAVES>
__device__ __forceinline__ void sum_runs(const uint32_t* all, uint32_t runs, uint32_t r, uint32_t bins, uint32_t* total, uint32_t* ahead) {
  constexpr uint32_t THREADS = WAVES * 64;
  for (uint32_t b = threadIdx.x; b < bins; b += THREADS) total[b] = ahead[b] = 0;
  __syncthreads();
  const uint32_t shares = bins >= THREADS ? 1 : THREADS / bins, share = bins >= THREADS ? 0 : threadIdx.x / bins;
  if (share < shares) {
    for (uint32_t b = bins >= THREADS ? threadIdx.x : threadIdx.x % bins; b < bins; b += THREADS) {
      uint32_t sum = 0, before = 0;
#pragma unroll 8
      for (uint32_t q = share; q < runs; q += shares) {
        const uint32_t c = all[(uint64_t)q * bins + b];
        sum += c;
        before += q < r ? c : 0;
      }
      if (sum) atomicAdd(&total[b], sum);
      if (before) atomicAdd(&ahead[b], before);
    }
  }
  __syncthreads();
}

// How a worker's n keys are cut into runs of a workgroup each, whole rounds of `round` keys: few enough that every workgroup can add up what the runs counted.
struct Runs { uint32_t each, count; };
constexpr uint32_t kMostRuns = 128;
inline Runs cut_runs(uint32_t n, uint32_t round) {
  const uint32_t rounds = (uint32_t)(((uint64_t)n + round - 1) / round), each = (rounds + kMostRuns - 1) / kMostRuns * round;
  return {each, n ? (uint32_t)(((uint64_t)n + each - 1) / each) : 0};
}

}  // namespace evg
