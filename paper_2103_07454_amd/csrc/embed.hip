// Embeddings and their gradient by sorted tokens (include/evg_nn.h, evg_embed_*).
//
//     y[t] = s table[id[t]],    d_table[v] = s sum over t with id[t] = v of dy[t]
//
// Forward: a wavefront takes 64 vectors of 16 bytes of one token's row.  Bound by memory, rows of the table in any order.
//
// Backward: the tokens are sorted by their number, those of one number stay in their order; then a wavefront adds up the rows of a
// chunk of 16 sorted tokens, 64 vectors wide, and writes a sum where the number changes.  Numbers that go on in the next chunk leave partial sums in 32 bits,
// which a launch behind adds in the chunks' order, a wavefront all those of a number and 256 columns: no atomics, so the same tokens give the same bits.  A number that
// very many tokens have is waited for there: of 16384 tokens 2048 wide a gradient takes 87 us with up to a sixteenth of them the same, 106 with a quarter, 129 with half, 174 with all.
// The rows that no token names are zeroed by the launch of the sums; a mark for each number says which.
// Bound by memory: dy once, the gradient's table once.
//
// 16384 tokens, 50257 x 2048 in bfloat16, half of the tokens of 224 numbers: rows 20 us (87 MB, 4.4 TB/s), sorting 2 x (5 + 11), sums and zeros 45 (273 MB, 6.1 TB/s; 82
// with zeros through the caches and rows not asked for ahead), join 9 (22 with a load at a time).
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "key_sort_device.h"
#include "nn_device.h"
#include "nn_host.h"

namespace evg {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kChunk = 16;          // sorted tokens that a wavefront adds up (16384 tokens 2048 wide: 8 / 16 / 32 take 63 / 54 / 67 us with the joining)
constexpr uint32_t kFewTokens = 512;     // most tokens of a worker that are sorted by comparing each with all (eight times 333: 7.0 us instead of 8.8)
constexpr int kOneWaves = 16;            // of the workgroup that sorts alone
constexpr int kPer = 4;                  // keys of a thread in a round
// Most tokens of a worker that one workgroup sorts.  Ranking keeps a CU's vector units busy: 16384 tokens took one workgroup 57 us, sixteen 24.
constexpr uint32_t kOneSort = kOneWaves * 64 * kPer;
constexpr uint32_t kZeroRows = 4;        // rows that a wavefront may have to zero: a word of marks

struct EmbedArgs {
  const void* ids;
  int64_t ids_worker;
  uint32_t wide;
  evg_mat table, rows;         // rows: y or dy
  uint32_t workers, tokens, vocab, width, blocks, lines;   // blocks: of 64 vectors across a row; lines: workers * tokens
  float scale;
  uint32_t accumulate;
  uint32_t first;              // workgroup of a launch in pieces
  // workspace
  uint32_t *key[2], *pos[2];   // [workers][tokens]
  uint32_t *counts;            // [workers][runs][bins]
  uint32_t *real;              // [workers]: sorted tokens
  uint8_t *seen;               // [workers][vocab, up to a multiple of 4]: is a number some token's?
  float *partial;              // [workers][chunks][2][width]
  uint32_t run, runs, bins, bits, shift, last;   // of a sorting pass
  uint32_t chunks, sum_groups;
};

constexpr uint32_t kNoToken = 0xFFFFFFFFu;

__device__ __forceinline__ uint32_t token_id(const EmbedArgs& a, uint32_t w, uint32_t t) {
  const int64_t at = (int64_t)w * a.ids_worker + t;
  const int64_t id = a.wide ? ((const int64_t*)a.ids)[at] : (int64_t)((const int32_t*)a.ids)[at];
  return id >= 0 && id < (int64_t)a.vocab ? (uint32_t)id : kNoToken;
}

// U neighbouring units of 64 vectors to a wavefront, all their loads under way at once.
template <typename T, int U>
__global__ __launch_bounds__(kThreads) void k_embed_rows(EmbedArgs a) {
  constexpr int E = 16 / sizeof(T);
  const uint32_t unit = ((a.first + blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * U;
  uint32_t line = unit / a.blocks, block = unit % a.blocks;
  float v[U][E] = {};
  T* out[U];
  int n[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t w = line / a.tokens, t = line % a.tokens, col = block * 64 * E + (threadIdx.x & 63) * E;
    n[u] = line < a.lines ? (int)a.width - (int)col : 0;
    const uint32_t id = line < a.lines ? token_id(a, w, t) : kNoToken;
    if (id != kNoToken) load_upto<E>((const T*)a.table.p + (int64_t)w * a.table.worker + (int64_t)id * a.table.row + col, n[u], v[u]);
    out[u] = (T*)a.rows.p + (int64_t)w * a.rows.worker + (int64_t)t * a.rows.row + col;
    if (++block == a.blocks) block = 0, ++line;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int i = 0; i < E; ++i) v[u][i] *= a.scale;
    store_upto<E>(out[u], n[u], v[u]);
  }
}

// ---- sorting -----------------------------------------------------------------------------------------------------------------

// Bytes, not bits: what thousands of tokens set takes no atomic operations, which would meet at a few addresses (100 us of 16384 tokens).
__device__ __forceinline__ uint32_t seen_words(uint32_t vocab) { return (vocab + 3) / 4; }
__device__ __forceinline__ uint8_t* seen_of(const EmbedArgs& a, uint32_t w) { return a.seen + (uint64_t)w * seen_words(a.vocab) * 4; }

// Few tokens: each thread compares its token with all others.  A number and its place are one word, so that a comparison tells both.
__global__ __launch_bounds__(kFewTokens) void k_embed_sort_few(EmbedArgs a, int place_bits) {
  __shared__ __attribute__((aligned(16))) uint32_t words[kFewTokens];
  __shared__ uint32_t part[kFewTokens / 64];
  const uint32_t w = a.first + blockIdx.x, i = threadIdx.x;
  uint8_t* const seen = seen_of(a, w);
  const uint32_t key = i < a.tokens ? token_id(a, w, i) : kNoToken, word = key == kNoToken ? kNoToken : key << place_bits | i;
  words[i] = word;   // of 31 bits where there is a token
  for (uint32_t v = i; v < seen_words(a.vocab); v += kFewTokens) ((uint32_t*)seen)[v] = 0;
  __syncthreads();   // marks come behind
  uint32_t rank = 0;
  for (uint32_t j = 0; j < a.tokens; j += 32) {
    uint4 q[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) q[u] = *reinterpret_cast<const uint4*>(words + j + u * 4);
#pragma unroll
    for (int u = 0; u < 8; ++u) rank += (q[u].x < word) + (q[u].y < word) + (q[u].z < word) + (q[u].w < word);
  }
  uint32_t real;
  (void)sum_ahead<kFewTokens / 64>(key != kNoToken, part, &real);
  if (key != kNoToken) {
    a.key[0][(uint64_t)w * a.tokens + rank] = key;
    a.pos[0][(uint64_t)w * a.tokens + rank] = i;
    seen[key] = 1;
  }
  if (i == 0) a.real[w] = real;
}

// A worker's tokens by one workgroup, digits of 8 bits from the lowest up: keys and places stay in registers and change threads through LDS.
template <int PER>
__global__ __launch_bounds__(kOneWaves * 64) void k_embed_sort_alone(EmbedArgs a, int bits) {
  constexpr uint32_t BINS = 256, THREADS = kOneWaves * 64;
  __shared__ uint32_t keys[THREADS * PER];
  __shared__ uint16_t poss[THREADS * PER];
  __shared__ uint32_t counts[kOneWaves * BINS], first[BINS], part[kOneWaves];
  const uint32_t w = a.first + blockIdx.x;
  uint8_t* const seen = seen_of(a, w);
  uint32_t key[PER], pos[PER], rank[PER], n = a.tokens;
  each_key<PER>(n, [&](int j, uint32_t i, bool real) {
    key[j] = real ? token_id(a, w, i) : kNoToken;
    pos[j] = i;
  });
  for (uint32_t i = threadIdx.x; i < seen_words(a.vocab); i += THREADS) ((uint32_t*)seen)[i] = 0;   // marks come behind barriers
  for (int shift = 0; shift == 0 || shift < bits; shift += 8) {
    for (uint32_t i = threadIdx.x; i < kOneWaves * BINS; i += THREADS) counts[i] = 0;
    // Tokens outside the table are left out by the first pass.
    auto digit = [&](int j) { return key[j] == kNoToken ? BINS : key[j] >> shift & (BINS - 1); };
    __syncthreads();
    uint32_t* const own = counts + threadIdx.x / 64 * BINS;
    rank_keys<PER>(digit, rank, own, BINS, 8);
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < BINS; b += THREADS) {
      uint32_t sum = 0;
#pragma unroll
      for (int v = 0; v < kOneWaves; ++v) sum += counts[v * BINS + b];
      first[b] = sum;
    }
    __syncthreads();
    n = scan_bins<kOneWaves>(first, BINS, part);
    places_of_waves<kOneWaves>(counts, first, BINS);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (key[j] != kNoToken) {
        const uint32_t at = own[digit(j)] + rank[j];
        keys[at] = key[j];
        poss[at] = (uint16_t)pos[j];
      }
    __syncthreads();
    each_key<PER>(n, [&](int j, uint32_t i, bool real) {
      key[j] = real ? keys[i] : kNoToken;
      pos[j] = real ? poss[i] : 0;
    });
  }
  each_key<PER>(n, [&](int j, uint32_t i, bool real) {
    if (!real) return;
    a.key[0][(uint64_t)w * a.tokens + i] = key[j];
    a.pos[0][(uint64_t)w * a.tokens + i] = pos[j];
    seen[key[j]] = 1;
  });
  if (threadIdx.x == 0) a.real[w] = n;
}

// Many tokens: a pass over one digit is two launches, counting and placing.  The first pass reads the tokens themselves.
__device__ __forceinline__ void load_keys(const EmbedArgs& a, const uint32_t* keys, uint32_t w, uint32_t begin, uint32_t n, uint32_t* key) {
  each_key<kPer>(n, [&](int j, uint32_t i, bool real) { key[j] = !real ? kNoToken : keys ? keys[begin + i] : token_id(a, w, begin + i); });
}

__device__ __forceinline__ uint32_t sort_digit(const EmbedArgs& a, uint32_t k) { return k == kNoToken ? a.bins : k >> a.shift & (a.bins - 1); }

__global__ __launch_bounds__(kThreads) void k_embed_count(EmbedArgs a, const uint32_t* keys) {
  __shared__ uint32_t counts[kMostBins];
  const uint32_t block = a.first + blockIdx.x, w = block / a.runs, r = block % a.runs;
  const uint32_t n = keys ? a.real[w] : a.tokens, end = min(n, (r + 1) * a.run);
  for (uint32_t i = threadIdx.x; i < a.bins; i += kThreads) counts[i] = 0;
  if (!keys) {   // numbers are marked by the last pass
    uint8_t* const seen = seen_of(a, w);
    for (uint32_t i = r * kThreads + threadIdx.x; i < seen_words(a.vocab); i += a.runs * kThreads) ((uint32_t*)seen)[i] = 0;
  }
  __syncthreads();
  const uint32_t* const own = keys ? keys + (uint64_t)w * a.tokens : nullptr;
  for (uint32_t begin = r * a.run; begin < end; begin += kThreads * kPer) {
    uint32_t key[kPer], rank[kPer];
    load_keys(a, own, w, begin, end - begin, key);
    rank_keys<kPer>([&](int j) { return sort_digit(a, key[j]); }, rank, counts, a.bins, (int)a.bits);
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < a.bins; i += kThreads) a.counts[((uint64_t)w * a.runs + r) * a.bins + i] = counts[i];
}

__global__ __launch_bounds__(kThreads) void k_embed_place(EmbedArgs a, const uint32_t* keys, const uint32_t* poss, uint32_t* key_out, uint32_t* pos_out) {
  __shared__ uint32_t counts[kWaves * kMostBins], first[kMostBins], ahead[kMostBins], part[kWaves];
  const uint32_t block = a.first + blockIdx.x, w = block / a.runs, r = block % a.runs;
  const uint32_t n = keys ? a.real[w] : a.tokens, end = min(n, (r + 1) * a.run);
  sum_runs<kWaves>(a.counts + (uint64_t)w * a.runs * a.bins, a.runs, r, a.bins, first, ahead);
  const uint32_t left = scan_bins<kWaves>(first, a.bins, part);
  for (uint32_t b = threadIdx.x; b < a.bins; b += kThreads) first[b] += ahead[b];
  const uint32_t* const own = keys ? keys + (uint64_t)w * a.tokens : nullptr;
  uint8_t* const seen = seen_of(a, w);
  uint32_t* const mine = counts + threadIdx.x / 64 * a.bins;
  for (uint32_t begin = r * a.run; begin < end; begin += kThreads * kPer) {
    uint32_t key[kPer], rank[kPer], pos[kPer];
    load_keys(a, own, w, begin, end - begin, key);
    auto digit = [&](int j) { return sort_digit(a, key[j]); };
    each_key<kPer>(end - begin, [&](int j, uint32_t i, bool real) { pos[j] = !real ? 0 : own ? poss[(uint64_t)w * a.tokens + begin + i] : begin + i; });
    for (uint32_t i = threadIdx.x; i < kWaves * a.bins; i += kThreads) counts[i] = 0;
    __syncthreads();
    rank_keys<kPer>(digit, rank, mine, a.bins, (int)a.bits);
    __syncthreads();
    places_of_waves<kWaves>(counts, first, a.bins);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (key[j] != kNoToken) {
        const uint64_t at = (uint64_t)w * a.tokens + mine[digit(j)] + rank[j];
        key_out[at] = key[j];
        pos_out[at] = pos[j];
        if (a.last) seen[key[j]] = 1;
      }
    __syncthreads();
  }
  // All passes place the same tokens, so that what the first finds holds for the others.
  if (!keys && r == 0 && threadIdx.x == 0) a.real[w] = left;
}

// ---- sums --------------------------------------------------------------------------------------------------------------------

template <int E, typename T>
__device__ __forceinline__ void leave_sum(const EmbedArgs& a, uint32_t w, uint32_t id, uint32_t col, int n, float* v) {
  T* const p = (T*)a.table.p + (int64_t)w * a.table.worker + (int64_t)id * a.table.row + col;
  float old[E] = {};
  if (a.accumulate) load_upto<E>(p, n, old);
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = a.accumulate ? fmaf(v[i], a.scale, old[i]) : v[i] * a.scale;
  store_upto<E>(p, n, v);
}

template <typename T, bool ONCE>
__global__ __launch_bounds__(kThreads) void k_embed_sum(EmbedArgs a) {
  constexpr int E = 16 / sizeof(T);
  constexpr uint32_t AHEAD = 8;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t group = a.first + blockIdx.x;
  if (group >= a.sum_groups) {   // rows that no token names
    const uint32_t sets = (a.vocab + kZeroRows - 1) / kZeroRows, job = (group - a.sum_groups) * kWaves + wave;
    const uint32_t w = job / sets, v0 = job % sets * kZeroRows;
    if (w >= a.workers) return;
    const uint32_t marks = *(const uint32_t*)(seen_of(a, w) + v0);   // of four rows
    const Pack<T, E> zero = {};
    for (uint32_t v = v0; v < min(v0 + kZeroRows, a.vocab); ++v) {
      if (marks >> (v - v0) * 8 & 1) continue;
      T* const p = (T*)a.table.p + (int64_t)w * a.table.worker + (int64_t)v * a.table.row;
      for (uint32_t col = lane * E; col < a.width; col += 64 * E) store_pack<E, ONCE>(p + col, (int)(a.width - col), zero);
    }
    return;
  }
  const uint32_t job = group * kWaves + wave, line = job / a.blocks;
  const uint32_t w = line / a.chunks, c = line % a.chunks;
  if (w >= a.workers) return;
  const uint32_t real = a.real[w], begin = c * kChunk;
  if (begin >= real) return;
  const uint32_t m = min(kChunk, real - begin), col = job % a.blocks * 64 * E + lane * E;
  const int n = (int)a.width - (int)col;
  const uint32_t* const keys = a.key[0] + (uint64_t)w * a.tokens;
  const uint32_t* const poss = a.pos[0] + (uint64_t)w * a.tokens;
  const uint32_t my_key = keys[begin + min((uint32_t)lane, m - 1)], my_pos = poss[begin + min((uint32_t)lane, m - 1)];
  const uint32_t before = begin ? keys[begin - 1] : 0xFFFFFFFFu, after = begin + m < real ? keys[begin + m] : 0xFFFFFFFFu;
  const T* const dy = (const T*)a.rows.p + (int64_t)w * a.rows.worker + col;
  float* const partial = a.partial + ((uint64_t)w * a.chunks + c) * 2 * a.width + col;
  float acc[E] = {};
  uint32_t now = (uint32_t)__builtin_amdgcn_readlane((int)my_key, 0);
  bool head = true;   // the chunk's first number
  auto leave = [&](bool tail) {
    const bool goes_back = head && before == now, goes_on = tail && after == now;
    if (n > 0) {
      if (goes_back || goes_on) store_upto<E>(partial + (goes_back ? 0 : a.width), n, acc);
      else leave_sum<E, T>(a, w, now, col, n, acc);
    }
  };
  Pack<T, E> v[2][AHEAD];   // the next rows are under way while these are added
  auto ask = [&](uint32_t i, int to) {
#pragma unroll
    for (uint32_t j = 0; j < AHEAD; ++j) {
      const uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)my_pos, (int)min(i + j, m - 1));
      if (i < m) v[to][j] = load_pack<E, ONCE>(dy + (int64_t)at * a.rows.row, n);
    }
  };
  ask(0, 0);
#pragma unroll
  for (uint32_t i = 0; i < kChunk; i += AHEAD) {
    if (i >= m) break;
    ask(i + AHEAD, (i / AHEAD + 1) & 1);
#pragma unroll
    for (uint32_t j = 0; j < AHEAD; ++j) {
      if (i + j >= m) break;
      const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)my_key, (int)(i + j));
      if (k != now) {
        leave(false);
        now = k;
        head = false;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += to_f(v[(i / AHEAD) & 1][j].v[e]);
    }
  }
  leave(true);
}

// The numbers that go on from chunk c, where they begin, into the next ones.  A wavefront has 256 columns, sixteen partial sums under way at once: a number that
// every sixteenth of 16384 tokens has goes through 64 chunks.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_embed_join(EmbedArgs a) {
  constexpr int E = 4, AT_ONCE = 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t job = (a.first + blockIdx.x) * kWaves + wave, across = (a.width + 64 * E - 1) / (64 * E), line = job / across;
  const uint32_t w = line / a.chunks, c = line % a.chunks;
  if (w >= a.workers) return;
  const uint32_t real = a.real[w], begin = c * kChunk;
  if (begin + kChunk >= real) return;
  const uint32_t* const keys = a.key[0] + (uint64_t)w * a.tokens;
  const uint32_t k = keys[begin + kChunk - 1], next = keys[begin + kChunk], head = keys[begin], before = begin ? keys[begin - 1] : kNoToken;
  if (next != k || (head == k && before == k)) return;   // ends here, or begins further ahead
  const uint32_t col = (job % across * 64 + lane) * E;
  const int n = (int)a.width - (int)col;
  const float* p = a.partial + ((uint64_t)w * a.chunks + c) * 2 * a.width + col;
  float acc[E];
  load_upto<E>(p + a.width, n, acc);
  for (uint32_t at = begin + kChunk;;) {
    // In how many of the next 64 chunks does it go on?
    const uint64_t there = at + (uint64_t)lane * kChunk;
    const uint64_t not_on = ~__ballot(there < real && keys[there] == k);
    const int on = not_on ? __ffsll((unsigned long long)not_on) - 1 : 64;
    for (int i = 0; i < on; i += AT_ONCE) {
      float v[AT_ONCE][E];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) load_upto<E>(p + (uint64_t)(min(i + j, on - 1) + 1) * 2 * a.width, n, v[j]);
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += i + j < on ? v[j][e] : 0.f;
    }
    if (on < 64) break;
    p += 64 * 2 * (uint64_t)a.width;
    at += 64 * kChunk;
  }
  if (n > 0) leave_sum<E, T>(a, w, k, col, n, acc);
}

}  // namespace
}  // namespace evg

using namespace evg;

struct evg_embed {
  evg_embed_config cfg{};
  hipStream_t stream = nullptr;
  void* owned = nullptr;
  EmbedArgs at{};       // the workspace's parts
  int bits = 1;         // of a token's number
  uint32_t passes = 1;  // of the sort in many workgroups
};

namespace {

template <typename Kernel, typename... More>
hipError_t launch(uint64_t groups, uint32_t threads, hipStream_t s, EmbedArgs& a, Kernel kernel, More... more) {
  launch_pieces(groups, threads, [&](uint32_t first, uint32_t grid) {
    a.first = first;
    kernel<<<grid, threads, 0, s>>>(a, more...);
  });
  return hipGetLastError();
}

uint64_t ids_bytes(const evg_ids* ids, uint32_t workers, uint32_t tokens) {
  return ((uint64_t)(workers - 1) * (uint64_t)ids->worker + tokens) * (ids->wide ? 8 : 4);
}

evg_status check_ids(const evg_ids* ids, uint32_t workers, uint32_t tokens) {
  if (!ids || (tokens && !ids->p)) return fail(EVG_ERR_INVALID, "ids must be given");
  if (!tokens) return EVG_OK;
  if ((uintptr_t)ids->p % (ids->wide ? 8 : 4)) return fail(EVG_ERR_ALIGN, "ids is not aligned to its numbers");
  if (workers > 1 && (ids->worker < 0 || ids->worker >> 44)) return fail(EVG_ERR_INVALID, "ids: the stride is out of range");
  evg_ids one = *ids;
  if (workers <= 1) one.worker = 0;
  return check_device_array(ids->p, ids_bytes(&one, workers, tokens), "ids");
}

Span ids_span(const evg_ids* ids, uint32_t workers, uint32_t tokens) {
  Span s;
  s.what = "ids";
  if (!tokens) return s;
  evg_ids one = *ids;
  if (workers <= 1) one.worker = 0;
  s.begin = (uintptr_t)ids->p;
  s.end = s.begin + ids_bytes(&one, workers, tokens);
  return s;
}

EmbedArgs embed_args(const evg_embed* c, uint32_t tokens, const evg_ids* ids, const evg_mat* table, const evg_mat* rows) {
  const evg_embed_config& g = c->cfg;
  EmbedArgs a = c->at;
  a.ids = ids->p;
  a.ids_worker = g.workers > 1 ? ids->worker : 0;
  a.wide = ids->wide;
  a.table = *table;
  a.rows = *rows;
  if (g.workers <= 1) a.table.worker = a.rows.worker = 0;
  if (tokens <= 1) a.rows.row = 0;
  if (g.vocab <= 1) a.table.row = 0;
  a.workers = g.workers, a.lines = g.workers * tokens, a.tokens = tokens, a.vocab = g.vocab, a.width = g.width;
  const uint32_t across = 64 * 16 / type_bytes(g.type);
  a.blocks = (g.width + across - 1) / across;
  a.scale = g.scale;
  return a;
}

template <typename T>
hipError_t embed_forward(const evg_embed* c, EmbedArgs& a) {
  const uint64_t units = (uint64_t)a.lines * a.blocks;
  // Few units go to a wavefront each: the chip has room for 8192 of them.
  const uint32_t each = units <= 8192 ? 1 : 4;
  const uint64_t groups = (units + each * kWaves - 1) / (each * kWaves);
  return launch(groups, kThreads, c->stream, a, each == 1 ? k_embed_rows<T, 1> : k_embed_rows<T, 4>);
}

template <typename T>
hipError_t embed_sums(const evg_embed* c, EmbedArgs& a) {
  a.chunks = (a.tokens + kChunk - 1) / kChunk;
  const uint64_t groups = ((uint64_t)a.workers * a.chunks * a.blocks + kWaves - 1) / kWaves;
  const uint64_t zero = a.accumulate ? 0 : ((uint64_t)a.workers * ((a.vocab + kZeroRows - 1) / kZeroRows) + kWaves - 1) / kWaves;
  a.sum_groups = (uint32_t)groups;
  const bool once = (uint64_t)a.workers * a.vocab * a.width * sizeof(T) > (128u << 20);   // half of the last-level cache
  const hipError_t e = launch(groups + zero, kThreads, c->stream, a, once ? k_embed_sum<T, true> : k_embed_sum<T, false>);
  if (e != hipSuccess || a.chunks <= 1) return e;
  const uint64_t joins = (uint64_t)a.workers * a.chunks * ((a.width + 255) / 256);
  return launch((joins + kWaves - 1) / kWaves, kThreads, c->stream, a, k_embed_join<T>);
}

template <typename T>
hipError_t embed_backward(const evg_embed* c, EmbedArgs& a) {
  hipStream_t s = c->stream;
  hipError_t e;
  int place_bits = 1;
  while (a.tokens > 1u << place_bits) ++place_bits;
  if (a.tokens <= kFewTokens && c->bits + place_bits < 32) {
    if ((e = launch(a.workers, kFewTokens, s, a, k_embed_sort_few, place_bits)) != hipSuccess) return e;
  } else if (a.tokens <= kOneSort) {
    const uint32_t per = (a.tokens + kOneWaves * 64 - 1) / (kOneWaves * 64);
    if ((e = launch(a.workers, kOneWaves * 64, s, a, per <= 1 ? k_embed_sort_alone<1> : k_embed_sort_alone<kPer>, c->bits)) != hipSuccess)
      return e;
  } else {
    const Runs runs = cut_runs(a.tokens, kThreads * kPer);
    a.run = runs.each, a.runs = runs.count;
    a.bits = (c->bits + c->passes - 1) / c->passes;
    a.bins = 1u << a.bits;
    for (uint32_t p = 0; p < c->passes; ++p) {
      // The last pass ends in buffer 0.
      const uint32_t to = (c->passes - 1 - p) & 1;
      a.shift = p * a.bits;
      a.last = p + 1 == c->passes;
      const uint32_t* keys = p ? a.key[to ^ 1] : nullptr;
      if ((e = launch((uint64_t)a.workers * a.runs, kThreads, s, a, k_embed_count, keys)) != hipSuccess) return e;
      if ((e = launch((uint64_t)a.workers * a.runs, kThreads, s, a, k_embed_place, keys, (const uint32_t*)a.pos[to ^ 1], a.key[to], a.pos[to])) != hipSuccess) return e;
    }
  }
  return embed_sums<T>(c, a);
}

}  // namespace

extern "C" {

evg_status evg_embed_init(evg_embed** out, const evg_embed_config* cfg, void* hip_stream) {
  if (!out || !cfg) return fail(EVG_ERR_INVALID, "out and cfg must be non-NULL");
  *out = nullptr;
  if (cfg->workers < 1 || cfg->workers > 65535) return fail(EVG_ERR_INVALID, "workers must be 1 .. 65535");
  if (cfg->vocab < 1 || cfg->vocab > (1u << 24)) return fail(EVG_ERR_INVALID, "vocab must be 1 .. 2^24");
  if (cfg->width < 1 || cfg->width > (1u << 20)) return fail(EVG_ERR_INVALID, "width must be 1 .. 2^20");
  if (cfg->max_tokens > (1u << 26)) return fail(EVG_ERR_INVALID, "max_tokens must be at most 2^26");
  evg_status st;
  if ((st = check_type(cfg->type, "type")) != EVG_OK) return st;
  // Kernels count units of 64 vectors, and sets of rows, in 32 bits.
  const uint64_t across = ((uint64_t)cfg->width * type_bytes(cfg->type) + 1023) / 1024;
  if (cfg->workers * (uint64_t)cfg->max_tokens * across > 0x7FFFFFFFull || cfg->workers * (uint64_t)cfg->vocab > 0x7FFFFFFFull)
    return fail(EVG_ERR_INVALID, "workers, width and max_tokens or vocab together are out of range");
  if (!std::isfinite(cfg->scale)) return fail(EVG_ERR_INVALID, "scale must be finite");
  evg_embed* c = new (std::nothrow) evg_embed();
  if (!c) return fail(EVG_ERR_OOM, "host allocation failed");
  c->cfg = *cfg;
  c->stream = static_cast<hipStream_t>(hip_stream);
  while ((cfg->vocab - 1) >> c->bits) ++c->bits;
  c->passes = (uint32_t)(c->bits + 9) / 10;
  if (cfg->train) {
    const uint64_t W = cfg->workers, T = cfg->max_tokens;
    const bool many = T > kOneSort;
    // Fewer tokens may be cut into as many runs.
    const uint32_t bins = 1u << ((c->bits + c->passes - 1) / c->passes), runs = many ? kMostRuns : 0;
    const uint64_t chunks = (T + kChunk - 1) / kChunk;
    const uint64_t words[] = {W * T, W * T, many && c->passes > 1 ? W * T : 0, many && c->passes > 1 ? W * T : 0, W * runs * bins, W,
                              W * ((cfg->vocab + 3) / 4), chunks > 1 ? W * chunks * 2 * cfg->width : 0};
    uint64_t total = 0;
    for (uint64_t n : words) total += (n + 63) / 64 * 64;
    const hipError_t e = total >> 46 ? hipErrorOutOfMemory : hipMalloc(&c->owned, total * 4);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      delete c;
      return fail(e == hipErrorOutOfMemory ? EVG_ERR_OOM : EVG_ERR_HIP, "workspace: %s", hipGetErrorString(e));
    }
    uint32_t* p = (uint32_t*)c->owned;
    uint32_t** const to[] = {&c->at.key[0], &c->at.pos[0], &c->at.key[1], &c->at.pos[1], &c->at.counts, &c->at.real, (uint32_t**)&c->at.seen, (uint32_t**)&c->at.partial};
    for (int i = 0; i < 8; ++i) {
      *to[i] = p;
      p += (words[i] + 63) / 64 * 64;
    }
  }
  *out = c;
  return EVG_OK;
}

evg_status evg_embed_forward(evg_embed* c, uint32_t tokens, const evg_ids* ids, const evg_mat* table, const evg_mat* y) {
  if (!c) return fail(EVG_ERR_INVALID, "context must be non-NULL");
  const evg_embed_config& g = c->cfg;
  if (tokens > g.max_tokens) return fail(EVG_ERR_INVALID, "tokens exceeds the context's max_tokens");
  evg_status st;
  if ((st = check_ids(ids, g.workers, tokens)) != EVG_OK) return st;
  if ((st = check_mat(table, g.workers, g.vocab, g.width, g.type, false, "table")) != EVG_OK) return st;
  if ((st = check_mat(y, g.workers, tokens, g.width, g.type, true, "y")) != EVG_OK) return st;
  const Span ins[] = {mat_span(table, g.workers, g.vocab, g.width, g.type, "table"), ids_span(ids, g.workers, tokens)};
  const Span outs[] = {mat_span(y, g.workers, tokens, g.width, g.type, "y")};
  if ((st = check_apart(outs, 1, ins, 2)) != EVG_OK) return st;
  if (!tokens) return EVG_OK;
  EmbedArgs a = embed_args(c, tokens, ids, table, y);
  HIP_TRY(g.type == EVG_F32 ? embed_forward<float>(c, a) : g.type == EVG_F16 ? embed_forward<half_t>(c, a) : embed_forward<bf16_t>(c, a));
  return EVG_OK;
}

evg_status evg_embed_backward(evg_embed* c, uint32_t tokens, const evg_ids* ids, const evg_mat* dy, const evg_mat* d_table, uint32_t accumulate) {
  if (!c) return fail(EVG_ERR_INVALID, "context must be non-NULL");
  const evg_embed_config& g = c->cfg;
  if (!g.train) return fail(EVG_ERR_STATE, "the context was made without train");
  if (tokens > g.max_tokens) return fail(EVG_ERR_INVALID, "tokens exceeds the context's max_tokens");
  evg_status st;
  if ((st = check_ids(ids, g.workers, tokens)) != EVG_OK) return st;
  if ((st = check_mat(dy, g.workers, tokens, g.width, g.type, false, "dy")) != EVG_OK) return st;
  if ((st = check_mat(d_table, g.workers, g.vocab, g.width, g.type, true, "d_table")) != EVG_OK) return st;
  const Span ins[] = {mat_span(dy, g.workers, tokens, g.width, g.type, "dy"), ids_span(ids, g.workers, tokens)};
  const Span outs[] = {mat_span(d_table, g.workers, g.vocab, g.width, g.type, "d_table")};
  if ((st = check_apart(outs, 1, ins, 2)) != EVG_OK) return st;
  EmbedArgs a = embed_args(c, tokens, ids, d_table, dy);
  a.accumulate = accumulate != 0;
  HIP_TRY(g.type == EVG_F32 ? embed_backward<float>(c, a) : g.type == EVG_F16 ? embed_backward<half_t>(c, a) : embed_backward<bf16_t>(c, a));
  return EVG_OK;
}

evg_status evg_embed_destroy(evg_embed* c) {
  if (!c) return EVG_OK;
  hipError_t e = hipStreamSynchronize(c->stream);
  if (c->owned) { const hipError_t f = hipFree(c->owned); if (e == hipSuccess) e = f; }
  delete c;
  HIP_TRY(e);
  return EVG_OK;
}

}  // extern "C"
