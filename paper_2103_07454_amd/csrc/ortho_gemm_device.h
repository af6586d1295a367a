// The products of orthogonal updates on the matrix cores: float16 operands, sums in 32 bits.
//
// C[m][n] = f_acc sum_k A(m, k) B(n, k) + f_own own[m][n].  A workgroup has a tile of BM x BM; tiles, the way of units through LDS and the order of a lane's results
// are those of gemm_tile_device.h.  A step is 128 bytes of k: 64 elements of hi, or (SPLIT) 32 of hi and the same 32 of lo, from which three products are made: of hi
// and hi, of hi and lo and of lo and hi (lo and lo is 2^-22 of it and left out).  So a fragment that is read from LDS goes into one or two
// products, where three passes over k would read each for every product.
//
// S and P are symmetric: tiles below the diagonal are not computed, those above it are written twice, the second time turned round.
//
// Bound by the matrix cores, the clock that power leaves them and rounds of workgroups that do not fill the CUs (P of 4096 has 136 tiles of 256 for 256 CUs, S 408, X 704): 4096 x 11264, hi alone, X 386 us (0.98 PFLOP/s; 425 with what is added read four columns a lane), S 207 + 24
// (0.82), P 105.  Small ones by the steps' latency, 0.45 us each.
//
// Where tiles are few, k is shared out to several workgroups, whose sums go to memory in the accumulators' order; a launch behind adds them up in a fixed order.
#pragma once
#include "gemm_tile_device.h"
#include "ortho_choose.h"
#include "ortho_internal.h"

namespace evg {

// Which tile of a symmetric product: bands of four rows of tiles, each from its diagonal on, column by column.
__device__ __forceinline__ void symmetric_tile(uint32_t id, uint32_t tiles, uint32_t* tm, uint32_t* tn) {
  uint32_t first = 0;
  for (;;) {
    const uint32_t rows = min(4u, tiles - first), cells = rows * (tiles - first);
    if (id < cells) {
      *tm = first + id % rows;
      *tn = first + id / rows;
      return;
    }
    id -= cells;
    first += 4;
  }
}

template <bool SYMMETRIC>
__device__ __forceinline__ void tile_of(const OrthoArgs& g, uint32_t id, uint32_t* tm, uint32_t* tn) {
  if constexpr (SYMMETRIC) {
    symmetric_tile(id, g.tiles_m, tm, tn);
  } else {
    constexpr uint32_t BAND = 4;
    const uint32_t band = BAND * g.tiles_n, first = id / band * BAND, rows = min(BAND, g.tiles_m - first);
    *tm = first + id % band % rows;
    *tn = id % band / rows;
  }
}

// An operand's tile in LDS, in units of 16 bytes, permuted for LDS as this chip reads it: 64 banks, 256 bytes at a time.  K-contiguous: row m has 8 units, unit c at
// m * 8 + (c ^ (m >> 1 & 7)), so that the 16 lanes that read one unit each of 16 neighbouring rows meet all banks (by
// m & 7 half of LDS's cycles were conflicts, now none are; the products' time, which is not LDS's, stayed as it was).  M/N-contiguous: row k has BD / 8 units; 32 lanes of a transposing read take 4 units of each of 4 neighbouring rows.
template <int BD, bool KC>
struct HalvesTile {
  static constexpr int kUnits = BD * 8, kPerRow = KC ? 8 : BD / 8;
  static __device__ __forceinline__ int swizzle(int row) {
    if constexpr (KC) return row >> 1 & 7;
    else if constexpr (BD >= 128) return (row & 3) << 2;
    else return (row >> 1 & 1) << 2;
  }
};

// Fragment `ks` (0 .. 3: 32 bytes of k) of the 32 rows from d0 on, of a tile `from` units into a buffer.
template <int BD, bool KC>
__device__ __forceinline__ Frag<half_t> read_halves(const u32x4* s, int from, int d0, int ks, int lane) {
  using L = HalvesTile<BD, KC>;
  Frag<half_t> f;
  if constexpr (KC) {
    const int row = d0 + (lane & 31);
    f.v = s[from + row * 8 + ((ks * 2 + (lane >> 5)) ^ L::swizzle(row))];
  } else {
    const int q = lane >> 4, i = lane & 15;
    const int k = ks * 16 + (q >> 1) * 8 + (i >> 2);
    const int unit = (d0 >> 3) + (q & 1) * 2 + ((i & 3) >> 1);
    const int byte = (from + k * L::kPerRow + (unit ^ L::swizzle(k))) * 16 + (i & 1) * 8;
    using P = __attribute__((address_space(3))) s16x4*;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)((const char*)s + byte));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)((const char*)s + (byte + 4 * L::kPerRow * 16)));   // 4 rows on, which are permuted alike
    struct { s16x4 a, b; } both{lo, hi};
    f.v = __builtin_bit_cast(u32x4, both);
  }
  return f;
}

// One operand's way into LDS.
template <int BD, bool KC, int WAVES, bool SPLIT>
struct HalvesLoader {
  using L = HalvesTile<BD, KC>;
  static constexpr int N = L::kUnits / 64 / WAVES;            // loads of a wavefront in a step
  static constexpr int kApart = KC ? 8 : 64 / L::kPerRow;     // rows between them
  static constexpr int BK = SPLIT ? 32 : 64;
  const char* base;   // the tile's first element at the next step
  uint64_t left;      // bytes from there to the matrix's end
  uint64_t stride;    // bytes from step to step
  uint32_t off[N];    // of this lane's units
  uint32_t k;         // of its first unit, within a step

  __device__ __forceinline__ void start(const Halves& o, uint32_t w, uint32_t lead, uint32_t dim, uint32_t K, uint32_t step, int wave, int lane) {
    const uint64_t ld = (uint64_t)o.ld * 2, from = KC ? lead * ld : (uint64_t)halves_col(SPLIT, lead) * 2;
    stride = KC ? 128 : BK * ld;
    const uint64_t bytes = (KC ? (uint64_t)dim : (uint64_t)K) * ld, at = from + step * stride;
    base = (const char*)(o.p + (int64_t)w * o.worker) + at;
    left = bytes > at ? bytes - at : 0;
    const int place = wave * N * 64 + lane;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int row = place / L::kPerRow + j * kApart, unit = (place % L::kPerRow) ^ L::swizzle(row);
      if constexpr (KC) {
        off[j] = (uint32_t)(row * ld) + unit * 16;   // rows beyond the last one lie beyond `left`
        if (j == 0) k = SPLIT ? (unit & 3) * 8 : unit * 8;
      } else {
        const uint32_t d = unit * 8, kr = SPLIT ? row & 31 : row;
        off[j] = lead + d < dim ? (uint32_t)(kr * ld) + (SPLIT ? ((d & ~31u) * 2 + (d & 31) + (row & 32)) : d) * 2 : kOut;
        if (j == 0) k = row;
      }
    }
  }

  // Does unit j lie behind the last k?
  __device__ __forceinline__ bool behind(int j, int k_left) const {
    if constexpr (KC) return (int)(SPLIT ? k : k ^ (j & 1) * 32) >= k_left;   // in rows 8 apart unit c is where c ^ 4 is
    else return (int)(SPLIT ? (k + j * kApart) & 31 : k + j * kApart) >= k_left;
  }

  // The next step, of which k_left elements of k are there; zeros where that is none.
  __device__ __forceinline__ void fetch(int k_left, u32x4* lds, int wave) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)(uint32_t)min(left, (uint64_t)0x7FFFFFF0u), 0x00020000);
    auto load = [&](int j, uint32_t at) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (wave * N + j) * 64), 16, (int)at, 0, 0, 0);
    };
#pragma unroll
    for (int j = 0; j < N; ++j) load(j, off[j] | (behind(j, k_left) ? kOut : 0));
    base += stride;
    left -= min(left, stride);
  }
};

// This wavefront's loads into LDS have arrived but for the last `MORE`, its reads of LDS are done; then the workgroup meets.
template <int MORE>
__device__ __forceinline__ void wait_but_and_meet() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt((MORE & 15) | (MORE >> 4) << 14 | 7 << 4);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// 32 rows from rows0 on and 32 TN columns from cols0 on of the result, from their sums acc(j, q): a lane has, of its row, four times four neighbouring columns of each
// 32.  Rows leave through `room`, 32 * 4 * TN units of LDS of the wavefront's own, as whole lines.  turned: they are written as columns too.
template <int OP, bool LAST, int TN, typename Acc>
__device__ __forceinline__ void finish_rows(const OrthoArgs& g, uint32_t w, uint32_t rows0, uint32_t cols0, bool turned, u32x4* room, int lane, Acc acc) {
  typedef half_t T;
  constexpr int PER = TN * 4;   // 16-byte units of a row
  const uint32_t m = rows0 + (lane & 31), limit = (g.N + 7) & ~7u;   // columns up to a whole unit are 0
  Pack<T, 4> hi[TN][4], lo[TN][4], own[TN][4], own_lo[TN][4];
  // A lane's four columns of 32 j + 8 q in `room`, of which the wavefront moves whole units.
  auto place = [&](int j, int q) { return (Pack<T, 4>*)((char*)(room + (lane & 31) * PER + ((j * 4 + q) ^ (lane & (PER - 1)))) + (lane >> 5) * 8); };
  if constexpr (OP != ORTHO_GRAM) {
    u32x4 unit[2][PER / 2];
#pragma unroll
    for (int r = 0; r < PER / 2; ++r) {
      const uint32_t at = r * 64 + lane, row = rows0 + at / PER, n = cols0 + at % PER * 8;
      unit[0][r] = unit[1][r] = u32x4{0, 0, 0, 0};
      if (row < g.M && n < limit) {
        const uint16_t* const p = g.own.p + (int64_t)w * g.own.worker + (int64_t)row * g.own.ld + halves_col(g.own.paired, n);
        unit[0][r] = *(const u32x4*)p;
        if (g.own.apart) unit[1][r] = *(const u32x4*)(p + g.own.apart);
      }
    }
    auto spread = [&](const u32x4* v, Pack<T, 4> (&to)[TN][4]) {
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int r = 0; r < PER / 2; ++r) {
        const int at = r * 64 + lane, row = at / PER;
        room[row * PER + (at % PER ^ (row & (PER - 1)))] = v[r];
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) to[j][q] = *place(j, q);
    };
    spread(unit[0], own);
    spread(unit[1], own_lo);
  }
  auto value = [&](int j, int q, int e) {
    const float p = acc(j, q)[e] * g.f_acc;
    if constexpr (OP == ORTHO_GRAM) return p;
    else return fmaf(to_f(own[j][q].v[e]) + to_f(own_lo[j][q].v[e]), g.f_own, p);
  };
  if constexpr (LAST) {
    if (g.out_type == EVG_F32) {
      if (m >= g.M) return;
      float* const p = (float*)g.out.p + (int64_t)w * g.out.worker + (int64_t)m * g.out.row;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t n = cols0 + j * 32 + 8 * q + 4 * (lane >> 5);
          const float x[4] = {value(j, q, 0), value(j, q, 1), value(j, q, 2), value(j, q, 3)};
          store_upto<4>(p + n, n < g.N ? (int)(g.N - n) : 0, x);
        }
    } else {
      auto leave_as = [&](auto type) {
        typedef decltype(type) U;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            Pack<U, 4> x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x.v[e] = from_f<U>(value(j, q, e));
            *place(j, q) = __builtin_bit_cast(Pack<T, 4>, x);
          }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int r = 0; r < PER / 2; ++r) {
          const int at = r * 64 + lane, row = at / PER, unit = at % PER;
          const Pack<U, 8> x = __builtin_bit_cast(Pack<U, 8>, room[row * PER + (unit ^ (row & (PER - 1)))]);
          const uint32_t n = cols0 + unit * 8;
          if (rows0 + row < g.M) store_pack<8>((U*)g.out.p + (int64_t)w * g.out.worker + (int64_t)(rows0 + row) * g.out.row + n, n < g.N ? (int)(g.N - n) : 0, x);
        }
      };
      if (g.out_type == EVG_F16) leave_as(half_t{});
      else leave_as(bf16_t{});
    }
  } else {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) halves_of(value(j, q, e), &hi[j][q].v[e], &lo[j][q].v[e]);
    uint16_t* const to = g.to.p + (int64_t)w * g.to.worker;
    auto leave = [&](const Pack<T, 4> (&v)[TN][4], int64_t apart) {
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) *place(j, q) = v[j][q];
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int r = 0; r < PER / 2; ++r) {
        const int at = r * 64 + lane, row = at / PER, unit = at % PER;
        const u32x4 x = room[row * PER + (unit ^ (row & (PER - 1)))];
        const uint32_t n = cols0 + unit * 8;
        if (rows0 + row < g.M && n < limit) *(u32x4*)(to + (int64_t)(rows0 + row) * g.to.ld + halves_col(g.to.paired, n) + apart) = x;
      }
    };
    // Turned tiles lie below the diagonal: their columns are all real.
    auto leave_turned = [&](const Pack<T, 4> (&v)[TN][4], int64_t apart) {
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) ((T*)room)[(j * 32 + 8 * q + 4 * (lane >> 5) + e) * 32 + (lane & 31)] = v[j][q].v[e];
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int r = 0; r < TN * 2; ++r) {
        const int at = r * 64 + lane, row = at / 4, unit = at % 4;
        const u32x4 x = room[at];
        if (cols0 + row < g.N) *(u32x4*)(to + (int64_t)(cols0 + row) * g.to.ld + halves_col(g.to.paired, rows0 + unit * 8) + apart) = x;
      }
    };
    leave(hi, 0);
    if (g.to.apart) leave(lo, g.to.apart);
    if (turned) {
      leave_turned(hi, 0);
      if (g.to.apart) leave_turned(lo, g.to.apart);
    }
  }
}

template <int OP, bool TALL, bool SPLIT, bool LAST, int BM, int WAVES_M, int WAVES_N>
__global__ __launch_bounds__(WAVES_M * WAVES_N * 64, 2) void k_ortho_gemm(OrthoArgs g) {
  typedef half_t T;
  constexpr bool SYMMETRIC = OP != ORTHO_APPLY;
  constexpr bool AKC = !(OP == ORTHO_GRAM && TALL), BKC = OP == ORTHO_SQUARE || (OP == ORTHO_GRAM ? !TALL : TALL);
  constexpr int WAVES = WAVES_M * WAVES_N, WM = BM / WAVES_M, TM = WM / 32, WN = BM / WAVES_N, TN = WN / 32;
  using LA = HalvesLoader<BM, AKC, WAVES, SPLIT>;
  using LB = HalvesLoader<BM, BKC, WAVES, SPLIT>;
  constexpr int A_UNITS = LA::L::kUnits, UNITS = A_UNITS + LB::L::kUnits, LOADS = LA::N + LB::N, BK = LA::BK;
  // Tiles of 64 have steps of four products a wavefront: three of them are under way ahead of the one that is multiplied.
  constexpr bool DEEP = BM == 64;
  __shared__ u32x4 lds0[UNITS], lds1[UNITS], lds2[DEEP ? UNITS : 1], lds3[DEEP ? UNITS : 1];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t id = place_by_xcd(g.first);
  const uint32_t cell = id % g.cells, part = id / g.cells % g.parts, w = id / g.cells / g.parts;
  uint32_t tm, tn;
  tile_of<SYMMETRIC>(g, cell, &tm, &tn);
  if (SYMMETRIC && tn < tm) return;
  const uint32_t m0 = tm * BM, n0 = tn * BM;

  LA la;
  LB lb;
  const uint32_t first = part * g.part_steps, steps = min(g.part_steps, (g.K + BK - 1) / BK - first);
  int k_left = (int)min(g.K - first * BK, steps * BK);   // what lies behind is another part's
  auto fetch = [&](u32x4* lds) {
    la.fetch(k_left, lds, wave);
    lb.fetch(k_left, lds + A_UNITS, wave);
    k_left -= BK;
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  const int wm = wave / WAVES_N * WM, wn = wave % WAVES_N * WN;
  Frag<T> a[2][TM], b[2][TN];
  auto multiply = [&](const u32x4* lds) {
    auto read = [&](int ks, int to) {
#pragma unroll
      for (int j = 0; j < TN; ++j) b[to][j] = read_halves<BM, BKC>(lds, A_UNITS, wn + j * 32, ks, lane);
#pragma unroll
      for (int i = 0; i < TM; ++i) a[to][i] = read_halves<BM, AKC>(lds, 0, wm + i * 32, ks, lane);
    };
    auto product = [&](int of_a, int of_b) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mfma(b[of_b][j], a[of_a][i], acc[i][j]);
    };
    if constexpr (SPLIT) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        read(half, 0);
        read(half + 2, 1);
        product(0, 0);
        product(0, 1);
        product(1, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      read(0, 0);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        if (ks < 3) read(ks + 1, (ks + 1) & 1);
        product(ks & 1, ks & 1);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  la.start(g.a, w, m0, g.M, g.K, first, wave, lane);
  lb.start(g.b, w, n0, g.N, g.K, first, wave, lane);
  fetch(lds0);
  if constexpr (DEEP) {
    fetch(lds1);
    fetch(lds2);
    for (uint32_t step = 0; step < steps; step += 4) {   // steps behind the last one are of zeros and left out
      wait_but_and_meet<2 * LOADS>();
      fetch(lds3);
      multiply(lds0);
      wait_but_and_meet<2 * LOADS>();
      fetch(lds0);
      if (step + 1 < steps) multiply(lds1);
      wait_but_and_meet<2 * LOADS>();
      fetch(lds1);
      if (step + 2 < steps) multiply(lds2);
      wait_but_and_meet<2 * LOADS>();
      fetch(lds2);
      if (step + 3 < steps) multiply(lds3);
    }
    wait_but_and_meet<0>();   // LDS is free for the results
  } else {
    for (uint32_t step = 0; step < steps; step += 2) {   // an odd last step is followed by one of zeros
      const bool more = step + 2 < steps;
      wait_but_and_meet<0>();
      fetch(lds1);
      multiply(lds0);
      wait_but_and_meet<0>();
      if (more) fetch(lds0);
      multiply(lds1);
      if (!more) wait_but_and_meet<0>();   // LDS is free for the results
    }
  }

  if (g.parts > 1) {
    float* const to = g.partial + (((uint64_t)w * g.parts + part) * g.cells + cell) * (BM * BM) + wave * (TM * TN * 1024) + lane * 4;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 v = {acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
          *(f32x4*)(to + (i * TN + j) * 1024 + q * 256) = v;
        }
    return;
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const uint32_t rows0 = m0 + wm + i * 32;
    if (rows0 >= g.M) break;
    finish_rows<OP, LAST, TN>(g, w, rows0, n0 + wn, SYMMETRIC && tm != tn, lds0 + wave * (32 * TN * 4), lane, [&](int j, int q) {
      return f32x4{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
    });
  }
}

// Adds up the parts of 32 rows of a tile's wavefront's columns, in their order, and finishes them.
template <int OP, bool LAST, int BM, int WAVES_M, int WAVES_N>
__global__ __launch_bounds__(256) void k_ortho_join(OrthoArgs g) {
  constexpr bool SYMMETRIC = OP != ORTHO_APPLY;
  constexpr int WAVES = WAVES_M * WAVES_N, WM = BM / WAVES_M, TM = WM / 32, WN = BM / WAVES_N, TN = WN / 32;
  __shared__ u32x4 room[4][32 * TN * 4];
  const int lane = threadIdx.x & 63, own = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t job = (g.first + blockIdx.x) * 4 + own, i = job % TM, wave = job / TM % WAVES, cell = job / (TM * WAVES) % g.cells, w = job / (TM * WAVES) / g.cells;
  if (w >= g.matrices) return;
  uint32_t tm, tn;
  tile_of<SYMMETRIC>(g, cell, &tm, &tn);
  const uint32_t rows0 = tm * BM + wave / WAVES_N * WM + i * 32, cols0 = tn * BM + wave % WAVES_N * WN;
  if ((SYMMETRIC && tn < tm) || rows0 >= g.M) return;
  const uint64_t apart = (uint64_t)g.cells * (BM * BM);
  const float* p = g.partial + ((uint64_t)w * g.parts * g.cells + cell) * (BM * BM) + (wave * TM + i) * (TN * 1024) + lane * 4;
  f32x4 sum[TN][4];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[j][q] = *(const f32x4*)(p + j * 1024 + q * 256);
#pragma unroll 2
  for (uint32_t part = 1; part < g.parts; ++part) {
    p += apart;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) sum[j][q] += *(const f32x4*)(p + j * 1024 + q * 256);
  }
  finish_rows<OP, LAST, TN>(g, w, rows0, cols0, SYMMETRIC && tm != tn, room[own], lane, [&](int j, int q) { return sum[j][q]; });
}

template <int OP, bool TALL, bool SPLIT, bool LAST, int BM, int WAVES_M, int WAVES_N>
hipError_t launch_ortho_tile(OrthoArgs a, uint32_t parts, hipStream_t s) {
  constexpr uint32_t BK = SPLIT ? 32 : 64;
  a.tiles_m = (a.M + BM - 1) / BM;
  a.tiles_n = (a.N + BM - 1) / BM;
  const uint64_t cells = ortho_cells(OP != ORTHO_APPLY, a.tiles_m, a.tiles_n);
  const uint32_t steps = (a.K + BK - 1) / BK;
  a.cells = (uint32_t)cells;
  a.part_steps = (steps + parts - 1) / parts;
  a.parts = (steps + a.part_steps - 1) / a.part_steps;
  const uint64_t groups = cells * a.matrices * a.parts;
  if (groups > 0x7FFFFFFFull || (a.parts > 1 && groups * (BM * BM) > a.room)) return hipErrorInvalidValue;
  launch_pieces(groups, WAVES_M * WAVES_N * 64, [&](uint32_t first, uint32_t grid) {
    a.first = first;
    k_ortho_gemm<OP, TALL, SPLIT, LAST, BM, WAVES_M, WAVES_N><<<grid, WAVES_M * WAVES_N * 64, 0, s>>>(a);
  });
  if constexpr (BM < 256 || OP != ORTHO_APPLY) if (a.parts > 1) {
    const uint64_t joins = (cells * a.matrices * (BM / 32) * WAVES_N + 3) / 4;
    launch_pieces(joins, 256, [&](uint32_t first, uint32_t grid) {
      a.first = first;
      k_ortho_join<OP, LAST, BM, WAVES_M, WAVES_N><<<grid, 256, 0, s>>>(a);
    });
  }
  return hipGetLastError();
}

template <int OP, bool TALL, bool SPLIT, bool LAST>
hipError_t launch_ortho_op(const OrthoArgs& a, hipStream_t s) {
  const OrthoChoice c = choose_ortho({a.M, a.N, a.K, a.matrices, a.room}, OP != ORTHO_APPLY, SPLIT);
  if (c.tile == 64) return launch_ortho_tile<OP, TALL, SPLIT, LAST, 64, 2, 2>(a, c.parts, s);
  if (c.tile == 128) return launch_ortho_tile<OP, TALL, SPLIT, LAST, 128, 2, 2>(a, c.parts, s);
  if constexpr (SPLIT) return hipErrorInvalidValue;
  else return launch_ortho_tile<OP, TALL, SPLIT, LAST, 256, 2, 4>(a, c.parts, s);
}

template <bool SPLIT>
hipError_t launch_ortho_any(OrthoOp op, bool tall, bool last, const OrthoArgs& a, hipStream_t s) {
  if (op == ORTHO_GRAM) return tall ? launch_ortho_op<ORTHO_GRAM, true, SPLIT, false>(a, s) : launch_ortho_op<ORTHO_GRAM, false, SPLIT, false>(a, s);
  if (op == ORTHO_SQUARE) return launch_ortho_op<ORTHO_SQUARE, false, SPLIT, false>(a, s);
  if (last) return tall ? launch_ortho_op<ORTHO_APPLY, true, SPLIT, true>(a, s) : launch_ortho_op<ORTHO_APPLY, false, SPLIT, true>(a, s);
  return tall ? launch_ortho_op<ORTHO_APPLY, true, SPLIT, false>(a, s) : launch_ortho_op<ORTHO_APPLY, false, SPLIT, false>(a, s);
}

}  // namespace evg
