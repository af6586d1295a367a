// Tiles of matrix products on the matrix cores: operands' ways through LDS into fragments.
//
// An operand is K-contiguous (rows of k) or M/N-contiguous (rows of m or n).  Each step of 128 bytes of k (64 elements of 16 bits, 32 of 32) is staged
// through LDS.
//
// LDS, in units of 16 bytes.  K-contiguous: row m has 8 units, unit c at m * 8 + (c ^ (m & 7)): the 8 lanes that read one unit each
// of 8 neighbouring rows meet 8 different groups of banks.  M/N-contiguous: row k has BM / E units (E elements to a unit).  16-bit
// fragments come by transposing reads: 16 lanes read 4 rows of 32 bytes and each gets 4 k of one m.  A read touches 16 rows k; units
// are permuted in pairs by ((k & 3) | (k >> 3 & 1) << 2), so that 8 of them meet all banks.  32-bit fragments are read element by
// element; rows that differ in bit 2 of k go to different halves of the banks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gemm_operand.h"
#include "nn_device.h"

namespace evg {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Frag { u32x4 v; };   // 16 bytes of k of one m or n

__device__ __forceinline__ f32x16 mfma(const Frag<half_t>& a, const Frag<half_t>& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a.v), __builtin_bit_cast(f16x8, b.v), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.v), __builtin_bit_cast(bf16x8, b.v), c, 0, 0, 0);
}
// The instruction takes 2 k, one from each half of the wavefront; four of them take the 8 that the fragments hold.
__device__ __forceinline__ f32x16 mfma(const Frag<float>& a, const Frag<float>& b, f32x16 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.v[i]), __uint_as_float(b.v[i]), c, 0, 0, 0);
  return c;
}

constexpr uint32_t kOut = 0x80000000u;   // a byte offset beyond every buffer: such loads give 0

template <typename T, int BD, bool KC>   // one operand's tile: BD rows or columns of the product, K-contiguous or not
struct Tile {
  static constexpr int E = 16 / sizeof(T), BK = 128 / sizeof(T);
  static constexpr int kUnits = BD * 8;
  static constexpr int kPerRow = KC ? 8 : BD / E;   // units of a row in LDS
  // The unit that lies at a place, as (row, unit of the row).
  static __device__ __forceinline__ int swizzle(int row) {
    if constexpr (KC) return row & 7;
    else if constexpr (sizeof(T) == 4) return BD >= 64 ? (row >> 2 & 1) << 3 : 0;
    else if constexpr (BD >= 128) return ((row & 3) | (row >> 3 & 1) << 2) << 1;
    else if constexpr (BD == 64) return ((row >> 1 & 1) | (row >> 3 & 1) << 1) << 1;
    else return (row >> 3 & 1) << 1;
  }
};

// Fragment `ks` (0 .. 3: 32 bytes of k) of the 32 rows from d0 on, of a tile `from` units into a buffer.  Addresses are one offset from
// the buffer: the compiler follows them no further when it looks for loads into LDS that a read has to wait for.
template <typename T, int BD, bool KC>
__device__ __forceinline__ Frag<T> read_frag(const u32x4* s, int from, int d0, int ks, int lane) {
  using L = Tile<T, BD, KC>;
  Frag<T> f;
  if constexpr (KC) {
    const int row = d0 + (lane & 31);
    f.v = s[from + row * 8 + ((ks * 2 + (lane >> 5)) ^ (row & 7))];
  } else if constexpr (sizeof(T) == 2) {
    const int q = lane >> 4, i = lane & 15;
    const int k = ks * 16 + (q >> 1) * 8 + (i >> 2);
    const int unit = (d0 >> 3) + (q & 1) * 2 + ((i & 3) >> 1);
    const int byte = (from + k * L::kPerRow + (unit ^ L::swizzle(k))) * 16 + (i & 1) * 8;
    using P = __attribute__((address_space(3))) s16x4*;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)((const char*)s + byte));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)((const char*)s + (byte + 4 * L::kPerRow * 16)));   // 4 rows on, which are permuted alike
    struct { s16x4 a, b; } both{lo, hi};
    f.v = __builtin_bit_cast(u32x4, both);
  } else {
    const int d = d0 + (lane & 31);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = (ks * 2 + (lane >> 5)) * 4 + j;
      f.v[j] = ((const uint32_t*)s)[(from + k * L::kPerRow + ((d >> 2) ^ L::swizzle(k))) * 4 + (d & 3)];
    }
  }
  return f;
}

// One operand's way into LDS: what a thread loads of each step's tile, 16 bytes at a time.
template <typename T, int BD, bool KC, int WAVES, bool ALIGNED, bool PAIRED>
struct Loader {
  using L = Tile<T, BD, KC>;
  static constexpr int E = L::E, BK = L::BK, N = L::kUnits / 64 / WAVES;   // loads of a wavefront in a step
  static constexpr int kApart = KC ? 8 : 64 / L::kPerRow;                  // rows between them
  const char* base;      // the tile's first element at the next step
  uint64_t left;         // bytes from there to the operand's last row's end
  uint64_t stride;       // bytes from step to step
  uint32_t off[N];       // of this lane's units
  uint32_t k;            // of its first unit, within a step
  uint32_t ld, d, room;  // elements between rows; the first unit's row or column of the tile, and how many the product has from the tile on

  // PAIRED: rows of the tile are 32 of one matrix and 32 of another in turn, and this wavefront's are all of one.
  __device__ __forceinline__ void start(const GemmOperand& o, uint32_t w, uint32_t lead, uint32_t dim, uint32_t K, int wave, int lane) {
    ld = (uint32_t)o.ld;
    base = (const char*)((const T*)o.p + (int64_t)w * o.worker + (KC ? (int64_t)lead * o.ld : (int64_t)lead));
    // Rows are whole units where they are loaded as such: the caller's by the rule for that variant, the library's own by their padding.
    const uint64_t last = KC ? (uint64_t)(dim - 1 - lead) * o.ld + (K + E - 1) / E * E : (uint64_t)(K - 1) * o.ld + ((dim + E - 1) / E * E - lead);
    // A tile may lie wholly in the padding behind the last column: it loads nothing.
    room = lead < dim ? dim - lead : 0;
    left = room ? last * sizeof(T) : 0;
    stride = (KC ? (uint64_t)BK : (uint64_t)BK * o.ld) * sizeof(T);
    const int place = wave * N * 64 + lane, row = place / L::kPerRow, unit = (place % L::kPerRow) ^ L::swizzle(row);
    if constexpr (KC) { d = PAIRED ? (row >> 6) * 32 + (row & 31) : row; k = unit * E; }
    else { d = unit * E; k = row; }
    if constexpr (ALIGNED) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if constexpr (KC) {
          off[j] = ((d + j * kApart) * ld + k) * (uint32_t)sizeof(T);         // rows beyond the last one lie beyond `left`
        } else {
          const int r = row + j * kApart, c = (place % L::kPerRow ^ L::swizzle(r)) * E;
          off[j] = (uint32_t)c < room ? (r * ld + c) * (uint32_t)sizeof(T) : kOut;
        }
      }
    }
  }

  // The step whose first k is K - k_left; zeros where that is none.
  __device__ __forceinline__ void fetch(int k_left, u32x4* lds, u32x4* held, int wave, int lane) {
    if constexpr (ALIGNED) {
      const uint32_t bytes = (uint32_t)min(left, (uint64_t)0x7FFFFFF0u);
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)bytes, 0x00020000);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const uint32_t none = (int)(KC ? k : k + j * kApart) >= k_left ? kOut : 0;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (wave * N + j) * 64), 16, (int)(off[j] | none), 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int place = (wave * N + j) * 64 + lane, row = place / L::kPerRow, unit = (place % L::kPerRow) ^ L::swizzle(row);
        const uint32_t dj = KC ? d + j * kApart : unit * E, kj = KC ? k : row;
        u32x4 v = {0, 0, 0, 0};
        if (dj < room && (int)kj < k_left) {
          const T* p = (const T*)base + (KC ? (int64_t)dj * ld + kj : (int64_t)kj * ld + dj);
          const uint32_t n = KC ? k_left - kj : room - dj;
          if (n >= E) {
            __builtin_memcpy(&v, __builtin_assume_aligned(p, sizeof(T)), 16);
          } else {
            T e[E];
#pragma unroll
            for (int i = 0; i < E; ++i) e[i] = i < (int)n ? p[i] : (T)0.f;
            __builtin_memcpy(&v, e, 16);
          }
        }
        held[j] = v;
      }
    }
    base += stride;
    left -= min(left, stride);
  }

  __device__ __forceinline__ void skip(uint32_t steps) {
    base += steps * stride;
    left -= min(left, steps * stride);
  }

  __device__ __forceinline__ void put(u32x4* lds, const u32x4* held, int wave, int lane) const {
    if constexpr (!ALIGNED) {
#pragma unroll
      for (int j = 0; j < N; ++j) lds[(wave * N + j) * 64 + lane] = held[j];
    }
  }
};

// This wavefront's loads into LDS have arrived and its reads of LDS are done; then the workgroup meets.
__device__ __forceinline__ void wait_and_meet() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(7 << 4);   // vmcnt and lgkmcnt 0
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Workgroups go to the eight XCDs in turn.  Each XCD gets a contiguous part of the tiles' order, so that what they share lies in its own L2.
__device__ __forceinline__ uint32_t place_by_xcd(uint32_t first) {
  const uint32_t x = blockIdx.x & 7, each = gridDim.x >> 3, more = gridDim.x & 7;
  return first + x * each + min(x, more) + (blockIdx.x >> 3);
}

}  // namespace evg
