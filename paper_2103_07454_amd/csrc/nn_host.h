// Checks that the host sides of the operators of include/evg_nn.h share.
#pragma once
#include <stdint.h>

#include "../../include/evg_nn.h"
#include "evg_host.h"
#include "launch_pieces.h"

namespace evg {

inline uint32_t type_bytes(uint32_t type) { return type == EVG_F32 ? 4u : 2u; }

inline evg_status check_type(uint32_t type, const char* what) {
  if (type != EVG_F32 && type != EVG_F16 && type != EVG_BF16) return fail(EVG_ERR_INVALID, "%s must be EVG_F32, EVG_F16 or EVG_BF16", what);
  return EVG_OK;
}

// Elements from a matrix's first to its last one's end, 0 if there are none; false where that does not fit 62 bits.
inline bool mat_extent(const evg_mat& m, uint32_t workers, uint64_t rows, uint64_t cols, uint64_t* out) {
  *out = 0;
  if (!workers || !rows || !cols) return true;
  const unsigned __int128 n = (unsigned __int128)(workers - 1) * (uint64_t)m.worker + (unsigned __int128)(rows - 1) * (uint64_t)m.row + cols;
  if (n >> 60) return false;
  *out = (uint64_t)n;
  return true;
}

// A matrix that a kernel is about to be handed.  A written one may not meet itself.
inline evg_status check_mat(const evg_mat* m, uint32_t workers, uint64_t rows, uint64_t cols, uint32_t type, bool written, const char* what) {
  if (!m || !m->p) return fail(EVG_ERR_INVALID, "%s must be given", what);
  const uint32_t e = type_bytes(type);
  if ((uintptr_t)m->p % e) return fail(EVG_ERR_ALIGN, "%s is not aligned to its elements", what);
  if ((workers > 1 && m->worker < 0) || (rows > 1 && m->row < 0)) return fail(EVG_ERR_INVALID, "%s has a negative stride", what);
  evg_mat one = *m;
  if (workers <= 1) one.worker = 0;
  if (rows <= 1) one.row = 0;
  uint64_t n = 0;
  if (!mat_extent(one, workers, rows, cols, &n)) return fail(EVG_ERR_INVALID, "%s: strides out of range", what);
  if (!n) return EVG_OK;
  if (written) {
    if (rows > 1 && (uint64_t)one.row < cols) return fail(EVG_ERR_INVALID, "%s is written and its rows overlap", what);
    const uint64_t slice = (rows - 1) * (uint64_t)one.row + cols, across = (uint64_t)(workers - 1) * (uint64_t)one.worker + cols;
    if (workers > 1 && (uint64_t)one.worker < slice && !((uint64_t)one.worker >= cols && (rows == 1 || (uint64_t)one.row >= across)))
      return fail(EVG_ERR_INVALID, "%s is written and its workers overlap", what);
  }
  return check_device_array(m->p, n * e, what);
}

// Where a matrix lies, in bytes.
struct Span {
  uintptr_t begin = 0, end = 0;   // equal: nothing
  uint64_t worker = 0, slice = 0, row = 0, cols = 0;   // strides, and the lengths of a worker's slice and of a row
  uint32_t workers = 0;
  const char* what = "";
};

inline Span mat_span(const evg_mat* m, uint32_t workers, uint64_t rows, uint64_t cols, uint32_t type, const char* what) {
  Span s;
  s.what = what;
  if (!m || !m->p || !rows) return s;
  evg_mat one = *m;
  if (workers <= 1) one.worker = 0;
  if (rows <= 1) one.row = (int64_t)cols;
  uint64_t n = 0;
  mat_extent(one, workers, rows, cols, &n);
  const uint64_t e = type_bytes(type);
  s.begin = (uintptr_t)m->p;
  s.end = s.begin + n * e;
  s.worker = (uint64_t)one.worker * e;
  s.row = (uint64_t)one.row * e;
  s.cols = cols * e;
  s.slice = (rows - 1) * s.row + s.cols;
  s.workers = workers;
  return s;
}

// Do pieces of `a` and `b` bytes, each repeated every `every` bytes, `apart` bytes from one another, stay clear of each other?
inline bool pieces_apart(uint64_t a, uint64_t b, uint64_t every, uintptr_t from, uintptr_t to) {
  if (!every) return false;
  const uint64_t apart = (to % every + every - from % every) % every;
  return a <= apart && apart + b <= every;
}

// May two matrices share a byte?  Tensors of one arena (workers equally far apart) and column blocks of one matrix (rows
// equally far apart) lie within each other's ends without meeting; other ways to interlace count as meeting.
inline bool spans_meet(const Span& a, const Span& b) {
  if (a.begin >= b.end || b.begin >= a.end) return false;
  if (a.workers > 1 && a.workers == b.workers && a.worker == b.worker && pieces_apart(a.slice, b.slice, a.worker, a.begin, b.begin)) return false;
  const bool in_step = a.row == b.row && a.row && (a.workers <= 1 || (a.worker % a.row == 0 && b.worker % a.row == 0));
  return !(in_step && pieces_apart(a.cols, b.cols, a.row, a.begin, b.begin));
}

// Outputs may meet neither each other nor an input, but for output `same`, which may lie exactly on input `on` (-1: none).
inline evg_status check_apart(const Span* out, int outs, const Span* in, int ins, int same = -1, int on = -1) {
  for (int i = 0; i < outs; ++i) {
    for (int j = 0; j < i; ++j)
      if (spans_meet(out[i], out[j])) return fail(EVG_ERR_INVALID, "%s overlaps %s", out[i].what, out[j].what);
    for (int j = 0; j < ins; ++j) {
      const bool one = i == same && j == on && out[i].begin == in[j].begin && out[i].worker == in[j].worker && out[i].row == in[j].row;
      if (!one && spans_meet(out[i], in[j])) return fail(EVG_ERR_INVALID, "%s overlaps %s", out[i].what, in[j].what);
    }
  }
  return EVG_OK;
}

}  // namespace evg
