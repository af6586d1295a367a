// Host side of the gated feed-forward block (include/evg_nn.h, evg_ffn_*).
//
// For each worker:  g = x Wg^T, u = x Wu^T, h = act(g) * u, y = h Wd^T.  Backward, from dy:
//     dh = dy Wd,  dg = dh * u * act'(g),  du = dh * act(g)            one product, the rest in its epilogue
//     dx = dg Wg + du Wu                                               one product over both
//     dWg = dg^T x, dWu = du^T x                                       one launch
//     dWd = dy^T h
// g and u are kept in 32 bits: rounded to 16 they would add their error to that of dg and du, which the matrix cores take in
// 16 bits, and to make them anew would be two more products.  dg and du, as h, are rounded once, to the tensors' type.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "ffn_internal.h"
#include "nn_device.h"
#include "nn_host.h"

using namespace evg;

struct evg_ffn {
  evg_ffn_config cfg{};
  hipStream_t stream = nullptr;
  uint32_t pitch = 0;      // hidden, padded to 64: columns beyond `hidden` are 0
  void* hidden = nullptr;  // h where nothing is saved: [workers][max_rows][pitch]
  void* grads = nullptr;   // dg and du: [workers][max_rows][2][pitch]
  // Where a width is no whole number of 16-byte units: room for copies with rows that are (null: not needed).
  uint32_t width_pitch = 0;
  void *x = nullptr, *dy = nullptr, *w_gate = nullptr, *w_up = nullptr, *w_down = nullptr;
};

namespace evg {
namespace {

// A wavefront copies a row, 16 bytes to a lane.  Reads need no alignment beyond their elements'.
template <typename T>
__global__ __launch_bounds__(256) void k_ffn_pack(PackArgs a) {
  constexpr int E = 16 / sizeof(T);
  const uint64_t id = ((uint64_t)a.first + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (id >= a.lines) return;
  uint32_t k = 0;
  while (k + 1 < a.count && id >= a.one[k + 1].first) ++k;
  const PackOne& o = a.one[k];
  const uint64_t line = id - o.first;
  const T* from = (const T*)o.from.p + (int64_t)(line / o.rows) * o.from.worker + (int64_t)(line % o.rows) * o.from.ld;
  T* to = (T*)o.to + line * o.pitch;
#pragma unroll 4
  for (uint32_t c = (threadIdx.x & 63) * E; c < o.cols; c += 64 * E) {
    Pack<T, E> v;
    const int n = (int)(o.cols - c);
    if (n >= E) {
      v = *reinterpret_cast<const Pack<T, E>*>(from + c);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) v.v[i] = i < n ? from[c + i] : (T)0.f;
    }
    *reinterpret_cast<uint4*>(to + c) = __builtin_bit_cast(uint4, v);
  }
}

}  // namespace

hipError_t launch_pack(uint32_t type, PackArgs a, hipStream_t s) {
  if (!a.lines) return hipSuccess;
  const uint64_t groups = (a.lines + 3) / 4;
  if (groups > 0x7FFFFFFFull) return hipErrorInvalidValue;
  launch_pieces(groups, 256, [&](uint32_t first, uint32_t grid) {
    a.first = first;
    if (type == EVG_F32) k_ffn_pack<float><<<grid, 256, 0, s>>>(a);
    else k_ffn_pack<half_t><<<grid, 256, 0, s>>>(a);   // bits
  });
  return hipGetLastError();
}

}  // namespace evg

namespace {

// Rows of the projections that are kept: whole accumulators of 32.
uint64_t proj_rows(uint32_t rows) { return ((uint64_t)rows + 31) / 32 * 32; }

// Can a product read it by 16-byte units?  Addresses, strides and rows are whole units, and a tile's rows lie within 31 bits.
bool whole_units(const GemmOperand& o, uint64_t cols, uint32_t bytes) {
  const uint64_t e = 16 / bytes;
  return (uintptr_t)o.p % 16 == 0 && o.ld % e == 0 && o.worker % e == 0 && cols % e == 0 && (uint64_t)o.ld * bytes < (1u << 22);
}

GemmOperand operand(const evg_mat& m, uint32_t workers, uint64_t rows, uint64_t cols) {
  return {m.p, workers > 1 ? m.worker : 0, rows > 1 ? m.row : (int64_t)cols};
}

hipError_t product(const evg_ffn* c, GemmOp op, bool aligned, GemmArgs& g) {
  g.workers = c->cfg.workers;
  const bool tanh_form = c->cfg.activation == EVG_ACT_GELU_TANH;   // 2 sqrt(2 / pi) (x + 0.044715 x^3)
  g.activation = {tanh_form ? 1.5957691216057308f : 1.f, tanh_form ? 1.5957691216057308f * 0.044715f : 0.f, c->cfg.activation == EVG_ACT_RELU,
                  c->cfg.activation == EVG_ACT_GELU};
  g.pitch = c->pitch;
  const bool padded = op == GEMM_GATED || op == GEMM_GATED_BWD;
  const GemmTile tile = choose_tile(op, {g.M, padded ? g.pitch : g.N, g.K, g.workers, g.parts}, aligned, c->cfg.type == EVG_F32);
  if (c->cfg.type == EVG_F32) return launch_gemm<float>(op, tile, aligned, g, c->stream);
  if (c->cfg.type == EVG_F16) return launch_gemm<half_t>(op, tile, aligned, g, c->stream);
  return launch_gemm<bf16_t>(op, tile, aligned, g, c->stream);
}

// Collects the operands that need whole-unit copies.
struct Packer {
  const evg_ffn* c;
  PackArgs a{};
  explicit Packer(const evg_ffn* ctx) : c(ctx) {}
  // The operand, or its copy to be: products read the latter by whole units.  There is room where the width is odd; what only begins beside a unit stays as
  // it is (bf16, forward and backward, 8 bytes beside one: 1024 tokens 1024 x 4096 138 -> 213 us, 2048 tokens 2048 x 8192 688 -> 1205).
  GemmOperand take(const GemmOperand& o, void* room, uint32_t rows, uint32_t cols, uint32_t pitch) {
    if (!room || whole_units(o, cols, type_bytes(c->cfg.type))) return o;
    a.one[a.count++] = {o, room, rows, cols, pitch, a.lines};
    a.lines += (uint64_t)c->cfg.workers * rows;
    return {room, (int64_t)rows * pitch, (int64_t)pitch};
  }
  // Of an operand after take: by whole units?
  bool whole(const GemmOperand& o, uint32_t cols) const {
    for (uint32_t i = 0; i < a.count; ++i)
      if (a.one[i].to == o.p) return true;
    return whole_units(o, cols, type_bytes(c->cfg.type));
  }
  hipError_t launch() const { return launch_pack(c->cfg.type, a, c->stream); }
};

// What every call is handed: x, dy and y are rows x D, w_gate and w_up F x D, w_down D x F.
struct Shape { uint32_t W, rows, D, F, type; };

// As check_mat, and rows near enough for 31 bits.
evg_status check_operand(const evg_mat* m, const Shape& s, uint64_t rows, uint64_t cols, bool written, const char* what) {
  const evg_status st = check_mat(m, s.W, rows, cols, s.type, written, what);
  if (st == EVG_OK && rows > 1 && m->row > 0x7FFFFFFF) return fail(EVG_ERR_INVALID, "%s: rows more than 2^31 elements apart", what);
  return st;
}

evg_status check_weights(const Shape& s, const evg_mat* x, const evg_mat* w_gate, const evg_mat* w_up, const evg_mat* w_down) {
  evg_status st;
  if ((st = check_operand(x, s, s.rows, s.D, false, "x")) != EVG_OK) return st;
  if ((st = check_operand(w_gate, s, s.F, s.D, false, "w_gate")) != EVG_OK) return st;
  if ((st = check_operand(w_up, s, s.F, s.D, false, "w_up")) != EVG_OK) return st;
  return check_operand(w_down, s, s.D, s.F, false, "w_down");
}

evg_status check_saved(const evg_ffn* c, const void* saved, uint32_t rows) {
  if ((uintptr_t)saved % 16) return fail(EVG_ERR_ALIGN, "saved is not 16-byte aligned");
  return rows ? check_device_array(saved, evg_ffn_saved_bytes(c, rows), "saved") : EVG_OK;
}

Span saved_span(const evg_ffn* c, const void* saved, uint32_t rows) {
  Span s;
  s.what = "saved";
  s.begin = (uintptr_t)saved;
  s.end = s.begin + (saved ? evg_ffn_saved_bytes(c, rows) : 0);
  return s;
}

}  // namespace

extern "C" {

evg_status evg_ffn_init(evg_ffn** out, const evg_ffn_config* cfg, void* hip_stream) {
  if (!out || !cfg) return fail(EVG_ERR_INVALID, "out and cfg must be non-NULL");
  *out = nullptr;
  if (cfg->workers < 1 || cfg->workers > 65535) return fail(EVG_ERR_INVALID, "workers must be 1 .. 65535");
  if (cfg->width < 1 || cfg->width > (1u << 20) || cfg->hidden < 1 || cfg->hidden > (1u << 20)) return fail(EVG_ERR_INVALID, "width and hidden must be 1 .. 2^20");
  if (cfg->max_rows > 0x7FFF0000u) return fail(EVG_ERR_INVALID, "max_rows is out of range");
  evg_status st;
  if ((st = check_type(cfg->type, "type")) != EVG_OK) return st;
  if (cfg->activation > EVG_ACT_RELU) return fail(EVG_ERR_INVALID, "activation must be one of EVG_ACT_*");
  evg_ffn* c = new (std::nothrow) evg_ffn();
  if (!c) return fail(EVG_ERR_OOM, "host allocation failed");
  c->cfg = *cfg;
  c->stream = static_cast<hipStream_t>(hip_stream);
  c->pitch = (cfg->hidden + 63) / 64 * 64;
  const uint64_t one = (uint64_t)cfg->workers * cfg->max_rows * c->pitch * type_bytes(cfg->type);   // < 2^71 / 2^8: checked by hipMalloc
  if ((unsigned __int128)cfg->workers * cfg->max_rows * c->pitch >> 56) {
    delete c;
    return fail(EVG_ERR_INVALID, "workers, max_rows and hidden together are out of range");
  }
  const uint32_t bytes = type_bytes(cfg->type), unit = 16 / bytes;
  c->width_pitch = (cfg->width + 63) / 64 * 64;
  const uint64_t tokens = (uint64_t)cfg->workers * cfg->max_rows * c->width_pitch * bytes, up = (uint64_t)cfg->workers * cfg->hidden * c->width_pitch * bytes,
                 down = (uint64_t)cfg->workers * cfg->width * c->pitch * bytes;
  const bool odd_width = cfg->width % unit, odd_hidden = cfg->hidden % unit, copies = cfg->max_rows > kMostRows;
  struct { void** p; uint64_t bytes; bool need; } rooms[] = {
      {&c->hidden, one, true}, {&c->grads, 2 * one, cfg->train != 0}, {&c->x, tokens, copies && odd_width}, {&c->dy, tokens, copies && odd_width && cfg->train},
      {&c->w_gate, up, copies && odd_width}, {&c->w_up, up, copies && odd_width}, {&c->w_down, down, copies && odd_hidden}};
  hipError_t e = hipSuccess;
  for (auto& r : rooms)
    if (r.need && e == hipSuccess) e = hipMalloc(r.p, r.bytes ? r.bytes : 16);
  if (e != hipSuccess) {
    for (auto& r : rooms)
      if (*r.p) (void)hipFree(*r.p);
    delete c;
    return fail(e == hipErrorOutOfMemory ? EVG_ERR_OOM : EVG_ERR_HIP, "workspace: %s", hipGetErrorString(e));
  }
  *out = c;
  return EVG_OK;
}

uint64_t evg_ffn_saved_bytes(const evg_ffn* c, uint32_t rows) {
  if (!c) return 0;
  return (uint64_t)c->cfg.workers * c->pitch * (proj_rows(rows) * 2 * sizeof(float) + (uint64_t)rows * type_bytes(c->cfg.type));
}

evg_status evg_ffn_forward(evg_ffn* c, uint32_t rows, const evg_mat* x, const evg_mat* w_gate, const evg_mat* w_up,
                           const evg_mat* w_down, const evg_mat* y, void* saved) {
  if (!c) return fail(EVG_ERR_INVALID, "context must be non-NULL");
  const Shape s{c->cfg.workers, rows, c->cfg.width, c->cfg.hidden, c->cfg.type};
  if (rows > c->cfg.max_rows) return fail(EVG_ERR_INVALID, "rows exceeds the context's max_rows");
  evg_status st;
  if ((st = check_weights(s, x, w_gate, w_up, w_down)) != EVG_OK) return st;
  if ((st = check_operand(y, s, rows, s.D, true, "y")) != EVG_OK) return st;
  if (saved && (st = check_saved(c, saved, rows)) != EVG_OK) return st;
  const Span ins[] = {mat_span(x, s.W, rows, s.D, s.type, "x"), mat_span(w_gate, s.W, s.F, s.D, s.type, "w_gate"),
                      mat_span(w_up, s.W, s.F, s.D, s.type, "w_up"), mat_span(w_down, s.W, s.D, s.F, s.type, "w_down")};
  const Span outs[] = {mat_span(y, s.W, rows, s.D, s.type, "y"), saved_span(c, saved, rows)};
  if ((st = check_apart(outs, 2, ins, 4)) != EVG_OK) return st;
  if (!rows) return EVG_OK;
  const uint64_t proj = (uint64_t)s.W * proj_rows(rows) * 2 * c->pitch;
  const GemmOperand h{saved ? (char*)saved + proj * sizeof(float) : c->hidden, (int64_t)rows * c->pitch, (int64_t)c->pitch};

  // Few tokens are multiplied straight from the tensors, whatever their alignment.
  const bool copies = rows > kMostRows;
  Packer p(c);
  const GemmOperand X = p.take(operand(*x, s.W, rows, s.D), copies ? c->x : nullptr, rows, s.D, c->width_pitch);
  const GemmOperand WG = p.take(operand(*w_gate, s.W, s.F, s.D), copies ? c->w_gate : nullptr, s.F, s.D, c->width_pitch);
  const GemmOperand WU = p.take(operand(*w_up, s.W, s.F, s.D), copies ? c->w_up : nullptr, s.F, s.D, c->width_pitch);
  const GemmOperand WD = p.take(operand(*w_down, s.W, s.D, s.F), copies ? c->w_down : nullptr, s.D, s.F, c->pitch);
  HIP_TRY(p.launch());
  GemmArgs g{};
  g.a[0] = X;
  g.b[0] = WG;
  g.b[1] = WU;
  g.c[0] = h;
  g.M = rows, g.N = s.F, g.K = s.D, g.parts = 1;
  g.proj = (float*)saved;
  g.proj_worker = proj_rows(rows) * 2 * c->pitch;
  HIP_TRY(product(c, GEMM_GATED, p.whole(X, s.D) && p.whole(WG, s.D) && p.whole(WU, s.D), g));

  g = GemmArgs{};
  g.a[0] = h;
  g.b[0] = WD;
  g.c[0] = operand(*y, s.W, rows, s.D);
  g.M = rows, g.N = s.D, g.K = s.F, g.parts = 1;
  HIP_TRY(product(c, GEMM_DOWN, p.whole(WD, s.F), g));
  return EVG_OK;
}

evg_status evg_ffn_backward(evg_ffn* c, uint32_t rows, const evg_mat* dy, const evg_mat* x, const evg_mat* w_gate,
                            const evg_mat* w_up, const evg_mat* w_down, const void* saved, const evg_mat* dx,
                            const evg_mat* dw_gate, const evg_mat* dw_up, const evg_mat* dw_down) {
  if (!c) return fail(EVG_ERR_INVALID, "context must be non-NULL");
  if (!c->cfg.train) return fail(EVG_ERR_STATE, "the context was made without train");
  const Shape s{c->cfg.workers, rows, c->cfg.width, c->cfg.hidden, c->cfg.type};
  if (rows > c->cfg.max_rows) return fail(EVG_ERR_INVALID, "rows exceeds the context's max_rows");
  if (!saved && rows) return fail(EVG_ERR_INVALID, "saved must be given");
  evg_status st;
  if ((st = check_weights(s, x, w_gate, w_up, w_down)) != EVG_OK) return st;
  if ((st = check_operand(dy, s, rows, s.D, false, "dy")) != EVG_OK) return st;
  if ((st = check_saved(c, saved, rows)) != EVG_OK) return st;
  const bool has[4] = {dx && dx->p, dw_gate && dw_gate->p, dw_up && dw_up->p, dw_down && dw_down->p};
  if (has[0] && (st = check_operand(dx, s, rows, s.D, true, "dx")) != EVG_OK) return st;
  if (has[1] && (st = check_operand(dw_gate, s, s.F, s.D, true, "dw_gate")) != EVG_OK) return st;
  if (has[2] && (st = check_operand(dw_up, s, s.F, s.D, true, "dw_up")) != EVG_OK) return st;
  if (has[3] && (st = check_operand(dw_down, s, s.D, s.F, true, "dw_down")) != EVG_OK) return st;
  const Span ins[] = {mat_span(x, s.W, rows, s.D, s.type, "x"), mat_span(w_gate, s.W, s.F, s.D, s.type, "w_gate"),
                      mat_span(w_up, s.W, s.F, s.D, s.type, "w_up"), mat_span(w_down, s.W, s.D, s.F, s.type, "w_down"),
                      mat_span(dy, s.W, rows, s.D, s.type, "dy"), saved_span(c, saved, rows)};
  const Span outs[] = {mat_span(dx, s.W, rows, s.D, s.type, "dx"), mat_span(dw_gate, s.W, s.F, s.D, s.type, "dw_gate"),
                       mat_span(dw_up, s.W, s.F, s.D, s.type, "dw_up"), mat_span(dw_down, s.W, s.D, s.F, s.type, "dw_down")};
  if ((st = check_apart(outs, 4, ins, 6)) != EVG_OK) return st;
  const uint32_t e = type_bytes(s.type);
  const uint64_t proj = (uint64_t)s.W * proj_rows(rows) * 2 * c->pitch;
  const int64_t two = 2 * (int64_t)c->pitch;
  const GemmOperand h{(const char*)saved + proj * sizeof(float), (int64_t)rows * c->pitch, (int64_t)c->pitch};
  const GemmOperand dg{c->grads, (int64_t)rows * two, two}, du{(const char*)c->grads + (uint64_t)c->pitch * e, (int64_t)rows * two, two};
  // Few tokens: copies of the weights would cost more than reading them element by element where they are cut.
  const bool copies = rows > kMostRows, up = has[0] || has[1] || has[2];
  Packer p(c);
  auto take = [&](bool need, const GemmOperand& o, void* room, uint32_t r, uint32_t cols, uint32_t pitch) { return p.take(o, need && copies ? room : nullptr, r, cols, pitch); };
  const GemmOperand X = take(has[1] || has[2], operand(*x, s.W, rows, s.D), c->x, rows, s.D, c->width_pitch);
  const GemmOperand DY = take(true, operand(*dy, s.W, rows, s.D), c->dy, rows, s.D, c->width_pitch);
  const GemmOperand WD = take(up, operand(*w_down, s.W, s.D, s.F), c->w_down, s.D, s.F, c->pitch);
  HIP_TRY(p.launch());
  GemmArgs g{};
  if (rows && up) {
    g.a[0] = DY;
    g.b[0] = WD;
    g.c[0] = dg;
    g.M = rows, g.N = s.F, g.K = s.D, g.parts = 1;
    g.proj = (float*)saved;
    g.proj_worker = proj_rows(rows) * 2 * c->pitch;
    HIP_TRY(product(c, GEMM_GATED_BWD, p.whole(DY, s.D) && p.whole(WD, s.F), g));
  }
  if (rows && has[0]) {
    Packer pw(c);
    const GemmOperand WG = pw.take(operand(*w_gate, s.W, s.F, s.D), copies ? c->w_gate : nullptr, s.F, s.D, c->width_pitch);
    const GemmOperand WU = pw.take(operand(*w_up, s.W, s.F, s.D), copies ? c->w_up : nullptr, s.F, s.D, c->width_pitch);
    HIP_TRY(pw.launch());
    g = GemmArgs{};
    g.a[0] = dg, g.a[1] = du;
    g.b[0] = WG, g.b[1] = WU;
    g.c[0] = operand(*dx, s.W, rows, s.D);
    g.M = rows, g.N = s.D, g.K = s.F, g.parts = 1;
    HIP_TRY(product(c, GEMM_INPUT, pw.whole(WG, s.D) && pw.whole(WU, s.D), g));
  }
  if (has[1] || has[2]) {
    g = GemmArgs{};
    uint32_t n = 0;
    if (has[1]) { g.a[n] = dg; g.c[n++] = operand(*dw_gate, s.W, s.F, s.D); }
    if (has[2]) { g.a[n] = du; g.c[n++] = operand(*dw_up, s.W, s.F, s.D); }
    g.b[0] = X;
    g.M = s.F, g.N = s.D, g.K = rows, g.parts = n;
    HIP_TRY(product(c, GEMM_WEIGHT, p.whole(X, s.D), g));
  }
  if (has[3]) {
    g = GemmArgs{};
    g.a[0] = DY;
    g.b[0] = h;
    g.c[0] = operand(*dw_down, s.W, s.D, s.F);
    g.M = s.D, g.N = s.F, g.K = rows, g.parts = 1;
    HIP_TRY(product(c, GEMM_WEIGHT, p.whole(DY, s.D), g));
  }
  return EVG_OK;
}

evg_status evg_ffn_destroy(evg_ffn* c) {
  if (!c) return EVG_OK;
  hipError_t e = hipStreamSynchronize(c->stream);
  for (void* p : {c->hidden, c->grads, c->x, c->dy, c->w_gate, c->w_up, c->w_down})
    if (p) { const hipError_t f = hipFree(p); if (e == hipSuccess) e = f; }
  delete c;
  HIP_TRY(e);
  return EVG_OK;
}

}  // extern "C"
