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
};

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

// The largest tile of which there are enough to occupy the chip.
GemmTile choose_tile(GemmOp op, const GemmArgs& g, uint32_t n, uint32_t share, bool aligned, uint32_t type) {
  if ((op == GEMM_GATED || op == GEMM_DOWN) && g.M <= kMostRows) return TILE_ROWS;
  auto count = [&](uint64_t bm, uint64_t bn) { return ((g.M + bm - 1) / bm) * ((n + bn / share - 1) / (bn / share)) * g.workers * g.parts; };
  if (aligned && type != EVG_F32 && count(256, 256) >= 200) return TILE_256;
  if (count(128, 128) >= 256) return TILE_128;
  return TILE_64;
}

hipError_t product(const evg_ffn* c, GemmOp op, bool aligned, GemmArgs& g) {
  g.workers = c->cfg.workers;
  const bool tanh_form = c->cfg.activation == EVG_ACT_GELU_TANH;   // 2 sqrt(2 / pi) (x + 0.044715 x^3)
  g.activation = {tanh_form ? 1.5957691216057308f : 1.f, tanh_form ? 1.5957691216057308f * 0.044715f : 0.f, c->cfg.activation == EVG_ACT_RELU,
                  c->cfg.activation == EVG_ACT_GELU};
  g.pitch = c->pitch;
  const bool padded = op == GEMM_GATED || op == GEMM_GATED_BWD;
  const GemmTile tile = choose_tile(op, g, padded ? g.pitch : g.N, op == GEMM_GATED ? 2 : 1, aligned, c->cfg.type);
  if (c->cfg.type == EVG_F32) return launch_gemm<float>(op, tile, aligned, g, c->stream);
  if (c->cfg.type == EVG_F16) return launch_gemm<half_t>(op, tile, aligned, g, c->stream);
  return launch_gemm<bf16_t>(op, tile, aligned, g, c->stream);
}

// What every call is handed: x, dy and y are rows x D, w_gate and w_up F x D, w_down D x F.
struct Shape { uint32_t W, rows, D, F, type; };

evg_status check_weights(const Shape& s, const evg_mat* x, const evg_mat* w_gate, const evg_mat* w_up, const evg_mat* w_down) {
  evg_status st;
  if ((st = check_mat(x, s.W, s.rows, s.D, s.type, false, "x")) != EVG_OK) return st;
  if ((st = check_mat(w_gate, s.W, s.F, s.D, s.type, false, "w_gate")) != EVG_OK) return st;
  if ((st = check_mat(w_up, s.W, s.F, s.D, s.type, false, "w_up")) != EVG_OK) return st;
  return check_mat(w_down, s.W, s.D, s.F, s.type, false, "w_down");
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
  if (cfg->max_rows > 0x7FFFFF00u) return fail(EVG_ERR_INVALID, "max_rows is out of range");
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
  hipError_t e = hipMalloc(&c->hidden, one ? one : 16);
  if (e == hipSuccess && cfg->train) e = hipMalloc(&c->grads, one ? 2 * one : 16);
  if (e != hipSuccess) {
    if (c->hidden) (void)hipFree(c->hidden);
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
  if ((st = check_mat(y, s.W, rows, s.D, s.type, true, "y")) != EVG_OK) return st;
  if (saved && (st = check_saved(c, saved, rows)) != EVG_OK) return st;
  const Span ins[] = {mat_span(x, s.W, rows, s.D, s.type, "x"), mat_span(w_gate, s.W, s.F, s.D, s.type, "w_gate"),
                      mat_span(w_up, s.W, s.F, s.D, s.type, "w_up"), mat_span(w_down, s.W, s.D, s.F, s.type, "w_down")};
  const Span outs[] = {mat_span(y, s.W, rows, s.D, s.type, "y"), saved_span(c, saved, rows)};
  if ((st = check_apart(outs, 2, ins, 4)) != EVG_OK) return st;
  if (!rows) return EVG_OK;
  const uint32_t e = type_bytes(s.type);
  const uint64_t proj = (uint64_t)s.W * proj_rows(rows) * 2 * c->pitch;
  const GemmOperand h{saved ? (char*)saved + proj * sizeof(float) : c->hidden, (int64_t)rows * c->pitch, (int64_t)c->pitch};

  GemmArgs g{};
  g.a[0] = operand(*x, s.W, rows, s.D);
  g.b[0] = operand(*w_gate, s.W, s.F, s.D);
  g.b[1] = operand(*w_up, s.W, s.F, s.D);
  g.c[0] = h;
  g.M = rows, g.N = s.F, g.K = s.D, g.parts = 1;
  g.proj = (float*)saved;
  g.proj_worker = proj_rows(rows) * 2 * c->pitch;
  HIP_TRY(product(c, GEMM_GATED, whole_units(g.a[0], s.D, e) && whole_units(g.b[0], s.D, e) && whole_units(g.b[1], s.D, e), g));

  g = GemmArgs{};
  g.a[0] = h;
  g.b[0] = operand(*w_down, s.W, s.D, s.F);
  g.c[0] = operand(*y, s.W, rows, s.D);
  g.M = rows, g.N = s.D, g.K = s.F, g.parts = 1;
  HIP_TRY(product(c, GEMM_DOWN, whole_units(g.b[0], s.F, e), g));
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
  if ((st = check_mat(dy, s.W, rows, s.D, s.type, false, "dy")) != EVG_OK) return st;
  if ((st = check_saved(c, saved, rows)) != EVG_OK) return st;
  const bool has[4] = {dx && dx->p, dw_gate && dw_gate->p, dw_up && dw_up->p, dw_down && dw_down->p};
  if (has[0] && (st = check_mat(dx, s.W, rows, s.D, s.type, true, "dx")) != EVG_OK) return st;
  if (has[1] && (st = check_mat(dw_gate, s.W, s.F, s.D, s.type, true, "dw_gate")) != EVG_OK) return st;
  if (has[2] && (st = check_mat(dw_up, s.W, s.F, s.D, s.type, true, "dw_up")) != EVG_OK) return st;
  if (has[3] && (st = check_mat(dw_down, s.W, s.D, s.F, s.type, true, "dw_down")) != EVG_OK) return st;
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
  const GemmOperand X = operand(*x, s.W, rows, s.D), DY = operand(*dy, s.W, rows, s.D);
  GemmArgs g{};
  if (rows && (has[0] || has[1] || has[2])) {
    g.a[0] = DY;
    g.b[0] = operand(*w_down, s.W, s.D, s.F);
    g.c[0] = dg;
    g.M = rows, g.N = s.F, g.K = s.D, g.parts = 1;
    g.proj = (float*)saved;
    g.proj_worker = proj_rows(rows) * 2 * c->pitch;
    HIP_TRY(product(c, GEMM_GATED_BWD, whole_units(g.a[0], s.D, e) && whole_units(g.b[0], s.F, e), g));
  }
  if (rows && has[0]) {
    g = GemmArgs{};
    g.a[0] = dg, g.a[1] = du;
    g.b[0] = operand(*w_gate, s.W, s.F, s.D), g.b[1] = operand(*w_up, s.W, s.F, s.D);
    g.c[0] = operand(*dx, s.W, rows, s.D);
    g.M = rows, g.N = s.D, g.K = s.F, g.parts = 1;
    HIP_TRY(product(c, GEMM_INPUT, whole_units(g.b[0], s.D, e) && whole_units(g.b[1], s.D, e), g));
  }
  if (has[1] || has[2]) {
    g = GemmArgs{};
    uint32_t n = 0;
    if (has[1]) { g.a[n] = dg; g.c[n++] = operand(*dw_gate, s.W, s.F, s.D); }
    if (has[2]) { g.a[n] = du; g.c[n++] = operand(*dw_up, s.W, s.F, s.D); }
    g.b[0] = X;
    g.M = s.F, g.N = s.D, g.K = rows, g.parts = n;
    HIP_TRY(product(c, GEMM_WEIGHT, whole_units(X, s.D, e), g));
  }
  if (has[3]) {
    g = GemmArgs{};
    g.a[0] = DY;
    g.b[0] = h;
    g.c[0] = operand(*dw_down, s.W, s.D, s.F);
    g.M = s.D, g.N = s.F, g.K = rows, g.parts = 1;
    HIP_TRY(product(c, GEMM_WEIGHT, whole_units(DY, s.D, e), g));
  }
  return EVG_OK;
}

evg_status evg_ffn_destroy(evg_ffn* c) {
  if (!c) return EVG_OK;
  hipError_t e = hipStreamSynchronize(c->stream);
  for (void* p : {c->hidden, c->grads})
    if (p) { const hipError_t f = hipFree(p); if (e == hipSuccess) e = f; }
  delete c;
  HIP_TRY(e);
  return EVG_OK;
}

}  // extern "C"
