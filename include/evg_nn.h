/* evg_nn.h -- C ABI of the operators that make, train and bound the gradients of feed-forward blocks for a ring's workers.
 *
 * Scope.  evg_step takes each worker's gradient (EVG_GRAD_BUFFER); these operators are what comes before it when the workers
 * train transformer feed-forward blocks: the norms on both sides of a block with its gate and residual scale (evg_blocknorm),
 * the gated feed-forward block (evg_ffn), both with their backward passes, and clipping by the global norm over a worker's
 * tensors (evg_clip).  All W workers of a ring, each with its own weights and tokens, go in one call; W = 1 is one model.
 *
 * Conventions: those of evg.h (statuses, evg_error_text, the current device, one stream for each context, calls on one
 * context must not overlap).  Calls other than init and destroy only enqueue work on the context's stream, call no
 * allocating or synchronising routine and record no memset, so they can be captured into a HIP graph; what a call reads is
 * read, and what it writes is written, in stream order.  Device memory that the library needs is allocated by init.
 * Nothing is carried from one call to the next.  Sums, norms and statistics are held in 32 bits or more whatever the tensors'
 * type; results are rounded once.  Orders of summation are fixed: the same call on the same values gives the same bits.
 */
#ifndef EVG_NN_H
#define EVG_NN_H

#include "evg.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { EVG_F32 = 0, EVG_F16 = 1, EVG_BF16 = 2 };

/* A DEVICE tensor of `workers` matrices: element (w, i, j) at p + w * worker + i * row + j, in elements of its type.  The
 * last axis has stride 1.  Rows may be further apart than they are long.  Those of a tensor that is only read may also be
 * closer, or one and the same (row or worker 0: broadcast); a written one's rows and workers may not overlap.  p == NULL:
 * absent.  Any alignment of p and any stride that its type allows. */
typedef struct {
  void* p;
  int64_t worker;
  int64_t row;
} evg_mat;

/* ---- clipping by the global norm --------------------------------------------------------------------------------
 * For each worker r, over all its tensors' elements (and nothing that lies between the tensors):
 *     norm[r] = |scale| * sqrt(sum of g^2)                                    (squares and sum in 64 bits)
 *     out     = g * (scale * min(1, max_norm / (norm[r] + eps)))              (the factor and the product in 32 bits)
 * where a quotient of two zeros or of two infinities is 1: what does not exceed the bound is not clipped.
 * Arenas are laid out as evg_step's: evg_padded_numel elements for each worker, tensors at evg_layer_offsets, here of
 * any of the types; padding is neither read nor written. */
enum {
  EVG_NONFINITE_PASS = 0, /* the formula as it stands: a NaN makes all of a worker's gradient NaN, an infinity (or a norm beyond 32
                             bits) makes the finite elements 0 and the infinite ones NaN where max_norm is finite            */
  EVG_NONFINITE_ZERO = 1  /* a worker whose norm is not finite gets zeros: it sits the step out                              */
};

typedef struct evg_clip evg_clip;

typedef struct {
  uint32_t P;                  /* workers, >= 1                                                         */
  uint32_t L;                  /* tensors of each worker, >= 1                                            */
  const uint64_t* layer_numel; /* [L], each 1 .. 2^31-8; read during init only                            */
  uint32_t grad_type;          /* EVG_F32, EVG_F16 or EVG_BF16                                            */
  uint32_t out_type;           /* grad_type or EVG_F32 (what evg_step takes)                              */
  float eps;                   /* >= 0                                                                    */
  uint32_t nonfinite;          /* EVG_NONFINITE_*                                                         */
} evg_clip_config;

evg_status evg_clip_init(evg_clip** out, const evg_clip_config* cfg, void* hip_stream);
/* grad, out: DEVICE arenas, 16-byte aligned (ones of 16-bit types: 8).  out may be grad where the types are the same (workers whose factor is 1
 * are then not written), else they may not overlap.  norm: DEVICE float[P], or NULL.  max_norm: >= 0 and not NaN (infinity: never clips);
 * scale: finite (it undoes a loss scale, or averages accumulated gradients). */
evg_status evg_clip_run(evg_clip* c, const void* grad, void* out, float max_norm, float scale, float* norm);
evg_status evg_clip_destroy(evg_clip* c);

/* ---- norms before and after a block, with its gate and residual scale ----------------------------------------------
 * For each row (token) of each worker, D = width:
 *     after      = N(branch; post, post_bias)    or branch itself without post
 *     residual'  = residual_scale * residual + branch_scale * gate * after
 *     normed     = N(residual'; pre, pre_bias)   (of the unrounded residual')
 * N(z; w, b) = z / sqrt(mean(z^2) + eps) * w              with EVG_NORM_RMS (no biases)
 *            = (z - mean) / sqrt(var + eps) * w + b       with EVG_NORM_LAYER (b may be absent)
 * so that one call ends one block and begins the next.  Token t's gate is row t / gate_rows of its worker's gate: gate_rows = 1
 * is a gate for every value, gate_rows = rows one for each channel, between them one for each sequence. */
enum { EVG_NORM_RMS = 0, EVG_NORM_LAYER = 1 };

typedef struct evg_blocknorm evg_blocknorm;

typedef struct {
  uint32_t workers;    /* >= 1                                   */
  uint32_t width;      /* D, 1 .. EVG_BLOCKNORM_MAX_WIDTH        */
  uint32_t max_rows;   /* most rows of a worker that a call has  */
  uint32_t type;       /* of all tensors                         */
  uint32_t kind;       /* EVG_NORM_RMS or EVG_NORM_LAYER         */
  float eps;           /* >= 0                                   */
  float residual_scale, branch_scale; /* finite                  */
  uint32_t forward_only; /* nonzero: backward will not be called; the sums that it keeps (a few thousand rows of D in 32 bits) are not
                            allocated                            */
} evg_blocknorm_config;
#define EVG_BLOCKNORM_MAX_WIDTH 16384u

/* Matrices of rows x D for each worker: residual, branch, residual_out, normed and their gradients; ceil(rows / gate_rows) x D:
 * gate, d_gate; 1 x D (row is not read): weights, biases and their gradients. */
typedef struct {
  uint32_t rows;      /* of each worker, 0 .. max_rows                        */
  uint32_t gate_rows; /* tokens that share a row of the gate, >= 1 if there is one */
  evg_mat residual;   /* needed                                               */
  evg_mat branch;     /* or absent: then gate, post and post_bias are too     */
  evg_mat gate;       /* or absent: 1                                         */
  evg_mat post, post_bias;
  evg_mat pre, pre_bias; /* pre absent: no normed                             */
} evg_blocknorm_in;

evg_status evg_blocknorm_init(evg_blocknorm** out, const evg_blocknorm_config* cfg, void* hip_stream);
/* residual_out may be absent, or residual itself; normed is given exactly if pre is. */
evg_status evg_blocknorm_forward(evg_blocknorm* c, const evg_blocknorm_in* in, const evg_mat* residual_out, const evg_mat* normed);

typedef struct {
  evg_mat residual, branch, gate, post, post_bias, pre, pre_bias;
} evg_blocknorm_grads;

/* d_residual, d_normed: gradients of residual' and normed (either may be absent: 0; d_normed only with pre).  out: the gradient
 * of each input, any of them may be absent; a gradient of an absent input is refused.  rows = 0 leaves d_residual,
 * d_branch and d_gate empty and the weights' gradients 0.  out->residual may be d_residual. */
evg_status evg_blocknorm_backward(evg_blocknorm* c, const evg_blocknorm_in* in, const evg_mat* d_residual, const evg_mat* d_normed,
                                  const evg_blocknorm_grads* out);
evg_status evg_blocknorm_destroy(evg_blocknorm* c);

/* ---- the gated feed-forward block ----------------------------------------------------------------------------------
 * For each worker, x of rows x D, w_gate and w_up of F x D, w_down of D x F (F = hidden):
 *     h = act(x w_gate^T) * (x w_up^T),   y = h w_down^T
 * h, and in the backward pass the gradients of both projections, are rounded to the tensors' type, as the matrix cores take them; all else
 * stays in 32 bits.  With 16-bit types the activation's exponential and quotient are the hardware's, a few units of 2^-23 off.
 * Rows are at most 2^31 elements apart.  Tensors whose addresses, strides and widths are multiples of 16 bytes are read as they are; a width that
 * is not is copied first where there are more than 64 tokens (init then allocates room for the copies).  Tensors of whole widths at other addresses or
 * strides, as at the offsets of 16-bit arenas (multiples of 4 elements), are not copied: a product that reads one takes all its operands
 * through registers, which took up to 1.75 times as long.  That, and rows of 4 MB and more, is a matter of speed alone. */
enum { EVG_ACT_SILU = 0, EVG_ACT_GELU = 1, EVG_ACT_GELU_TANH = 2, EVG_ACT_RELU = 3 };

typedef struct evg_ffn evg_ffn;

typedef struct {
  uint32_t workers;      /* 1 .. 65535                              */
  uint32_t width;        /* D, 1 .. 2^20                            */
  uint32_t hidden;       /* F, 1 .. 2^20                            */
  uint32_t max_rows;     /* most tokens of a worker that a call has */
  uint32_t type;         /* of all tensors                          */
  uint32_t activation;   /* EVG_ACT_*                               */
  uint32_t train;        /* nonzero: backward will be called        */
} evg_ffn_config;

evg_status evg_ffn_init(evg_ffn** out, const evg_ffn_config* cfg, void* hip_stream);
/* Bytes that forward leaves for backward for so many rows of each worker: the projections in 32 bits, and h.  0 if c is NULL. */
uint64_t evg_ffn_saved_bytes(const evg_ffn* c, uint32_t rows);
/* saved: DEVICE, 16-byte aligned, evg_ffn_saved_bytes of them, or NULL where no backward pass follows. */
evg_status evg_ffn_forward(evg_ffn* c, uint32_t rows, const evg_mat* x, const evg_mat* w_gate, const evg_mat* w_up,
                           const evg_mat* w_down, const evg_mat* y, void* saved);
/* The gradients of the four inputs from dy and what forward saved; each of the four may be absent.  rows = 0: the weights'
 * gradients are 0. */
evg_status evg_ffn_backward(evg_ffn* c, uint32_t rows, const evg_mat* dy, const evg_mat* x, const evg_mat* w_gate,
                            const evg_mat* w_up, const evg_mat* w_down, const void* saved, const evg_mat* dx,
                            const evg_mat* dw_gate, const evg_mat* dw_up, const evg_mat* dw_down);
evg_status evg_ffn_destroy(evg_ffn* c);

#ifdef __cplusplus
}
#endif
#endif /* EVG_NN_H */
