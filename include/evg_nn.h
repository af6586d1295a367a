/* evg_nn.h -- C ABI of the operators that make, train and bound the gradients of feed-forward blocks for a ring's workers.
 *
 * Scope.  evg_step takes each worker's gradient (EVG_GRAD_BUFFER); these operators are what comes before it when the workers
 * train transformer feed-forward blocks: the norms on both sides of a block with its gate and residual scale (evg_blocknorm),
 * the gated feed-forward block (evg_ffn), both with their backward passes, and clipping by the global norm over a worker's
 * tensors (evg_clip).  Tokens become rows of the residual stream (evg_embed); blocks of several experts need a router (evg_router) and
 * tokens in the experts' order and back (evg_experts), all three with their backward passes; matrices' gradients become orthogonal
 * updates (evg_ortho).  All W workers of a ring, each with its own weights and tokens, go in one call; W = 1 is one model.
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

/* ---- embeddings ------------------------------------------------------------------------------------------------------
 * For each worker, a table of V x D (V = vocab, D = width) and T tokens:
 *     y[t] = scale * table[id[t]],    d_table[v] = scale * sum of dy[t] over the tokens t with id[t] = v
 * A token whose number is not in 0 .. V-1 (padding) has a row of zeros and no part in the gradient.  Sums are in 32 bits, over a number's tokens
 * in their order.  W V, and W T times the KB of a row, are below 2^31. */
typedef struct evg_embed evg_embed;

typedef struct {
  uint32_t workers;    /* 1 .. 65535                              */
  uint32_t vocab;      /* V, 1 .. 2^24                            */
  uint32_t width;      /* D, 1 .. 2^20                            */
  uint32_t max_tokens; /* most tokens of a worker that a call has, <= 2^26 */
  uint32_t type;       /* of table, rows and their gradients      */
  float scale;         /* finite                                  */
  uint32_t train;      /* nonzero: backward will be called        */
} evg_embed_config;

/* DEVICE token numbers: that of worker w's token t at p + w * worker + t, of 32 or (wide) 64 bits, signed. */
typedef struct {
  const void* p;
  int64_t worker; /* in numbers, >= 0 */
  uint32_t wide;
} evg_ids;

evg_status evg_embed_init(evg_embed** out, const evg_embed_config* cfg, void* hip_stream);
evg_status evg_embed_forward(evg_embed* c, uint32_t tokens, const evg_ids* ids, const evg_mat* table, const evg_mat* y);
/* accumulate: the sums are added to d_table (in 32 bits, rounded once) and rows that no token names are left as they are;
 * otherwise those are 0. */
evg_status evg_embed_backward(evg_embed* c, uint32_t tokens, const evg_ids* ids, const evg_mat* dy, const evg_mat* d_table, uint32_t accumulate);
evg_status evg_embed_destroy(evg_embed* c);

/* ---- which experts a token goes to --------------------------------------------------------------------------------------
 * For each token, from E logits: the K experts with the largest, the largest first, equal ones in the order of their numbers, and
 *     w = softmax(logits) at the chosen, or (over_chosen) the softmax over the chosen alone.
 * An expert at minus infinity is never chosen: where there are fewer than K others, the last places have -1 and weight 0.  A NaN goes before
 * all else, and makes the weights that the formula makes of it.  Backward, from dw:
 *     d_logits = w (dw - sum w dw) at the chosen, 0 elsewhere (over_chosen),   or   p (dw - sum w dw),  p the softmax, dw = 0 elsewhere. */
typedef struct evg_router evg_router;

typedef struct {
  uint32_t workers;    /* >= 1                                    */
  uint32_t experts;    /* E, 1 .. EVG_ROUTER_MAX_EXPERTS          */
  uint32_t top;        /* K, 1 .. E                               */
  uint32_t max_tokens; /* most tokens of a worker that a call has */
  uint32_t type;       /* of logits and their gradient            */
  uint32_t over_chosen;
} evg_router_config;
#define EVG_ROUTER_MAX_EXPERTS 1024u

evg_status evg_router_init(evg_router** out, const evg_router_config* cfg, void* hip_stream);
/* logits: tokens x E for each worker.  chosen, weights: DEVICE, [workers][tokens][K]. */
evg_status evg_router_forward(evg_router* c, uint32_t tokens, const evg_mat* logits, int32_t* chosen, float* weights);
/* chosen: what forward wrote.  What d_weights has where chosen is -1 does not count.  d_logits may be logits itself. */
evg_status evg_router_backward(evg_router* c, uint32_t tokens, const float* d_weights, const evg_mat* logits, const int32_t* chosen,
                               const evg_mat* d_logits);
evg_status evg_router_destroy(evg_router* c);

/* ---- tokens by expert and back ----------------------------------------------------------------------------------------
 * For each worker, T tokens with K experts each (chosen, T x K numbers): entry i = t K + k.  Entries are sorted by expert, those of one expert stay in
 * their order, and each gets a slot:
 *     capacity 0:  the slots 0 .. T K - 1 one after the other, expert by expert; those behind the last entry stay empty
 *     capacity C:  expert e has the slots e C .. e C + C - 1; what exceeds them is left out
 * Entries whose number is not in 0 .. E-1 are left out too.  With capacity C the rows of all experts are E matrices of C x D, as evg_ffn with W E
 * workers takes them.
 *     dispatch            rows[slot[i]] = x[t],  empty slots 0
 *     combine             y[t] = sum_k weights[i] rows[slot[i]]                  (in 32 bits, in k's order; without weights: all 1)
 *     combine_backward    d_rows[slot[i]] = weights[i] dy[t], empty slots 0;  d_weights[i] = <dy[t], rows[slot[i]]>, 0 where left out
 * and the gradient of dispatch is combine without weights. */
typedef struct evg_experts evg_experts;

typedef struct {
  uint32_t workers;    /* 1 .. 65535                              */
  uint32_t experts;    /* E, 1 .. EVG_ROUTER_MAX_EXPERTS          */
  uint32_t top;        /* K, 1 .. E                               */
  uint32_t width;      /* D, 1 .. 2^20                            */
  uint32_t max_tokens; /* most tokens of a worker that a call has; K times as many below 2^28 */
  uint32_t capacity;   /* C, or 0; E C below 2^31                 */
  uint32_t type;       /* of rows and their gradients             */
} evg_experts_config;

/* Where entries went: DEVICE, [workers][tokens][K], [workers][slots], [workers][E]. */
typedef struct {
  int32_t* slot;   /* -1: left out                                                       */
  int32_t* source; /* the entry in a slot, -1: empty                                     */
  int32_t* counts; /* entries of each expert, with those that found no room              */
} evg_experts_plan;

evg_status evg_experts_init(evg_experts** out, const evg_experts_config* cfg, void* hip_stream);
/* Slots of each worker for so many tokens.  0 if c is NULL. */
uint64_t evg_experts_slots(const evg_experts* c, uint32_t tokens);
/* x: tokens x D; rows: slots x D.  The plan is written. */
evg_status evg_experts_dispatch(evg_experts* c, uint32_t tokens, const evg_mat* x, const int32_t* chosen, const evg_mat* rows,
                                const evg_experts_plan* plan);
/* Only the plan's slots are read; weights may be NULL. */
evg_status evg_experts_combine(evg_experts* c, uint32_t tokens, const evg_mat* rows, const float* weights, const evg_experts_plan* plan,
                               const evg_mat* y);
/* The plan's slots and sources are read.  d_rows or d_weights may be absent, rows is needed for d_weights only. */
evg_status evg_experts_combine_backward(evg_experts* c, uint32_t tokens, const evg_mat* dy, const evg_mat* rows, const float* weights,
                                        const evg_experts_plan* plan, const evg_mat* d_rows, float* d_weights);
evg_status evg_experts_destroy(evg_experts* c);

/* ---- orthogonal updates ------------------------------------------------------------------------------------------------
 * For each of W matrices G of R x C:
 *     m' = momentum * m + G,   u = G + momentum * m' (nesterov) or m'           (in 32 bits; without m: u = G)
 *     X  = u / (|u| + eps),    |u| = sqrt(sum u^2)                             (sum in 64 bits)
 *     steps times:  S = X X^T,  X <- a X + (b S + c S S) X                      (S = X^T X, X <- a X + X (b S + c S S) where R > C)
 *     out = scale * X
 * which takes every singular value s of X to p(s) = a s + b s^3 + c s^5, again and again: with the usual constants close to 1, singular vectors stay.
 * Products are of float16 operands with sums in 32 bits.  X is kept as two of them, 22 bits; S, b S + c S S and the products' operands are two as well, but for bfloat16 tensors
 * whose smaller side is above 256.  What five steps with the constants 3.4445, -4.7750 and 2.0315 leave, of the result's norm, beside its rounding and what sums in 32 bits do: 3e-7 to 4e-5, for
 * those bfloat16 tensors 1e-4 to 1.8e-3 (a 32-bit result of theirs is no more exact).  Other constants and more steps stretch errors as they stretch singular values, and what they, or an eps far
 * above |u|, make much smaller than the largest that a singular value can become is known to so many bits fewer.  A zero matrix stays zero, a matrix with a NaN or an infinity becomes NaN. */
typedef struct evg_ortho evg_ortho;

typedef struct {
  uint32_t matrices; /* W, 1 .. 65535                                                     */
  uint32_t rows, cols; /* 1 .. 65536, the smaller of them at most 16384                   */
  uint32_t type;     /* of G                                                              */
  uint32_t out_type; /* type or EVG_F32; the products' precision goes by type and sides   */
  uint32_t steps;    /* 1 .. 64                                                           */
  float a, b, c;     /* finite; constants under which a singular value of 0 .. 1 passes 3 are refused */
  float momentum;    /* finite                                                            */
  uint32_t nesterov;
  float eps;         /* >= 0, finite                                                      */
  float scale;       /* finite, 0 or at least 2^-80 in magnitude                          */
} evg_ortho_config;

evg_status evg_ortho_init(evg_ortho** out, const evg_ortho_config* cfg, void* hip_stream);
/* momentum: float, R x C for each matrix, or absent; momentum_out: where m' goes, momentum itself or apart from it, given exactly if momentum is.
 * out may be grad itself where the types are the same. */
evg_status evg_ortho_update(evg_ortho* c, const evg_mat* grad, const evg_mat* momentum, const evg_mat* momentum_out, const evg_mat* out);
evg_status evg_ortho_destroy(evg_ortho* c);

#ifdef __cplusplus
}
#endif
#endif /* EVG_NN_H */
