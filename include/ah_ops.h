/*
 * ah_ops.h — operators that a stage of a newer decoder trains with, one call each (C ABI, part of libahstage.so): attention
 * over a sliding window with visible first tokens, norms of the query and key heads with the position rotation, the
 * optimizer steps over a stage's tensors (AdamW, and Muon for its matrices), and what stands before the first stage and behind the last one: the
 * embedding of the tokens, the norm in front of the head, the loss of the logits.
 *
 * The rules of ah_stage.h hold: plain C, every function returns an ah_status_t and leaves a message for ah_last_error(), device
 * memory is the caller's, work is only enqueued on `hip_stream` (a hipStream_t cast to void*; NULL = the default stream) and
 * nothing synchronises or allocates, so that every call may be captured into a HIP graph.  The device that holds the buffers
 * must be the calling thread's current device.  Matrices are row-major, activations and parameters bf16 unless said otherwise.
 * A scratch buffer is used from the call's first kernel to its last: calls that may overlap (other streams, replays of
 * captured graphs) need one each.
 */
#ifndef AH_OPS_H
#define AH_OPS_H

#include "ah_stage.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- the optimizer step over the fp32 gradients that the K micro-batches of an iteration left (Section III-A) ---- */

typedef enum { AH_BF16 = 0, AH_FP32 = 1 } ah_type_t;

/* One tensor of a step.  Device pointers, each aligned to its element; n elements one behind the other.  What a call writes overlaps nothing else that
 * it reads or writes (an element of a tensor given twice would be stepped twice, in no order); gradients may be shared. */
typedef struct {
  void* param;          /* bf16 or fp32: ah_adamw_t.param_type */
  const void* grad;     /* bf16 or fp32: ah_adamw_t.grad_type */
  void* m;              /* first moment: fp32, or one byte an element */
  void* v;              /* second moment: likewise */
  uint8_t* m_scale;     /* 8-bit states: one byte for each 32 elements (the last may be short), else NULL */
  uint8_t* v_scale;
  float* master;        /* bf16 parameters kept in fp32 (the step reads and writes this one, param gets it rounded), or NULL: all tensors of a call alike */
  uint64_t n;           /* 0 is allowed */
  float weight_decay;   /* decoupled: param *= 1 - lr * weight_decay */
  uint32_t reserved;    /* 0 */
} ah_adamw_tensor_t;

/* The step: with g' = factor * g (factor: below),
 *   m += (1 - beta1) (g' - m);   v += (1 - beta2) (g'^2 - v);
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^step) m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * in fp32, the moments without fused multiply-adds (so that any IEEE machine gets the same bits).  bf16 parameters without a master copy are rounded
 * to nearest after every step: one below half a unit in a parameter's last place is lost.
 *
 * 8-bit states.  32 consecutive elements share a scale 2^(s - 127), the top binade of the block: the least for which the block's
 * largest value is within 1.75 (m) or 1.875 (v) times it.  m: sign, 4 bits of exponent, 3 of mantissa (the bit pattern
 * of e4m3); v: 5 bits of exponent, 3 of mantissa; both with gradual underflow below their last binade.  The step itself uses the
 * unrounded moments.  They are rounded to a neighbouring code at random, with the probability that keeps their expectation (a
 * step takes at most 1 - beta2 of v away, and the middle between a code and the one below it is 1/32 to 1/18 of the code away: rounded to nearest, v would never
 * shrink where 1 - beta2 is below 1/32, 0.99 or 0.999, and stop at some of its codes at 0.95); the random bits are a function of `seed` plus the step's number (modulo 2^32) and of the element's number alone (tensors are numbered
 * one behind the other, each from a multiple of 64 on; the bits repeat after 2^32 elements).  They have to differ from step to step: where an element is
 * rounded by the same ones every time, its moments stand still.  A captured step therefore needs `step_dev` (and its owner counts that up
 * between replays); without it the call is refused.  A v > 0 never becomes 0 (m / sqrt(v) would have no
 * bound).  A block whose moment is infinite or NaN stays so, as a single 32-bit state would.  Zero bytes stand for zeros. */
typedef struct {
  uint32_t struct_size;   /* sizeof(ah_adamw_t), checked */
  int32_t param_type, grad_type;   /* ah_type_t; master copies go with bf16 parameters */
  int32_t state_bits;     /* 32 or 8 */
  double lr, beta1, beta2, eps;    /* lr >= 0, betas in [0, 1), eps >= 1e-37 (its reciprocal is finite in fp32) */
  int64_t step;           /* 1, 2, ... */
  const float* lr_dev;    /* device, optional: read by the kernel in place of lr ... */
  const int32_t* step_dev;   /* ... and of step (at least 1): a captured step can be replayed with other values */
  const float* grad_norm; /* device, optional: the two values that ah_grad_norm left.  The second is the factor above; NaN leaves everything as it was. */
  uint32_t seed;          /* of the random rounding: the step's number is added to it, so one value serves all steps */
  uint32_t reserved;      /* 0 */
} ah_adamw_t;

/* tensors: HOST array, read during the call. */
int ah_adamw_step(const ah_adamw_t* cfg, const ah_adamw_tensor_t* tensors, int n_tensors, void* hip_stream);

/* out[0] = the 2-norm of all the tensors' gradients together, out[1] = min(1, max_norm / out[0]) (1 where max_norm is 0: no limit, else at least 2^-126;
 * NaN where the norm is not finite).  Reads the tensors' grad and n only.  out: device, two floats.  Sums in fp64, in an order that depends on the sizes alone.
 * workspace: device, of the size that ah_grad_norm_workspace gives, 8-byte aligned. */
int ah_grad_norm(const ah_adamw_tensor_t* tensors, int n_tensors, int grad_type, double max_norm, float* out, void* workspace, void* hip_stream);
int ah_grad_norm_workspace(int n_tensors, uint64_t* bytes);

/* What 8-bit states stand for, as bf16 (which holds every one of them exactly): m_out[i] and v_out[i] (device, n elements each) for
 * tensor i.  m_out and v_out: HOST arrays of n_tensors device pointers. */
int ah_adamw_state_values(const ah_adamw_tensor_t* tensors, int n_tensors, void* const* m_out, void* const* v_out, void* hip_stream);

/* ---- attention over a sliding window with visible first tokens ----
 *
 * n_seq sequences; position i of one sees position j of it iff j <= i and (i - j < window or j < sinks).  Row t of q holds n_heads heads of head_dim
 * columns, of k and v n_kv_heads; query head h reads key and value head h / (n_heads / n_kv_heads).  Scores are scaled by
 * 1 / sqrt(head_dim), softmax and sums in fp32; probabilities (and their gradients) are rounded to bf16 for the second product, as in
 * ah_attention_fwd and _bwd.  A NaN shows in all rows that see it (a score of -infinity counts as nothing); what is not finite may reach rows within 192 positions of
 * those too (a block of 128 queries walks tiles of 64 keys).  Sizes: seq_len at most 2^24, n_heads 4096, and n_seq * n_heads * (ceil(seq_len / 128) +
 * 8 ceil(sinks / 128)) at most 2^23, packed sequences counted at seq_len each: so is the memory of lse and of the workspace.
 *
 * Sequences of one length: seq_len rows each, one behind the other (offsets NULL).  Packed: sequence b has the rows offsets[b] .. offsets[b + 1] - 1
 * (device, int32 [n_seq + 1], ascending, each length 0 .. seq_len); rows of no sequence are neither read nor written.  A sequence that would begin or
 * end outside the `rows` rows of the buffers is cut there, one longer than seq_len at seq_len. */
typedef struct {
  uint32_t struct_size;   /* sizeof(ah_attention_window_t), checked */
  int32_t n_seq, seq_len; /* >= 1; any length */
  int32_t n_heads, n_kv_heads;   /* n_kv_heads divides n_heads */
  int32_t head_dim;       /* 64 or 128 */
  int32_t window;         /* >= 1: positions that a query sees, its own among them */
  int32_t sinks;          /* >= 0: first positions of the sequence that every later one sees */
  int64_t rows;           /* rows of the buffers (0: n_seq * seq_len, for offsets NULL at least that) */
  const int32_t* offsets;
  /* columns from row to row, multiples of 8; 0: the rows are dense */
  int64_t ld_q, ld_k, ld_v, ld_o, ld_do, ld_dq, ld_dk, ld_dv;
} ah_attention_window_t;

/* Results overlap neither each other nor what the call reads (columns of a packed matrix beside each other do not).
 * o (bf16, rows of n_heads * head_dim) and lse (fp32 [n_seq][n_heads][seq_len], natural logarithm; entries behind a sequence's end are left as they are). */
int ah_attention_window_fwd(const ah_attention_window_t* cfg, const void* q, const void* k, const void* v, void* o, float* lse, void* hip_stream);
/* dq, dk, dv (bf16) from the forward's inputs and results and d_o.  No atomics: the same bits every time.  workspace: device, 256-byte aligned, of the size that
 * ah_attention_window_bwd_workspace gives (which looks at the sizes only). */
int ah_attention_window_bwd(const ah_attention_window_t* cfg, const void* q, const void* k, const void* v, const void* o, const float* lse, const void* d_o,
                            void* dq, void* dk, void* dv, void* workspace, void* hip_stream);
int ah_attention_window_bwd_workspace(const ah_attention_window_t* cfg, uint64_t* bytes);

/* ---- norms of the query and key heads with the position rotation ----
 *
 * Row t of x holds n_heads query heads and behind them n_kv_heads key heads of head_dim columns each (the first columns of a packed
 * projection [Q | K | V]).  Each head by itself: n = x / sqrt(mean(x^2) + eps) * gain (gain_q or gain_k, bf16 [head_dim]); then
 * columns i and i + head_dim / 2 turn by the angle of the row's position p: y_i = n_i c - n_{i + d/2} s,
 * y_{i + d/2} = n_{i + d/2} c + n_i s with (c, s) = cos_sin[p][i].  In fp32, rounded once (a head whose sum of squares is above fp32's range, elements of 1e18 and
 * more, comes out as zeros). */
typedef struct {
  uint32_t struct_size;        /* sizeof(ah_qk_norm_rope_t), checked */
  int32_t rows;                /* T >= 0 */
  int32_t seq_len;             /* position of row t: t % seq_len (ignored with `positions`) */
  int32_t n_heads, n_kv_heads; /* >= 0, not both 0 */
  int32_t head_dim;            /* 64 or 128 */
  int32_t n_pos;               /* rows of cos_sin; without `positions` at least min(seq_len, rows) */
  float eps;                   /* >= 2^-126 */
  int64_t ld_x, ld_y, ld_dx;   /* columns from row to row of x, of y (or dy) and of dx: multiples of 8, at least (n_heads + n_kv_heads) * head_dim; 0: just that */
  const void *gain_q, *gain_k; /* device; gain_k may be NULL where n_kv_heads is 0, gain_q likewise */
  const float* cos_sin;        /* device [n_pos][head_dim / 2][2] (ah_rope_table); NULL: no rotation */
  const int32_t* positions;    /* device [rows], optional; a row whose position is outside [0, n_pos) comes out as NaN (and, backward, the gains' gradients) */
} ah_qk_norm_rope_t;

/* y may be x with the same row stride (each element is read before it is written); else it overlaps nothing that the call reads. */
int ah_qk_norm_rope_fwd(const ah_qk_norm_rope_t* cfg, const void* x, void* y, void* hip_stream);
/* dx (bf16) from x and dy; dx may be dy or x with the same row stride.  d_gain_q, d_gain_k (fp32 [head_dim]) = beta * themselves + the gains' gradients, beta in {0, 1}: sums in
 * an order that depends on the sizes alone.  Either may be NULL where there are no such heads.  workspace: device, 16-byte aligned, of the size that
 * ah_qk_norm_rope_bwd_workspace gives. */
int ah_qk_norm_rope_bwd(const ah_qk_norm_rope_t* cfg, const void* x, const void* dy, void* dx, float* d_gain_q, float* d_gain_k, int beta,
                        void* workspace, void* hip_stream);
int ah_qk_norm_rope_bwd_workspace(const ah_qk_norm_rope_t* cfg, uint64_t* bytes);
/* cos_sin[p][i] = (cos, sin)(p base^(-2 i / head_dim)) for p < n_pos, in fp64 rounded to fp32 (the table of the LLaMA-style stage). */
int ah_rope_table(float* cos_sin, int n_pos, int head_dim, double base, void* hip_stream);

/* ---- the optimizer step of matrices by their momentum's orthogonal factor (Muon) ----
 *
 * For each matrix of its own (a shard of one, as a tensor-parallel stage holds it, is another matrix: its factor is not the whole one's block), with g' = factor * g (as in ah_adamw_step),
 *   m += (1 - momentum) (g' - m);   u = nesterov ? m + (1 - momentum) (g' - m) : m
 *   X = u / (|u| + eps), |u| the root of the sum of squares, X transposed where there are more rows than columns;
 *   ns_steps times: A = X X^T; X = a X + (b A + c A A) X, (a, b, c) = (3.4445, -4.7750, 2.0315), which brings the singular values of 1 / 500 and more to 0.68 .. 1.21;
 *   p = p (1 - lr weight_decay) - lr scale X.
 * Momentum, norm, update in fp32 (the sum of squares in fp64).  X is kept between the products in 22 bits (two fp16 numbers); the products' operands are fp16
 * (11 bits; all of them are at most 12 in magnitude whatever u is), their sums fp32: X is up to 2.6e-3 of its norm off (16 x 40 of random elements; 1.6e-3 at 512 x 512, 1.2e-3 at 2048 x 2048; 1e-4 to 1e-3
 * where few directions make a matrix up).
 * With parameters or master copies in fp32, matrices of at most 256 rows or columns have operands of 22 bits too (1e-6 to 5e-6 off); larger ones, of any type, do not.  Where that is fewer products, the first two steps are taken at once.  That, and the order of sums, is chosen for the matrices that are worked on together: a
 * matrix's update may differ in its roundings with the sizes that share its call, and is the same for the same ones.  bf16 parameters without a master copy are rounded to nearest after every step. */
typedef struct {
  void* param;          /* [rows, cols], bf16 or fp32: ah_muon_t.param_type */
  const void* grad;     /* bf16 or fp32: ah_muon_t.grad_type */
  float* momentum;      /* read and written */
  float* master;        /* bf16 parameters kept in fp32, or NULL: all matrices of a call alike */
  int64_t rows, cols;   /* 0 is allowed; at most 32768, the larger one 131072 */
  int64_t ld_param, ld_grad, ld_momentum, ld_master;   /* elements from row to row (a block of a wider matrix's columns, for one), at least cols; 0: cols */
  float weight_decay;   /* decoupled */
  float scale;          /* of the update; 0.2 sqrt(max(rows, cols)) makes its elements as large as AdamW's */
} ah_muon_matrix_t;

typedef struct {
  uint32_t struct_size;   /* sizeof(ah_muon_t), checked */
  int32_t param_type, grad_type;   /* ah_type_t; master copies go with bf16 parameters */
  int32_t nesterov, ns_steps;      /* 0 or 1; 1 .. 32 */
  uint32_t reserved;      /* 0 */
  double lr, momentum, eps;        /* lr >= 0, momentum in [0, 1), eps >= 1e-37 */
  const float* lr_dev;    /* device, optional: read by the kernel in place of lr */
  const float* grad_norm; /* device, optional: the two values that ah_grad_norm left.  The second is the factor above; NaN leaves everything as it was. */
} ah_muon_t;

/* matrices: HOST array, read during the call.  What a call writes overlaps nothing else that it reads or writes (columns of a wider matrix beside each other do not).
 * A matrix whose momentum is or becomes infinite or NaN is NaN behind the step; the others are not touched by it.  workspace: device, 256-byte aligned, of the size that
 * ah_muon_workspace gives for these matrices (which looks at rows and cols only, so that it is enough for all types): the largest group of matrices that are worked on together. */
int ah_muon_step(const ah_muon_t* cfg, const ah_muon_matrix_t* matrices, int n_matrices, void* workspace, void* hip_stream);
int ah_muon_workspace(const ah_muon_matrix_t* matrices, int n_matrices, uint64_t* bytes);

/* ---- embedding: what the first stage's rows are made from ----
 *
 * y_t = scale * table[token_t] + pos_table[position_t] in fp32, rounded once.  A token of -1 is none (padding): its row of the table counts as zeros, and it has no
 * gradient.  Any other outside [0, vocab), or a position outside [0, n_pos), makes its row NaN (backward: such a token has no gradient). */
typedef struct {
  uint32_t struct_size;       /* sizeof(ah_embedding_t), checked */
  int32_t rows;               /* T, 0 .. 2^25 */
  int32_t vocab;              /* rows of the table, 1 .. 2^30 */
  int32_t width;              /* 1 .. 65536 */
  int32_t table_type, act_type;   /* ah_type_t of table and pos_table, and of y or dy */
  int32_t token_bits;         /* 32 or 64: signed numbers of as many bits */
  float scale;                /* finite */
  int64_t ld_table, ld_act, ld_pos;   /* elements from row to row of table (backward: of d_table), y or dy, pos_table; at least width; 0: width */
  const void* pos_table;      /* device [n_pos, width], optional */
  int32_t n_pos, seq_len;     /* position of row t: t % seq_len, or ... */
  const int32_t* positions;   /* ... device [rows], optional */
} ah_embedding_t;

/* Results overlap nothing that a call reads. */
int ah_embedding_fwd(const ah_embedding_t* cfg, const void* table, const void* tokens, void* y, void* hip_stream);
/* d_table (fp32 [vocab, width]) = beta * d_table + scale * the sum of dy_t over the rows t with that token; beta in {0, 1}; 0 writes all rows, 1 reads and writes only
 * those whose token occurs.  Sums in fp32, in an order that depends on the tokens alone (no atomics).  The gradient of pos_table is that of a table of n_pos rows
 * with the positions as tokens and a scale of 1.  workspace: device, 256-byte aligned, of the size that ah_embedding_bwd_workspace gives (which looks at rows, vocab and width). */
int ah_embedding_bwd(const ah_embedding_t* cfg, const void* tokens, const void* dy, float* d_table, int beta, void* workspace, void* hip_stream);
int ah_embedding_bwd_workspace(const ah_embedding_t* cfg, uint64_t* bytes);

/* ---- layer norm: what stands in front of the head ----
 *
 * n = (x - mean(x)) / sqrt(mean((x - mean(x))^2) + eps) of each row (rms: without the mean), y = n * gain + bias, in fp32, rounded once (a row whose sum of squares is above
 * fp32's range, elements of 1e18 and more, comes out as its bias, backward as zeros or NaN).  What is not finite in a row stays in it (backward: and in the gradients of gain and bias). */
typedef struct {
  uint32_t struct_size;       /* sizeof(ah_layer_norm_t), checked */
  int32_t rows;               /* T, 0 .. 2^25 */
  int32_t width;              /* 1 .. 16384 */
  int32_t rms;                /* 0 or 1 */
  int32_t act_type, param_type;   /* ah_type_t of x, y, dy, dx; of gain and bias */
  float eps;                  /* >= 2^-126 */
  uint32_t reserved;          /* 0 */
  int64_t ld_x, ld_y, ld_dx;  /* elements from row to row of x, of y (or dy) and of dx; at least width; 0: width */
  const void *gain, *bias;    /* device [width]; NULL: ones, zeros */
} ah_layer_norm_t;

/* y may be x with the same row stride; else it overlaps nothing that the call reads. */
int ah_layer_norm_fwd(const ah_layer_norm_t* cfg, const void* x, void* y, void* hip_stream);
/* dx from x and dy (statistics are computed again); dx may be x or dy with the same row stride.  d_gain, d_bias (fp32 [width], either may be NULL) = beta * themselves + the
 * gradients, beta in {0, 1}: sums in an order that depends on the sizes alone.  workspace: device, 16-byte aligned, of the size that ah_layer_norm_bwd_workspace gives. */
int ah_layer_norm_bwd(const ah_layer_norm_t* cfg, const void* x, const void* dy, void* dx, float* d_gain, float* d_bias, int beta, void* workspace, void* hip_stream);
int ah_layer_norm_bwd_workspace(const ah_layer_norm_t* cfg, uint64_t* bytes);

/* ---- loss of the logits, with its gradient ----
 *
 * With lse = log(sum over j of exp(z_j)) of row t and its target i: loss_t = lse - z_i; d_logits_tj = s (exp(z_j - lse) - [j = i]) with s = scale (or *scale_dev), in fp32, rounded once.
 * A target of -1 is none: loss and gradient 0.  Any other outside [0, vocab) makes both NaN, and so does a row whose logits are all -infinity, or of which one is
 * +infinity or NaN; a logit of -infinity beside finite ones has the probability 0. */
typedef struct {
  uint32_t struct_size;       /* sizeof(ah_cross_entropy_t), checked */
  int32_t rows;               /* T, 0 .. 2^25 */
  int32_t vocab;              /* columns, 1 .. 2^24 */
  int32_t act_type;           /* ah_type_t of logits and d_logits */
  int32_t target_bits;        /* 32 or 64: signed numbers of as many bits */
  float scale;                /* of the gradient: 1 / (number of targets), for one; finite */
  const float* scale_dev;     /* device, optional: read by the kernel in place of scale */
  int64_t ld_logits, ld_grad; /* elements from row to row, at least vocab; 0: vocab */
} ah_cross_entropy_t;

/* loss: fp32 [rows].  d_logits: NULL (the loss alone), logits themselves with the same row stride, or a buffer that overlaps nothing that the call reads. */
int ah_cross_entropy(const ah_cross_entropy_t* cfg, const void* logits, const void* targets, float* loss, void* d_logits, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* AH_OPS_H */
