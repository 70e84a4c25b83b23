/*
 * ah_ops.h — operators that a stage of a newer decoder trains with, one call each (C ABI, part of libahstage.so): attention
 * over a sliding window with visible first tokens, norms of the query and key heads with the position rotation, and the
 * optimizer step over a stage's tensors.
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

#ifdef __cplusplus
}
#endif
#endif /* AH_OPS_H */
