/*
 * choco_train.h - C ABI of the operators around the CHOCO-SGD step (choco.h) that a language model's
 * workers run between two gossip steps on one MI355X (gfx950): the embedding lookup out of the
 * workers' parameter rows and its gradient into their gradient rows, two ways to mix the looked-up
 * sequence with their backward passes (a gated linear recurrence, and linear attention whose states are
 * matrices), and two ways to update the tensors of all workers (AdamW, and along orthogonalised momentum).
 *
 * The conventions of choco.h hold: CHOCO_OK or a negative code, nothing printed, nothing aborts; *_dev are
 * device pointers, *_host host pointers; buffers belong to the caller, the library allocates no device memory;
 * work is enqueued on the caller's stream, with the device current that the stream and the pointers are of, and no call
 * waits for it, except choco_adamw_init and choco_muon_init (they copy a table of the tensors to the device).  Calls with nothing to do (no tokens, no sequences, no channels) return CHOCO_OK
 * and enqueue nothing.
 */
#ifndef CHOCO_TRAIN_H
#define CHOCO_TRAIN_H

#include "choco.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of entries. */
enum { CHOCO_F32 = 0, CHOCO_BF16 = 1, CHOCO_F16 = 2 };
enum { CHOCO_I32 = 0, CHOCO_I64 = 1 };

/* ---- embedding lookup and its gradient --------------------------------------------------------
 * Worker w looks up its tokens in its own table of vocab rows of dim entries, e.g. a tensor of its row of X:
 *   y[w, r, :] = scale * table[w, token[w, r], :], rounded once; zero where the token is not in [0, vocab)
 *   dtable[w, v, :] = scale * sum of dy[w, r, :] over the r with token[w, r] = v
 * The sums are taken in fp32, in an order that depends on the tokens alone: same inputs, same bits. */
typedef struct {
  int32_t n;             /* workers, 0 <= n <= 65535                                                 */
  int64_t tokens;        /* per worker, 0 <= tokens < 2^31                                           */
  int64_t vocab, dim;    /* 1 <= vocab < 2^31, 0 <= dim < 2^31                                       */
  int32_t token_type;    /* CHOCO_I32 / CHOCO_I64                                                    */
  int32_t table_type;    /* forward: CHOCO_F32 / BF16 / F16; the gradient is always CHOCO_F32        */
  int32_t row_type;      /* of y and dy: CHOCO_F32 / BF16 / F16                                      */
  int64_t token_stride;  /* entries from worker to worker, >= tokens                                 */
  int64_t table_stride;  /* ... of the table or its gradient, >= vocab * dim; a table's rows lie dim apart.  (Workers that
                            share one table are one worker with all their tokens.)                   */
  int64_t row_stride;    /* ... of y / dy, >= tokens * row_ld                                        */
  int64_t row_ld;        /* entries from one row of y / dy to the next, >= dim                       */
  float scale;
  void* stream;          /* hipStream_t; NULL = the null stream                                      */
} choco_embed_config;

/* Bytes of device workspace that choco_embed_backward needs (16-byte aligned); may be 0. */
int choco_embed_workspace_bytes(const choco_embed_config* cfg, size_t* bytes_host);
/* CHOCO_E_INVAL: a size, type or stride outside its range, a null pointer, a pointer that is not aligned to its
   entries.  CHOCO_E_UNSUPPORTED: more work than one launch holds. */
int choco_embed_forward(const choco_embed_config* cfg, const void* tokens_dev, const void* table_dev, void* y_dev);
/* accumulate = 0: every entry of the vocab x dim gradient is written (zero for tokens that do not occur);
   1: the sums are added to what is there, other rows are left alone (a table that is also the output layer).
   CHOCO_E_NOMEM: workspace too small. */
int choco_embed_backward(const choco_embed_config* cfg, const void* tokens_dev, const void* dy_dev, float* dtable_dev,
                         int accumulate, void* workspace_dev, size_t workspace_bytes);

/* ---- gated linear recurrence ------------------------------------------------------------------
 * For every sequence b and channel c, with a = sigmoid(f_t):
 *   h_t = a h_{t-1} + (1 - a) u_t,   y_t = sigmoid(o_t) h_t  (y_t = h_t without o)
 * States are fp32; y is rounded once.  A sequence of lengths[b] < steps steps keeps its state from there on
 * and its further y (and gradients) are zero, whatever its further inputs hold; lengths are clamped to [0, steps].
 * A state that is infinite stays so or becomes NaN (where the product of the gates since is below fp32's range), in its channel of
 * its sequence only.  In long sequences workgroups wait for the states of earlier ones; a wait that does not end within some
 * seconds is given up and the states after it are NaN, without an error code.
 * Inputs of 16 bits are multiplied by 16-bit matrix instructions, from a few steps on, with fp32 operands as sums of 16-bit numbers: to 2^-22 of what is added
 * up or nearer in CHOCO_F16; in CHOCO_BF16 to 2^-25 for states, dq, dk and dg and to 2^-17 for y and dv, which are rounded to 2^-9 next.  In CHOCO_F16 an
 * entry of a state counts relative to the largest of its column, and one step's product of q and k relative to the largest of its 64 steps': what is less than
 * 2^-39 of that is lost.
 * Generation is steps = 1 with h0 = the last state; h_last may be h0's own buffer. */
#define CHOCO_RECUR_SAVE_STEPS 8
typedef struct {
  int64_t batch, steps, dim; /* >= 0 each, below 2^31; batch * dim and batch * steps below 2^40                 */
  int32_t type;              /* of f, u, o, y and their gradients: CHOCO_F32 / BF16 / F16                */
  /* entries [0] from sequence to sequence, [1] from step to step; channels are next to one another.
     Strides are >= 0; those of outputs must keep entries apart.  (f, u and o may be columns of one matrix.) */
  int64_t f_stride[2], u_stride[2], o_stride[2], y_stride[2]; /* y_stride: of dy in the backward pass   */
  int64_t df_stride[2], du_stride[2], do_stride[2];           /* backward pass only                     */
  void* stream;
} choco_recur_config;

/* Bytes of what the forward pass keeps for the backward one: the fp32 state before every
   CHOCO_RECUR_SAVE_STEPS-th step, ceil(steps / CHOCO_RECUR_SAVE_STEPS) x batch x dim.  Errors as of the passes. */
int choco_recur_saved_bytes(const choco_recur_config* cfg, size_t* bytes_host);
/* Bytes of device workspace that either pass needs (16-byte aligned); may be 0. */
int choco_recur_workspace_bytes(const choco_recur_config* cfg, size_t* bytes_host);
/* Errors as above.  o_dev, h0_dev (batch x dim fp32; zero without), lengths_dev (batch int32), h_last_dev (batch x dim fp32) and
   saved_dev may be NULL. */
int choco_recur_forward(const choco_recur_config* cfg, const void* f_dev, const void* u_dev, const void* o_dev,
                        const float* h0_dev, const int32_t* lengths_dev, void* y_dev, float* h_last_dev, float* saved_dev,
                        void* workspace_dev, size_t workspace_bytes);
/* saved_dev as the forward pass on the same f, u, h0 and lengths wrote it.  With dlast the gradient of h_last (NULL:
   zero), s = sigmoid(o) (1 without o), from the last step of a sequence back:
     e_t = dy_t s_t + a_{t+1} e_{t+1}  (+ dlast at its last step),  do_t = dy_t h_t s_t (1 - s_t),
     du_t = (1 - a_t) e_t,  df_t = e_t (h_{t-1} - u_t) a_t (1 - a_t),  dh0 = a_1 e_1  (dlast for an empty one).
   do_dev is written iff o_dev is given; dh0_dev (batch x dim fp32) may be NULL. */
int choco_recur_backward(const choco_recur_config* cfg, const void* f_dev, const void* u_dev, const void* o_dev,
                         const int32_t* lengths_dev, const float* saved_dev, const void* dy_dev, const float* dlast_dev,
                         void* df_dev, void* du_dev, void* do_dev, float* dh0_dev, void* workspace_dev, size_t workspace_bytes);

/* ---- linear attention with a decay for each head ------------------------------------------------
 * For every sequence and head, with a state S of dim_k x dim_v and the logarithm g_t <= 0 of a decay:
 *   S_t = exp(g_t) S_{t-1} + k_t v_t^T,   y_t = S_t^T q_t
 * States and g are fp32; y is rounded once.  The attention has `heads` heads; q, k and v may have fewer: each of q_heads, k_heads
 * and v_heads divides heads, and head h reads q's head h / (heads / q_heads), and so on.
 * A sequence of lengths[b] < steps steps keeps its state from there on and its further y (and gradients) are zero, whatever its
 * further inputs hold; lengths are clamped to [0, steps].  g = -infinity starts over: nothing from before is left.
 * (Below -200 g counts as that, and so does a decay between two steps that is less than 2^-126.)
 * An input that is infinite or NaN makes y of its sequence and head NaN or infinite from up to 63 steps before it on (steps are taken
 * together), and the state; other sequences and heads are not touched.
 * Generation is steps = 1 with h0 = the last state; h_last may be h0's own buffer (also with more steps). */
#define CHOCO_LINEAR_SAVE_STEPS 256
#define CHOCO_LINEAR_MAX_DIM 256
typedef struct {
  int64_t batch, steps;     /* >= 0, below 2^31; batch * heads below 2^24                                      */
  int32_t heads;            /* >= 0                                                                            */
  int32_t q_heads, k_heads, v_heads; /* >= 1, divisors of heads                                                */
  int32_t dim_k, dim_v;     /* 1 .. CHOCO_LINEAR_MAX_DIM                                                       */
  int32_t type;             /* of q, k, v, y and their gradients: CHOCO_F32 / BF16 / F16                       */
  int32_t gate_steps;       /* 1: g is fp32 of every sequence, step and head; 0: one number for each head       */
  /* entries [0] from sequence to sequence, [1] from step to step, [2] from head to head; a head's entries are next to one
     another.  Strides are >= 0; those of outputs must keep entries apart.  (q, k and v may be columns of one matrix.) */
  int64_t q_stride[3], k_stride[3], v_stride[3], y_stride[3]; /* y_stride: of dy in the backward pass          */
  int64_t g_stride[3];                                        /* gate_steps = 0: only [2] is read              */
  int64_t dq_stride[3], dk_stride[3], dv_stride[3];           /* backward pass only                            */
  void* stream;
} choco_linear_config;

/* Bytes of what the forward pass keeps for the backward one, a buffer of fp32 states that only choco_linear_backward reads: of each
   sequence and head the state before every CHOCO_LINEAR_SAVE_STEPS-th step and the last one. */
int choco_linear_saved_bytes(const choco_linear_config* cfg, size_t* bytes_host);
/* Bytes of device workspace that the forward (backward = 0) or the backward pass needs (16-byte aligned); may be 0. */
int choco_linear_workspace_bytes(const choco_linear_config* cfg, int backward, size_t* bytes_host);
/* Errors as above; CHOCO_E_UNSUPPORTED: more than some 10^6 sequences' heads or a like number of their pieces of 256 steps.  h0_dev
   (batch x heads x dim_k x dim_v fp32; zero without), lengths_dev (batch int32), h_last_dev (as h0) and saved_dev may be NULL.
   Outputs may not overlap inputs, but for h_last and h0. */
int choco_linear_forward(const choco_linear_config* cfg, const void* q_dev, const void* k_dev, const void* v_dev,
                         const float* g_dev, const float* h0_dev, const int32_t* lengths_dev, void* y_dev, float* h_last_dev,
                         float* saved_dev, void* workspace_dev, size_t workspace_bytes);
/* saved_dev as the forward pass on the same k, v, g, h0 and lengths wrote it.  With dlast the gradient of h_last (NULL: zero),
   from the last step of a sequence back, E_t the gradient of S_t:
     E_t = q_t dy_t^T + exp(g_{t+1}) E_{t+1}  (+ dlast at its last step),
     dq_t = S_t dy_t,  dk_t = E_t v_t,  dv_t = E_t^T k_t,  dg_t = exp(g_t) <E_t, S_{t-1}>,  dh0 = exp(g_1) E_1 (dlast for an empty one);
   the gradients of heads that share a q, k or v are added up.  dg_t is added up of what passes step t alone, so that a gate that is
   nearly closed has as many places right as an open one.  dg_dev: batch x steps x heads fp32, or with gate_steps = 0
   heads sums over all steps.  dg_dev and dh0_dev (as h0) may be NULL.  Every sum is taken in an order that
   depends on the sizes alone: same inputs, same bits. */
int choco_linear_backward(const choco_linear_config* cfg, const void* q_dev, const void* k_dev, const void* v_dev,
                          const float* g_dev, const int32_t* lengths_dev, const float* saved_dev, const void* dy_dev,
                          const float* dlast_dev, void* dq_dev, void* dk_dev, void* dv_dev, float* dg_dev, float* dh0_dev,
                          void* workspace_dev, size_t workspace_bytes);

/* ---- AdamW ------------------------------------------------------------------------------------
 * One update of every tensor of every worker, x the n x ld fp32 parameter rows (the X of choco_init):
 *   g <- grad_scale g;  m <- beta1 m + (1 - beta1) g;  v <- beta2 v + (1 - beta2) g^2
 *   x <- x (1 - lr' wd) - lr' / (1 - beta1^t) * m / (sqrt(v / (1 - beta2^t)) + eps),  lr' = lr * lr_scale
 * with weight decay wd and lr_scale per tensor.  It takes the place of the local update before a gossip step
 * (choco_sgd_step, choco_momentum_step).
 * state_bits 32: m and v in fp32.  8: in a byte each, relative to a power of two that CHOCO_ADAMW_BLOCK consecutive
 * entries of a tensor share (blocks start at its first entry) and that brings the largest of them into (0.9375, 1.875].
 * m is a sign, 4 bits of exponent and 3 of mantissa, v 5 and 3, both with gradual underflow: m reaches down to 2^-17,
 * v to 2^-33 of its block's largest.  (A block whose largest lies below the normal numbers is held relative to 2^-126.)  Rounding is
 * stochastic: with nearest rounding a v that moves by 0.1 % a step would never leave its code.  The random bits
 * are those of the Philox word of (seed, step, worker, entry), stream 3, the lower 16 for m and the upper 16 for
 * v, so a run is reproducible.  A positive v is never held as zero (x would move by m / eps).  The update of x takes m and
 * v before they are rounded.
 * An infinite or NaN gradient makes its entry of x and its m and v NaN or infinite; in 8 bits m and v of its whole block.
 * One whose square is infinite in fp32 (above 1.8e19) does that to v. */
#define CHOCO_ADAMW_BLOCK 256
typedef struct choco_adamw choco_adamw; /* opaque, host memory, freed by choco_adamw_destroy */
typedef struct {
  int32_t n;             /* workers, 1 <= n <= 65535                                                  */
  int64_t d, ld;         /* as in choco_config (ld 0: d rounded up to a multiple of 4)                */
  /* The tensors as slices of a row, HOST arrays, copied: disjoint, ascending, anywhere in [0, d), start
     [t] >= start[t-1] + len[t-1], len >= 0.  Entries in no tensor are left alone.  ntensors = 0: the whole row is one. */
  int32_t ntensors;
  const int64_t* start_host;
  const int64_t* len_host;
  const float* weight_decay_host; /* per tensor (or one entry where ntensors = 0), >= 0; NULL: none  */
  const float* lr_scale_host;     /* likewise; NULL: 1                                                */
  double beta1, beta2;   /* in [0, 1)                                                                 */
  double eps;            /* >= 2^-60 / sqrt(1 - beta2) (2.8e-17 for 0.999): below that v's own range in fp32 shows in x */
  int32_t state_bits;    /* 32 or 8                                                                   */
  uint64_t seed;
  void* stream;          /* of choco_adamw_init and, until choco_adamw_set_stream, of the calls after it */
} choco_adamw_config;

/* CHOCO_E_UNSUPPORTED: more tensors, and gaps between them, than one launch holds (some 2^26 pieces of up to 1024 entries). */
int choco_adamw_workspace_bytes(const choco_adamw_config* cfg, size_t* bytes_host);
/* x_dev 16-byte, workspace_dev 256-byte aligned; moments start at zero, t at 0.  On error *out is NULL. */
int choco_adamw_init(const choco_adamw_config* cfg, float* x_dev, void* workspace_dev, size_t workspace_bytes,
                     choco_adamw** out);
/* g_dev: n x ld entries of grad_type (CHOCO_F32 or CHOCO_BF16), 16-byte aligned.  grad_scale_dev: n floats on the
   device, a factor for each worker's gradient (clipping, loss scale), NULL: 1; a worker whose factor is not finite is
   left as it is, moments and all (a step skipped without the host looking).  Asynchronous; advances t, which is
   an argument of the launch: a captured step replays with the t and lr it was captured with. */
int choco_adamw_step(choco_adamw* a, const void* g_dev, int32_t grad_type, float lr, const float* grad_scale_dev);
/* The moments as fp32 (what they stand for in 8 bits), n x ld floats each, zero in entries of no tensor.  Asynchronous. */
int choco_adamw_moments(choco_adamw* a, float* m_dev, float* v_dev);
/* The part of the workspace that holds the moments: what to save, and with t to put back, to resume a run.  In 32 bits it is m
   and then v, n x ld floats each, v on the next multiple of 256 bytes. */
int choco_adamw_state(choco_adamw* a, void** state_dev, size_t* bytes_host);
/* The stream of the calls that follow, at first the configuration's.  Waits for nothing: what is under way on the former stream is
   the caller's to order. */
int choco_adamw_set_stream(choco_adamw* a, void* stream);
int choco_adamw_get_step(choco_adamw* a, uint64_t* t_host);
int choco_adamw_set_step(choco_adamw* a, uint64_t t);
/* Does not wait for the stream.  NULL is allowed. */
int choco_adamw_destroy(choco_adamw* a);

/* ---- orthogonalised matrices, and an optimiser that steps along them -----------------------------------
 * The iteration on a matrix U, in fp32, from X = U / |U|_F (zero for a zero matrix):
 *   P = X X^T,   X <- a X + (b P + c P^2) X,   (a, b, c) = (3.4445, -4.7750, 2.0315)
 * brings singular values near one: into 0.68 .. 1.21 after five, those from 1 / 500 of |U|_F on.  Smaller ones grow 3.4-fold each time.  Where U has more rows
 * than columns it is taken transposed, which gives the same matrix.  Products are of fp32 accuracy: operands are two fp16 numbers
 * each, 22 bits, and sums are fp32.  A matrix with an infinite or NaN entry becomes NaN. */
typedef struct {
  int64_t batch;          /* matrices, >= 0                                                              */
  int64_t rows, cols;     /* 0 .. 65536 each                                                             */
  int32_t type;           /* of the input: CHOCO_F32 / BF16 / F16; the result is fp32                     */
  int64_t x_stride[2];    /* entries [0] from matrix to matrix, [1] from row to row, >= 0; a row's entries are next to one another */
  int64_t y_stride[2];    /* of the result, which must keep entries apart                                */
  int32_t iterations;     /* 1 .. 32                                                                     */
  void* stream;
} choco_orthogonalize_config;

/* Bytes of device workspace (256-byte aligned); may be 0. */
int choco_orthogonalize_workspace_bytes(const choco_orthogonalize_config* cfg, size_t* bytes_host);
/* y_dev may be x_dev (fp32, the same strides), else they may not overlap.  CHOCO_E_UNSUPPORTED: more work than one launch holds. */
int choco_orthogonalize(const choco_orthogonalize_config* cfg, const void* x_dev, float* y_dev, void* workspace_dev,
                        size_t workspace_bytes);

/* One update of matrices of every worker, slices of the n x ld fp32 parameter rows x (the X of choco_init):
 *   g <- grad_scale g;   m <- momentum m + g;   u = g + momentum m (nesterov) or m
 *   x <- x (1 - lr wd) - lr lr_scale O(u)
 * with O the iteration above.  It takes the place of the local update of these matrices; choco_adamw on the same rows may take the other
 * tensors. */
typedef struct choco_muon choco_muon; /* opaque, host memory, freed by choco_muon_destroy */
typedef struct {
  int32_t n;             /* workers, 1 <= n <= 65535                                                  */
  int64_t d, ld;         /* as in choco_config (ld 0: d rounded up to a multiple of 4)                */
  /* The matrices, rows x cols entries row after row from start on, HOST arrays, copied: disjoint, ascending, anywhere in
     [0, d), start[t] >= start[t-1] + rows[t-1] cols[t-1]; rows and cols 0 .. 65536.  Entries in none are left alone. */
  int32_t ntensors;      /* >= 1                                                                      */
  const int64_t* start_host;
  const int64_t* rows_host;
  const int64_t* cols_host;
  const float* weight_decay_host; /* per matrix, >= 0; NULL: none                                    */
  const float* lr_scale_host;     /* likewise; NULL: sqrt(max(1, rows / cols))                        */
  double momentum;       /* in [0, 1)                                                                 */
  int32_t nesterov;      /* 0 / 1                                                                     */
  int32_t iterations;    /* 1 .. 32                                                                   */
  void* stream;          /* of choco_muon_init and, until choco_muon_set_stream, of the calls after it */
} choco_muon_config;

int choco_muon_workspace_bytes(const choco_muon_config* cfg, size_t* bytes_host);
/* workspace_dev 256-byte aligned; momenta start at zero.  On error *out is NULL. */
int choco_muon_init(const choco_muon_config* cfg, float* x_dev, void* workspace_dev, size_t workspace_bytes, choco_muon** out);
/* g_dev: n x ld entries of grad_type (CHOCO_F32 or CHOCO_BF16).  grad_scale_dev: n floats on the device, a factor for each
   worker's gradient, NULL: 1; a worker whose factor is not finite is left as it is, momenta and all.  Asynchronous; a captured
   step replays with the lr it was captured with. */
int choco_muon_step(choco_muon* a, const void* g_dev, int32_t grad_type, float lr, const float* grad_scale_dev);
/* The part of the workspace that holds the momenta: fp32, matrix after matrix, of each n x rows x cols.  What to save to resume a run. */
int choco_muon_state(choco_muon* a, void** state_dev, size_t* bytes_host);
/* As choco_adamw_set_stream and choco_adamw_destroy. */
int choco_muon_set_stream(choco_muon* a, void* stream);
int choco_muon_destroy(choco_muon* a);

/* raw hipError_t behind the last CHOCO_E_HIP that a call of this header returned on this thread. */
int choco_train_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* CHOCO_TRAIN_H */
