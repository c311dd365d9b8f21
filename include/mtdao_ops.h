/*
 * mtdao_ops.h -- operators of a Peri-LN training step next to the optimizer
 * of mtdao.h, on MI355X (gfx950), in the same library:
 *
 *   mtdao_adamw_*      AdamW over many tensors at once, states in 32 or 8 bits
 *   mtdao_peri_norm*   the boundary of a Peri-LN block: the norm after the
 *                      block, its gate and residual scale, the norm before
 *                      the next block, and their gradients
 *   mtdao_quantize8,   matrices in 8-bit floating point with a scale for
 *   mtdao_product8     each block of 128, and their product
 *   mtdao_orthogonalize, mtdao_muon_*   updates of matrices orthogonalised by
 *                      Newton-Schulz products, and the optimizer of a model's
 *                      matrices that takes them
 *   mtdao_embedding*   rows of a table by token, and the table's gradient
 *   mtdao_cross_entropy   the loss over a vocabulary and its gradient
 *
 * Conventions are those of mtdao.h: caller-owned device memory, work that is
 * only enqueued on the HIP stream passed to each call (no allocation, no
 * host wait, no memset, so calls can be captured into a HIP graph), negative
 * MTDAO_ERR_* codes from host-side validation before anything is enqueued,
 * messages from mtdao_last_error(NULL) (calls without a handle),
 * mtdao_adamw_last_error or mtdao_muon_last_error.  Types are MTDAO_F32 / MTDAO_BF16.  Device pointers
 * are aligned to their element unless stated otherwise.
 *
 * 8-bit blocks.  A block holds e4m3 codes c_i (4 exponent bits of bias 7, 3
 * mantissa bits, largest 448) and one scale 2^e, stored as the byte e + 127:
 *   e = the smallest whole number with amax / 2^e <= 448, amax over the
 *       finite values of the block, e + 127 clamped to [1, 254];
 *   c_i = x_i / 2^e rounded to nearest, ties to even (the division is exact).
 * Infinities and NaN become NaN codes and leave their block's scale alone.
 * As the scales are powers of two, c_i 2^e is x_i rounded to four
 * significant bits wherever |x_i| >= 2^(e-6).
 */
#ifndef MTDAO_OPS_H
#define MTDAO_OPS_H

#include "mtdao.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MTDAO_BLOCK8 128 /* elements of a block along one axis */

/* ------------------------------------------------------------------ AdamW
 *
 * One step t = 1, 2, ... of every tensor, in fp32 from its stored values:
 *   g' = g min(1, max_norm / ||g||)   ||g||: L2 norm over all tensors
 *                                     (max_norm <= 0, or ||g|| = 0: g' = g)
 *   m  = beta1 m + (1 - beta1) g'
 *   v  = beta2 v + (1 - beta2) g'^2
 *   p  = p (1 - lr weight_decay) - lr m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps)
 * state_bits 32: m and v are fp32.  state_bits 8: m is held as 8-bit blocks
 * of 128 consecutive elements of its tensor (the last one may be short), and
 * v as such blocks of sqrt(v), whose positive values round to the smallest
 * positive code where they would round to 0.  p takes the new m and v before
 * they are rounded. */
typedef struct mtdao_adamw_tensor {
  void* p;             /* parameters, param_dtype                                      */
  const void* g;       /* gradients, grad_dtype                                        */
  void* m;             /* 32 bits: fp32; 8 bits: e4m3 codes.  16-byte aligned          */
  void* v;             /* as m, of v (8 bits: of sqrt(v))                              */
  uint8_t* m_scale;    /* 8 bits: one byte per block of m (NULL for 32 bits)           */
  uint8_t* v_scale;    /* 8 bits: one byte per block of v                              */
  int64_t numel;       /* >= 0                                                         */
  double weight_decay; /* >= 0                                                         */
} mtdao_adamw_tensor;

typedef struct mtdao_adamw_config {
  int32_t param_dtype;
  int32_t grad_dtype;
  int32_t state_bits;  /* 32 or 8                                                      */
  int32_t n_tensors;
  double beta1, beta2; /* in [0, 1)                                                    */
  double eps;          /* >= 0                                                         */
  double max_norm;     /* > 0: global-norm clip; <= 0: off                             */
  int64_t start_step;  /* steps already applied (0 fresh)                              */
} mtdao_adamw_config;

typedef struct mtdao_adamw mtdao_adamw;

/* Device workspace (bytes, 256-byte aligned, caller-owned, must outlive the
 * handle): a row per tensor, four bytes per 4096 elements, and with max_norm
 * > 0 the partial sums of the norm.  Reads the numel of tensors only.
 * Host-only. */
int32_t mtdao_adamw_workspace_bytes(const mtdao_adamw_config* cfg, const mtdao_adamw_tensor* tensors, size_t* bytes);

/* Validate and build a handle; enqueues the kernels that write the tensor
 * table into the workspace.  m, v and the scales are taken as they are (zero
 * them for a fresh run).  No two written buffers may overlap, nor a gradient
 * and a written buffer, unless it is its own tensor's, element on element. */
int32_t mtdao_adamw_init(const mtdao_adamw_config* cfg, const mtdao_adamw_tensor* tensors, void* workspace,
                         size_t workspace_bytes, void* hip_stream, mtdao_adamw** out);

/* Take the gradients of every tensor from other addresses from here on
 * (ordered on the stream). */
int32_t mtdao_adamw_set_grads(mtdao_adamw* h, const void* const* grads, void* hip_stream);

/* One step of all tensors.  The norm is summed in fp64 in a fixed order, so
 * results are deterministic.  t and lr are fixed at call time: a captured
 * step replays with them. */
int32_t mtdao_adamw_step(mtdao_adamw* h, double lr, void* hip_stream);

int64_t mtdao_adamw_step_count(const mtdao_adamw* h); /* -1 for NULL */
const char* mtdao_adamw_last_error(const mtdao_adamw* h);
void mtdao_adamw_destroy(mtdao_adamw* h);

/* -------------------------------------------------------- Peri-LN boundary
 *
 * For every row (token) t of D elements, in fp32:
 *   h  = norm(f) w_post
 *   x' = x + scale gate[t / rows_per_gate] h
 *   n  = norm(x') w_pre
 * norm(z) = (z - mu) / sqrt(mean((z - mu)^2) + eps), mu = 0 (MTDAO_NORM_RMS)
 * or mean(z) (MTDAO_NORM_LAYER).  f is a block's output, x the residual
 * stream, n the next block's input; n takes x' before it is rounded to its
 * type.  f == NULL: x' = x and only n is written (the first norm of a
 * model).  w_pre == NULL: only x' is written.  gate == NULL: 1.
 *
 * Backward: from the gradients dx' (d_out) and dn, and x', f as stored,
 *   D' = dx' + dL/dx' through n     dx = D'
 *   dh = scale gate D'              df through norm(f) w_post
 *   d_w_pre  = sum_t dn norm(x')    d_w_post = sum_t dh norm(f)
 *   d_gate[j] = scale sum over the rows of gate j of D' h
 * The sums over rows are fp32, in an order that sizes alone fix.
 * d_out == NULL or dn == NULL: that gradient is zero.  w_pre == NULL: there is
 * no n, and dn is not read. */
enum { MTDAO_NORM_RMS = 0, MTDAO_NORM_LAYER = 1 };

#define MTDAO_PERI_MAX_D 8192

typedef struct mtdao_peri_norm_args {
  int64_t rows;          /* T >= 0                                                     */
  int64_t d;             /* D, 1..MTDAO_PERI_MAX_D                                     */
  int32_t kind;          /* MTDAO_NORM_RMS / MTDAO_NORM_LAYER                          */
  int32_t stream_dtype;  /* of x, x', d_out, dx                                        */
  int32_t branch_dtype;  /* of f, n, dn, df                                            */
  int32_t weight_dtype;  /* of w_post, w_pre, gate                                     */
  float eps;             /* >= 0                                                       */
  float scale;           /* residual scale                                             */
  int64_t rows_per_gate; /* >= 1 (ignored without gate)                                */
  int64_t ld_x, ld_f, ld_d_out, ld_dn; /* elements from row to row of the inputs, >= D */
  const void* x;         /* forward: x; backward: x'                                   */
  const void* f;
  const void* w_post;    /* [D], needed with f                                         */
  const void* w_pre;     /* [D]                                                        */
  const void* gate;      /* [ceil(T / rows_per_gate)][D]                               */
  const void* d_out;     /* backward                                                   */
  const void* dn;        /* backward                                                   */
  void* x_out;           /* forward: x' [T][D] (may be x itself when ld_x == D); backward: dx */
  void* n_out;           /* forward: n [T][D]                                          */
  void* df;              /* backward                                                   */
  float* d_w_post;       /* backward, fp32 [D]                                         */
  float* d_w_pre;        /* backward, fp32 [D]                                         */
  float* d_gate;         /* backward, fp32 [ceil(T / rows_per_gate)][D]                */
} mtdao_peri_norm_args;

int32_t mtdao_peri_norm(const mtdao_peri_norm_args* a, void* hip_stream);

/* Device workspace of the backward pass (partial sums for the parameter
 * gradients).  Reads the sizes of a and which of f, w_pre and gate
 * are given.  Host-only. */
int32_t mtdao_peri_norm_backward_workspace_bytes(const mtdao_peri_norm_args* a, size_t* bytes);

int32_t mtdao_peri_norm_backward(const mtdao_peri_norm_args* a, void* workspace, size_t workspace_bytes,
                                 void* hip_stream);

/* ---------------------------------------------------------- 8-bit product
 *
 * A matrix of 8-bit blocks, rows x cols.  Blocks are 1 x 128 (scale_rows =
 * 1) or 128 x 128 (scale_rows = 128), the last ones short. */
typedef struct mtdao_matrix8 {
  uint8_t* codes;      /* [rows][ld], 16-byte aligned; zeros past cols up to the next  */
                       /* multiple of 128, nothing after it                            */
  uint8_t* scales;     /* [ceil(blocks of a row / 4)][ceil(rows / scale_rows)][4]:     */
                       /* rows of four blocks' bytes together, 4-byte aligned          */
  int64_t rows, cols;
  int64_t ld;          /* a multiple of 128 from cols on; odd multiples load fastest   */
  int64_t scale_ld;    /* bytes of four blocks' scales: 4 ceil(rows / scale_rows)      */
  int32_t scale_rows;  /* 1 or 128                                                     */
} mtdao_matrix8;

/* x [rows][cols] (dtype, row stride ld elements) as 8-bit blocks, into q
 * and/or, transposed, into qt (qt->rows = cols; either may be NULL).  q and
 * qt have the same scale_rows; with 128 both hold the same values, with 1
 * the blocks of qt lie along the rows of x.  Columns past cols up to a whole
 * block and scale bytes past the last block are written too (codes 0, scale
 * 1). */
int32_t mtdao_quantize8(const void* x, int32_t dtype, int64_t ld, const mtdao_matrix8* q, const mtdao_matrix8* qt,
                        void* hip_stream);

/* c [a->rows][b->rows] = a b^T: the sums over the common columns (a->cols ==
 * b->cols) in fp32, rounded once to c_dtype.  accumulate (fp32 c only): c +=.
 * An fp32 c takes every product whole.  A bf16 c is summed by the 8-bit matrix
 * instructions at twice the rate: of each eight products that they add at once
 * they leave out what lies more than 13 bits below the largest, 2^-10 of the sum
 * of magnitudes at the very most and up to 4e-5 of c in relative norm (normal
 * values with larger columns among them), where rounding to bf16 takes 1.7e-3.
 * Where that counts, ask for an fp32 c.
 * Without columns the sums are zero, and nothing of a or b is read.
 * The order of the sums depends on the sizes alone.
 * workspace: mtdao_product8_workspace_bytes, 256-byte aligned. */
int32_t mtdao_product8_workspace_bytes(int64_t m, int64_t n, int64_t k, size_t* bytes);
int32_t mtdao_product8(const mtdao_matrix8* a, const mtdao_matrix8* b, void* c, int32_t c_dtype, int64_t ldc,
                       int32_t accumulate, void* workspace, size_t workspace_bytes, void* hip_stream);

/* A linear layer with 8-bit weights w [n][k] (blocks of 128 x 128 or 1 x 128),
 * m rows (tokens) of x: y [m][n] = x w^T, x in blocks of 1 x 128 along its
 * rows.  Up to 16 rows it is one launch.
 * Backward, from dy [m][n] and x (both dtype) and wt [k][n], w transposed:
 * dx [m][k] = dy w (dtype), dy in blocks along its rows, and dw [n][k] = dy^T x
 * (fp32; accumulate: dw +=), dy and x in blocks along the tokens.  The same
 * results as mtdao_quantize8 and mtdao_product8 one after the other (so a bf16 y
 * or dx is summed as a bf16 c), with their 8-bit matrices in the workspace
 * (256-byte aligned). */
int32_t mtdao_linear8_workspace_bytes(int64_t m, int64_t n, int64_t k, size_t* forward, size_t* backward);
int32_t mtdao_linear8(const void* x, int32_t dtype, int64_t rows, int64_t ld, const mtdao_matrix8* w, void* y, int32_t y_dtype,
                      int64_t ldy, void* workspace, size_t workspace_bytes, void* hip_stream);
int32_t mtdao_linear8_backward(const void* dy, const void* x, int32_t dtype, int64_t rows, int64_t ld_dy, int64_t ld_x,
                               const mtdao_matrix8* wt, void* dx, int64_t ld_dx, float* dw, int64_t ld_dw, int32_t accumulate,
                               void* workspace, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------ orthogonalised updates
 *
 * For a matrix x [rows][cols], its transpose where rows > cols:
 *   X = x / (||x|| + eps)              ||x||: the root of the sum of squares
 *   `steps` times:  A = X X^T,  X <- a X + (b A + c A A) X
 *   with a, b, c = 3.4445, -4.7750, 2.0315
 * which leaves the singular vectors of x as they are and moves its singular
 * values towards 1 (after five steps those from 1/400 of ||x|| on lie in about
 * 0.7 to 1.2).  ||x|| is summed in fp64; products are of about the precision of fp32 (factors
 * in 23 bits, sums in fp32).  The order of sums depends on the sizes of all matrices of the
 * call (of the batch, or of the handle) alone: equal calls give equal bits, but a
 * matrix may give other last bits among others than alone.
 * Elements of X are held to 2^-39: a matrix with ||x|| far below eps, whose X is as
 * small, keeps fewer bits, or none.
 * x = 0 gives 0 (eps > 0); infinities and NaN make all of their matrix NaN. */
#define MTDAO_MUON_MAX_SIDE 16384 /* of a matrix's smaller side; the larger one: 2^20 */
#define MTDAO_MUON_MAX_STEPS 64

/* batch matrices, one after another without gaps, x (dtype) to out (out_dtype);
 * out may be x where the types are equal.  workspace: 256-byte aligned. */
int32_t mtdao_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols, size_t* bytes);
int32_t mtdao_orthogonalize(const void* x, int32_t dtype, int64_t batch, int64_t rows, int64_t cols, void* out, int32_t out_dtype,
                            int32_t steps, double eps, void* workspace, size_t workspace_bytes, void* hip_stream);

/* One step of every matrix:
 *   m = momentum m + g
 *   u = g + momentum m (nesterov) or m
 *   p = p (1 - lr weight_decay) - lr factor o,   o: u orthogonalised
 * m is fp32; o and the new p are formed in fp32, p rounded once. */
typedef struct mtdao_muon_matrix {
  void* p;             /* [rows][cols], param_dtype                                    */
  const void* g;       /* [rows][cols], grad_dtype                                     */
  float* m;            /* [rows][cols]                                                 */
  int64_t rows, cols;  /* >= 0                                                         */
  double weight_decay; /* >= 0                                                         */
  double factor;       /* of the update                                                */
} mtdao_muon_matrix;

typedef struct mtdao_muon_config {
  int32_t param_dtype;
  int32_t grad_dtype;
  int32_t n_matrices;
  int32_t nesterov;
  int32_t steps;       /* 1..MTDAO_MUON_MAX_STEPS                                      */
  int32_t reserved;    /* 0                                                            */
  double momentum;     /* in [0, 1)                                                    */
  double eps;          /* >= 0                                                         */
} mtdao_muon_config;

typedef struct mtdao_muon mtdao_muon;

/* Device workspace (bytes, 256-byte aligned, caller-owned, must outlive the
 * handle): a row per matrix, and the factors of the matrices that are worked
 * on together (4 GiB, or what a single larger matrix takes).  Reads the sizes of matrices
 * only.  Host-only. */
int32_t mtdao_muon_workspace_bytes(const mtdao_muon_config* cfg, const mtdao_muon_matrix* matrices, size_t* bytes);

/* Validate and build a handle; enqueues the kernels that write the table of
 * matrices into the workspace.  m is taken as it is.  No two of all p and m may
 * overlap, nor a gradient and one of them. */
int32_t mtdao_muon_init(const mtdao_muon_config* cfg, const mtdao_muon_matrix* matrices, void* workspace, size_t workspace_bytes,
                        void* hip_stream, mtdao_muon** out);

/* Take the gradients of every matrix from other addresses from here on
 * (ordered on the stream). */
int32_t mtdao_muon_set_grads(mtdao_muon* h, const void* const* grads, void* hip_stream);

/* One step of all matrices; lr is fixed at call time: a captured step replays
 * with it. */
int32_t mtdao_muon_step(mtdao_muon* h, double lr, void* hip_stream);

const char* mtdao_muon_last_error(const mtdao_muon* h);
void mtdao_muon_destroy(mtdao_muon* h);

/* ------------------------------------------------------------- embedding
 *
 * out[i] = scale table[tokens[i]], for n_tokens tokens (token_bits: 32 or 64)
 * and a table of rows x d with row stride ld, in fp32, rounded once to out_dtype.
 * A token below 0 stands for none: its row is zero.  One that the table does not
 * have makes its row NaN; no memory outside the table is read.
 *
 * Backward: dw[r] = scale sum of dy[i] over the places i with tokens[i] == r
 * (accumulate: dw[r] +=, and rows of tokens that do not come are not touched),
 * fp32 sums in the order of the places, in pieces of 32; tokens outside the
 * table are left out.  Results depend on the operands alone.
 * workspace: 256-byte aligned. */
int32_t mtdao_embedding(const void* tokens, int32_t token_bits, int64_t n_tokens, const void* table, int32_t table_dtype, int64_t rows,
                        int64_t d, int64_t ld, float scale, void* out, int32_t out_dtype, int64_t ld_out, void* hip_stream);
int32_t mtdao_embedding_backward_workspace_bytes(int64_t n_tokens, int64_t rows, int64_t d, size_t* bytes);
int32_t mtdao_embedding_backward(const void* dy, int32_t dy_dtype, int64_t ld_dy, const void* tokens, int32_t token_bits, int64_t n_tokens,
                                 float scale, float* dw, int64_t rows, int64_t d, int64_t ld_dw, int32_t accumulate, void* workspace,
                                 size_t workspace_bytes, void* hip_stream);

/* ---------------------------------------------------------- cross entropy
 *
 * For every row x of logits and its target y:
 *   lse = log sum_j exp(x_j)
 *   loss_i = lse - x_y + z_loss lse^2
 *   d_i = w_i (softmax(x) (1 + 2 z_loss lse) - [j = y])
 * in fp32.  A target below 0 stands for none: loss 0, gradient 0, whatever its
 * logits are.  One that the row does not have makes its loss and gradient NaN, as
 * does a row without a logit above minus infinity.  loss is the sum of the rows' losses, or their
 * mean over the rows with a target (0 where there is none), summed in fp64.  w_i = scale d_loss, over the
 * number of rows with a target for the mean; d_loss is one number, or for
 * MTDAO_LOSS_NONE one for each row (NULL: 1). */
enum { MTDAO_LOSS_NONE = 0, MTDAO_LOSS_SUM = 1, MTDAO_LOSS_MEAN = 2 };

typedef struct mtdao_cross_entropy_args {
  int64_t rows, cols;    /* 0..2^31, 1..2^31                                           */
  int64_t ld_logits;     /* elements from row to row, >= cols                          */
  int64_t ld_d;          /* of d_logits                                                */
  int32_t dtype;         /* of logits and d_logits                                     */
  int32_t target_bits;   /* 32 or 64                                                   */
  int32_t reduction;     /* MTDAO_LOSS_*                                               */
  float z_loss;
  float scale;           /* of the gradient                                            */
  int32_t reserved;      /* 0                                                          */
  const void* logits;
  const void* targets;
  const float* d_loss;   /* device; NULL: 1                                            */
  float* losses;         /* of every row, or NULL                                      */
  float* loss;           /* their sum or mean, or NULL                                 */
  void* d_logits;        /* or NULL; may be logits itself when the strides are equal   */
} mtdao_cross_entropy_args;

/* What is written overlaps no other operand, but for d_logits in place of logits. */
/* Reads the sizes and the reduction of a.  Host-only.  workspace: 256-byte aligned. */
int32_t mtdao_cross_entropy_workspace_bytes(const mtdao_cross_entropy_args* a, size_t* bytes);
int32_t mtdao_cross_entropy(const mtdao_cross_entropy_args* a, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* MTDAO_OPS_H */
