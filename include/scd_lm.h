/*
 * scd_lm.h -- what stands around the matrices that libscd.so packs, when a language model runs or learns: embedding rows
 * and their gradient, products in 8-bit integers (the other way to spend half of a bf16 matrix), and the cross entropy of
 * the output head with its gradients.
 *
 * Conventions of scd.h hold (device pointers owned by the caller, dense row-major arrays, status codes, void* streams)
 * with two differences, which these calls share with scd_col_signed_sum_noalloc: they only ENQUEUE their work on `stream`
 * and return, so that they can follow one another and be captured into a HIP graph; and they allocate nothing (work space
 * is the caller's, of the size the ..._workspace_bytes function gives, 16-byte aligned, in use until the stream has
 * passed the call; its contents need no initialisation and carry nothing from one call to the next).
 *
 *  - scd_real: the type of the real arrays of a call.  Arrays of it need only the alignment of the type; rows whose
 *    starts are aligned to 16 bytes are faster.  All sums are formed in f32 or wider (integer products: exactly, in
 *    int32) and rounded to the type once.
 *  - Index arrays (tokens, targets) hold int32 (index_bytes 4) or int64 (8).
 *  - Every result is the same bits from run to run: no float atomics, every sum in an order set by the sizes (cross entropy with rows
 *    of whole 16 bytes: and by whether W, in scd_xent also X, begins at a multiple of 16; if not, plainer sums serve the call, in
 *    f32 throughout).
 *  - Row counts may be 0 (nothing to do; gradients of weights are then zero).
 *  - SCD_EINVAL: null pointers, sizes below 1 (row counts: below 0) or above 2^31 - 1, an unknown type, a work space that
 *    is too small or misaligned.  SCD_EHIP: a launch failed (a call that takes 2^32 threads or more does: rows of odd lengths
 *    from about 2^34 entries on, cross entropy from 2^26 tokens or rows of the vocabulary on, embedding gradients from 2^28 rows on).
 *    Nothing is enqueued on SCD_EINVAL.
 */
#ifndef SCD_LM_H
#define SCD_LM_H

#include "scd.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SCD_REAL_F32 = 0, SCD_REAL_BF16 = 2, SCD_REAL_F16 = 3 } scd_real;

/* ---- embedding ---------------------------------------------------------------------------------
 * out (N x D): out_i = scale * E[t_i], E (V x D).  A token outside 0 .. V-1 gives a row of NaN. */
int scd_embed(const void* E, scd_real dt, int64_t V, int64_t D, const void* tokens, int index_bytes, int64_t N, float scale,
              void* out, void* stream);

/* dE (V x D, written whole): dE_v = scale * sum_{i: t_i = v} dY_i over dY (N x D), i ascending; rows without a token are
 * zero.  Tokens equal to `pad` or outside 0 .. V-1 count for nothing, whatever their rows of dY hold.
 * A few tokens need no work space (0 bytes; it may then be NULL). */
size_t scd_embed_grad_workspace_bytes(int64_t V, int64_t D, int64_t N);
int scd_embed_grad(const void* tokens, int index_bytes, int64_t N, const void* dY, scd_real dt, int64_t V, int64_t D, int64_t pad,
                   float scale, void* dE, void* workspace, size_t workspace_bytes, void* stream);

/* ---- products in 8-bit integers ------------------------------------------------------------------
 * A matrix of M rows of K entries is held as int8 rows of scd_q8_stride(K) bytes (K rounded up to a multiple of 128, zeros
 * behind the K entries; 16-byte aligned) and one f32 scale for each row:
 *     a_i = max(max_k |x_ik|, 2^-100),   q_ik = rint(x_ik * (127 * (1 / a_i))),   s_i = a_i / 127   (f32, ties to even)
 * so that x_ik ~ s_i q_ik.  A row with a NaN or an infinity has q = 0 and s = NaN.  Weights (one scale per output channel)
 * and activations (one per token) are held alike.  K <= SCD_Q8_MAX_K, which keeps every sum within int32. */
#define SCD_Q8_MAX_K 131072
int64_t scd_q8_stride(int64_t K);
int scd_q8_rows(const void* X, scd_real dt, int64_t M, int64_t K, int8_t* q, float* s, void* stream);

/* y (M x N) = xs_i ws_j sum_k xq_ik wq_jk (+ bias_j), for M tokens and N channels; the integer sum is exact, the rest f32.
 * bias: N entries of dt, or NULL. */
int scd_q8_matmul(const int8_t* xq, const float* xs, int64_t M, int64_t K, const int8_t* wq, const float* ws, int64_t N,
                  const void* bias, scd_real dt, void* y, void* stream);

/* The same from tokens that are not yet in 8 bits: scd_q8_rows of X (M x K, dt), then scd_q8_matmul; same bits.  One
 * token of up to about 114,000 entries and two of up to 57,000 need no work space (0 bytes; it may then be NULL). */
size_t scd_q8_linear_workspace_bytes(int64_t M, int64_t K);
int scd_q8_linear(const void* X, scd_real dt, int64_t M, int64_t K, const int8_t* wq, const float* ws, int64_t N, const void* bias,
                  void* y, void* workspace, size_t workspace_bytes, void* stream);

/* ---- cross entropy of the output head --------------------------------------------------------------
 * z = scale * X W^T for N hidden states X (N x D) and a vocabulary of V rows W (V x D):
 *     lse_i = log sum_v exp z_iv (every row),   loss_i = lse_i - z_{i,t_i}      (f32, N each)
 * loss is 0 where t_i == ignore, NaN where t_i is another value outside 0 .. V-1.  A logit that is NaN or +infinity makes its
 * row's lse and loss NaN.  In f32, D and V from 64 on, products are of three parts of bf16: entries below 2^-102 may lose some
 * of their 24 bits, finite ones beyond 3.39e38 may be taken for that.  Logits are formed tile by
 * tile and not kept: the work space holds two sums for each row and up to 128 of the vocabulary (where there are few logits in all: these). */
size_t scd_xent_workspace_bytes(scd_real dt, int64_t N, int64_t D, int64_t V);
int scd_xent(const void* X, const void* W, scd_real dt, int64_t N, int64_t D, int64_t V, const void* targets, int index_bytes,
             int64_t ignore, float scale, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* Gradients of sum_i g_i loss_i:  dz_iv = g_i (exp(z_iv - lse_i) - [v = t_i]),  dX = scale dz W (N x D),
 * dW = scale dz^T X (V x D), both of dt, written whole; either may be NULL (not both).  lse is scd_xent's.  The logits are
 * formed again, in pieces of the vocabulary.  A row with g_i = 0, t_i == ignore or t_i outside 0 .. V-1 counts for nothing,
 * whatever it holds: its dX is zero.  dz is rounded to dt before the products with W and X (16-bit types: the matrix cores
 * take 16-bit operands), held relative to the largest finite |g_i|, so that g carries no range of its own: in f16 in steps of 2^-39 of
 * that where its digits would be finer.  In bf16 and f32 it is lifted by 2^24 beside that, against the smallest numbers of the
 * type, and undone after the sums, which are therefore infinite where sum |dz x| / max |g| reaches 2^104 (2e31): entries of X and W
 * below 2^100 keep clear of it. */
size_t scd_xent_grad_workspace_bytes(scd_real dt, int64_t N, int64_t D, int64_t V);
int scd_xent_grad(const void* X, const void* W, scd_real dt, int64_t N, int64_t D, int64_t V, const void* targets, int index_bytes,
                  int64_t ignore, float scale, const float* lse, const float* g, void* dX, void* dW, void* workspace,
                  size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SCD_LM_H */
