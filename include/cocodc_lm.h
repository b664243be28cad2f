/*
 * cocodc_lm.h - operators of a worker's local step, for NVIDIA B200 (sm_100a).
 *
 * Between two synchronisations every worker trains a language model on its own (Section 2.1 of the paper: the
 * local steps whose result is the pseudo-gradient).  These entry points are the parts of that step that read or
 * write a vocabulary or a feed-forward width, each with its gradient:
 *
 *   embedding lookup   y[t] = scale * W[id_t]                                cocodc_lm_embed, cocodc_lm_embed_grad
 *   gated block        h = act(x Wg^T) * (x Wu^T)                            cocodc_lm_glu, cocodc_lm_glu_grad
 *   token scores       log p(y_t), entropy, top alternatives of a row        cocodc_lm_logprobs, cocodc_lm_logprobs_grad
 *
 * Conventions (those of cocodc.h, with these differences)
 *   - All pointers are device memory, except the handle.  Matrices are row-major with a row stride in elements
 *     (>= the width); columns are contiguous.  Types are given per call; sums, softmax statistics and matrix
 *     products are held in fp32 and every output is rounded to its type once.
 *   - Base pointers need the alignment of their element type.  Buffers whose base and row stride are multiples
 *     of 16 bytes take the vector / tensor-core paths; others run on slower kernels with the same results up
 *     to the order of fp32 sums.
 *   - Outputs must not overlap inputs or each other (COCODC_ERR_ALIAS), except where a call says so.  Different columns of one
 *     buffer (rows equally far apart) do not overlap; matrices with different distances of their rows must not lie within each other.
 *   - Calls are asynchronous on the given stream and allocate nothing.  Calls that need scratch take it as a
 *     workspace (16-byte aligned, at least cocodc_lm_*_workspace bytes, contents arbitrary and undefined
 *     afterwards; the size is 0 where the call refuses the sizes).  Nothing is kept from one call for the next, so one handle may be used on several streams
 *     and from several threads at the same time as long as the calls' workspaces differ.  Kernels are launched with
 *     programmatic dependence on the stream's previous kernel; they touch no memory before it has finished.
 *   - T = 0 (no tokens) is legal everywhere; pointers to nothing may then be NULL or not.
 *   - Token ids: a negative id means "no token here" (padding, ignored target).  An id >= V is an error that
 *     the kernel finds: it is treated as a negative one and COCODC_ERR_INVALID_ARG is recorded in the status
 *     word (cocodc_lm_poll_status).  It never leads to an access outside a buffer.
 *   - Results do not depend on scheduling: no floating-point atomics; the same call on the same inputs gives
 *     the same bits.
 */
#ifndef COCODC_LM_H
#define COCODC_LM_H

#include "cocodc.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { COCODC_F32 = 0, COCODC_BF16 = 1, COCODC_F16 = 2 } cocodc_dtype;
typedef enum { COCODC_I32 = 0, COCODC_I64 = 1 } cocodc_index_type;

/* Activation of the gated block: SILU g/(1+exp(-g)); GELU in its tanh form
 * g/2 * (1 + tanh(sqrt(2/pi) * (g + 0.044715 g^3))). */
typedef enum { COCODC_ACT_SILU = 0, COCODC_ACT_GELU = 1 } cocodc_activation;

typedef struct cocodc_lm cocodc_lm;   /* a device's status word and launch counter */

/* Errors of create: INVALID_ARG (NULL, no such device), NOMEM, CUDA. */
cocodc_status cocodc_lm_create(cocodc_lm** lm_out, int32_t device);
cocodc_status cocodc_lm_destroy(cocodc_lm* lm);

/* Waits for the stream, then returns and clears the status word (COCODC_OK if nothing was recorded). */
cocodc_status cocodc_lm_poll_status(cocodc_lm* lm, void* stream);

/* Number of kernels launched through this handle so far. */
int64_t cocodc_lm_launch_count(const cocodc_lm* lm);

/*
 * y[t][:] = scale * table[ids[t]][:] for t < T; a row of zeros where ids[t] < 0.
 *   table [V][D], any of the three types; y [T][D], any of the three types; ids [T]
 * The product is formed in fp32 and rounded once.
 */
cocodc_status cocodc_lm_embed(cocodc_lm* lm, const void* table, int32_t table_type, int64_t table_stride,
                              int64_t V, int64_t D, const void* ids, int32_t ids_type, int64_t T, float scale,
                              void* y, int32_t y_type, int64_t y_stride, void* stream);

/*
 * dtable[v][:] = scale * sum over t with ids[t] == v of dy[t][:]  (accumulate: added to what dtable holds).
 * Every row is written (zeros for tokens that do not occur); with accumulate only the rows of tokens that occur
 * are touched.  The tokens are sorted by id, equal ids by position, and each row is summed in fp32 in an order
 * that depends on the ids alone.  T <= 2^27, V <= 2^30.
 *   dy [T][D]; dtable [V][D]; types independent of each other
 */
uint64_t cocodc_lm_embed_grad_workspace(int64_t V, int64_t D, int64_t T);
cocodc_status cocodc_lm_embed_grad(cocodc_lm* lm, const void* dy, int32_t dy_type, int64_t dy_stride,
                                   const void* ids, int32_t ids_type, int64_t T, int64_t V, int64_t D, float scale,
                                   int32_t accumulate, void* dtable, int32_t dtable_type, int64_t dtable_stride,
                                   void* workspace, uint64_t workspace_bytes, void* stream);

/*
 * The gated feed-forward block: gate = x Wg^T, up = x Wu^T, h = act(gate) * up, in one kernel.
 *   x [T][D]; wg, wu [F][D] (one stride); h [T][F]; gate, up [T][F] (one stride) or both NULL: what
 *   cocodc_lm_glu_grad needs of the forward pass.  All of one type, BF16 or F16.
 * h is formed from the unrounded gate and up.
 */
cocodc_status cocodc_lm_glu(cocodc_lm* lm, int32_t act, int32_t type, const void* x, int64_t x_stride,
                            const void* wg, const void* wu, int64_t w_stride, int64_t T, int64_t D, int64_t F,
                            void* h, int64_t h_stride, void* gate, void* up, int64_t gu_stride, void* stream);

/*
 * Its gradient.  With dg = dh * up * act'(gate) and du = dh * act(gate):
 *   dx = dg Wg + du Wu   [T][D]        dwg = dg^T x, dwu = du^T x   [F][D] (one stride)
 * dx may be NULL; dwg and dwu may both be NULL.  dg and du are rounded to the type between the element-wise part
 * and the products, as tensor cores take them (F16: Inf beyond 65504); the products accumulate in fp32.  T = 0 sets dwg and dwu to zero.
 */
uint64_t cocodc_lm_glu_grad_workspace(int64_t T, int64_t D, int64_t F);
cocodc_status cocodc_lm_glu_grad(cocodc_lm* lm, int32_t act, int32_t type, const void* dh, int64_t dh_stride,
                                 const void* gate, const void* up, int64_t gu_stride, const void* x, int64_t x_stride,
                                 const void* wg, const void* wu, int64_t w_stride, int64_t T, int64_t D, int64_t F,
                                 void* dx, int64_t dx_stride, void* dwg, void* dwu, int64_t dw_stride,
                                 void* workspace, uint64_t workspace_bytes, void* stream);

/*
 * Row t of logits [T][V] (any type) gives z = scale * logits[t] (0 < scale <= 1e30: one over the temperature) and
 *   lse[t]     = log sum_j exp(z_j)
 *   logp[t]    = z_y - lse, y = targets[t]; 0 where y < 0
 *   entropy[t] = lse - sum_j p_j z_j,  p_j = exp(z_j - lse)
 *   top_ids[t][i], top_logp[t][i], i < top_k: the top_k largest logits in descending order, equal ones by
 *               ascending index (-0 equals +0), and their log probabilities
 * fp32 outputs, packed; each of logp (with targets), entropy, lse may be NULL, and top_k = 0 leaves the
 * alternatives out (top_ids and top_logp NULL).  top_k <= min(V, COCODC_LM_MAX_TOP).
 * Masked logits (-Inf) have p = 0 and add nothing to the entropy.  A row of nothing but -Inf has lse = -Inf,
 * entropy 0 and log probabilities -Inf.  A row with a NaN or +Inf has NaN in lse, entropy, logp (where y >= 0)
 * and top_logp; among its alternatives NaN ranks above +Inf.
 * Rows (where T is small, parts of a row) with such a value, with nothing left above a mask of -1e9 or lower or less than top_k, with
 * more than 1024 equal logits among the largest, or with |scale * logit| above 7e8 are read again element by element: once or twice for the
 * sums, top_k times for the alternatives (ten times the time for top_k = 8 where all of many rows are so).
 * All finite logits and all legal scales are good; lse is +-Inf where it leaves fp32's range, the other outputs do not suffer from it.
 */
#define COCODC_LM_MAX_TOP 32
cocodc_status cocodc_lm_logprobs(cocodc_lm* lm, const void* logits, int32_t type, int64_t stride, int64_t T, int64_t V,
                                 const void* targets, int32_t targets_type, float scale, float* logp, float* entropy,
                                 float* lse, int32_t top_k, int32_t* top_ids, float* top_logp, void* stream);

/*
 * Gradient of logp and entropy with respect to the logits, given d/dlogp [T] and d/dentropy [T] of a scalar:
 *   dlogits[t][j] = scale * ( dlogp[t] * (1[j = y] - p_j) - dentropy[t] * p_j * (log p_j + entropy[t]) )
 * with lse and entropy as the forward call wrote them.  dlogp is NULL (with targets NULL) or dentropy is NULL
 * (entropy is not read then) for "zero".  dlogp[t] is not used where y < 0.  p_j = exp(z_j - lse) with z_j rounded
 * to fp32, as lse is: good to |lse| 2^-23 relatively.  A row of nothing but -Inf (or whose lse is -Inf) gets zeros, a row whose lse
 * is NaN or +Inf gets NaN.  dlogits has the logits' type; dlogits == logits with the same stride
 * is legal (in place).
 */
cocodc_status cocodc_lm_logprobs_grad(cocodc_lm* lm, const void* logits, int32_t type, int64_t stride, int64_t T,
                                      int64_t V, const void* targets, int32_t targets_type, float scale,
                                      const float* lse, const float* entropy, const float* dlogp,
                                      const float* dentropy, void* dlogits, int64_t dlogits_stride, void* stream);

/*
 * The calls above with their arguments in one record of 64-bit words, for bindings that pay for every argument of a
 * foreign call (sixteen of them cost a microsecond more than one): record[0] is the operator, then come its
 * arguments in the order of its declaration, without the handle: pointers and integers as int64_t, scale as a
 * double.  Returns what the call returns; INVALID_ARG for an unknown operator.
 */
typedef enum {
  COCODC_LM_EMBED = 0, COCODC_LM_EMBED_GRAD = 1, COCODC_LM_GLU = 2, COCODC_LM_GLU_GRAD = 3, COCODC_LM_LOGPROBS = 4,
  COCODC_LM_LOGPROBS_GRAD = 5
} cocodc_lm_operator;
cocodc_status cocodc_lm_submit(cocodc_lm* lm, const void* record);

#ifdef __cplusplus
}
#endif
#endif /* COCODC_LM_H */
