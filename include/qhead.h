/*
 * qhead.h -- C ABI of the operators at the end of a network, beside the
 * quadratic layers of qlayer.h: the first-order fully-connected layer with its
 * epilogue, the log probabilities of given tokens (or class labels) with the
 * entropy and the most likely alternatives, and the distillation of a student
 * from a teacher's top logits; each with its gradients.
 *
 * Conventions: as in qlayer.h (device pointers owned by the caller, work
 * enqueued on `stream`, arguments validated before the first launch, status
 * codes, caller-allocated workspaces whose contents on entry are irrelevant,
 * no device memory allocated, nothing kept between calls), with these
 * differences:
 *  - Matrices are row-major with a row stride in elements (ld >= row length),
 *    so that rows may be cut out of wider tensors; what lies between a row's
 *    end and the next row's start is neither read nor written.
 *  - Pointers need the alignment of their element only (bf16 2, float 4,
 *    int64 8 bytes); workspaces 16 bytes.
 *  - A weight gradient is of the operands' dtype unless the caller asks for
 *    float32 (qlayer.h: always float32).
 *  - Row counts may be 0: the call then launches what zero rows leave to do
 *    (zeros in dw and db) and returns QL_OK.
 *  - Offsets are 64-bit: a matrix may hold more than 2^31 elements.
 *  - Results are deterministic: sums are taken in a fixed order, equal values
 *    rank by the lower index.
 */
#ifndef QHEAD_H
#define QHEAD_H

#include <stddef.h>
#include <stdint.h>

#include "qlayer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------
 * First-order fully-connected layer:
 *     z = x w^T + b,   y = act(z) + r
 *   x : m x k (ldx), w : n x k (ldw), r : m x n (ldr, or NULL), y : m x n (ldy),
 *   all of `dtype`; b : n float32, or NULL.  z : m x n dense of `dtype`, written
 *   if not NULL (what the backward of an activation needs).
 *   QL_ACT_GELU is z Phi(z) with the error function, QL_ACT_GELU_TANH its
 *   tanh approximation, QL_ACT_SILU z / (1 + e^-z).
 * Products are accumulated, and the epilogue computed, in fp32; z and y are
 * each rounded once (y from the unrounded z).  y may be r.
 *
 * Backward, with dy = dl/dy (m x n, ldy), from the stored z:
 *     dz = dy o act'(z),  dx = dz w,  dw = dz^T x,  db = column sums of dz
 *   (dr = dy).  dx : m x k dense of `dtype`; dw : n x k dense of `dtype`, or float32 (dw_f32); db : n float32.
 *   Each of dx, dw, db may be NULL (not all).  z may be NULL for QL_ACT_NONE;
 *   x is needed for dw, w for dx.  In bf16, dz is rounded once to bf16 as the
 *   operand of both products; db sums it unrounded.  relu'(0) = 0.
 * Operands whose rows are not whole, aligned 16-byte vectors are copied into the
 * workspace where a product is large enough to gain by it; the query covers the
 * copies that the descriptor shows (odd strides and sizes), and those of
 * misaligned pointers if `unaligned` is set.  With a misaligned pointer and the
 * flag unset results keep their accuracy, at lower speed.
 * Sizes: m >= 0, k >= 1, n >= 1; QL_EUNSUPPORTED within 65536 of 2^31.
 * ------------------------------------------------------------------------- */
typedef enum { QL_ACT_NONE = 0, QL_ACT_RELU = 1, QL_ACT_GELU = 2, QL_ACT_GELU_TANH = 3, QL_ACT_SILU = 4 } ql_act;

typedef struct {
    int m, k, n;
    long long ldx, ldw, ldr, ldy;
    ql_dtype dtype;
    ql_act act;
    int unaligned; /* nonzero: one of x, w, dy may not be 16-byte aligned (sizes the workspace for copies) */
    int dw_f32;    /* backward, nonzero: dw is float32 though the rest is bf16 */
} qhead_linear_desc;

size_t qhead_linear_fwd_workspace_size(const qhead_linear_desc *desc);
ql_status qhead_linear_fwd(const qhead_linear_desc *desc, const void *x, const void *w, const float *b, const void *r,
                           void *y, void *z, void *workspace, size_t workspace_bytes, void *stream);
size_t qhead_linear_bwd_workspace_size(const qhead_linear_desc *desc);
ql_status qhead_linear_bwd(const qhead_linear_desc *desc, const void *x, const void *w, const void *dy, const void *z,
                           void *dx, void *dw, float *db, void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * Rows of logits: `rows` rows of `vocab` values of `dtype`, row stride ld.
 * Statistics and sums are fp32.  The temperature T is finite and > 0, with
 * log2(e) / T and, for the distillation, T^2 finite in float32 (T from about
 * 4.3e-39, and up to about 1.8e19).
 * ------------------------------------------------------------------------- */
typedef struct {
    int rows, vocab;
    long long ld;  /* row stride of the logits */
    int top;       /* K: alternatives (0 .. min(vocab, QHEAD_MAX_TOP)), or the teacher's places per row */
    ql_dtype dtype;
    float temperature;
    float alpha;   /* distillation: share of the teacher's term, 0 .. 1 (ignored by the log probabilities) */
    int teacher_f32; /* distillation: nonzero where t_logits are float32 though the logits are bf16 */
} qhead_rows_desc;

#define QHEAD_MAX_TOP 128

/* ---------------------------------------------------------------------------
 * Log probabilities of given tokens under softmax(logits / T):
 *     lse = log sum_j e^{z_j / T},   logp = z_t / T - lse,
 *     entropy = -sum_j p_j log p_j,   p_j = e^{z_j / T - lse}
 *   target   : rows int64.  Negative: no token, logp = 0 and no gradient from
 *              it.  At or above vocab: logp = NaN (and no gradient).
 *   logp, lse, entropy : rows float32; lse and entropy may be NULL.
 *   stats    : rows x 2 float32 for the backward, or NULL.
 *   top_logp, top_ids : rows x K float32 / int64: the K most likely tokens, by
 *              falling value, equal values by rising index; both NULL if K = 0.
 * A row whose logits are all -inf has lse = -inf, logp = -inf, entropy = 0,
 * alternatives 0 .. K-1 at -inf, and a zero gradient.  A NaN or +inf in a row
 * makes its lse, logp, entropy and top_logp NaN; NaN ranks behind all values.
 *
 * Backward, for upstream gradients g of logp and h of entropy (float32, h may
 * be NULL), from the stats and entropy of the forward (entropy NULL if h is):
 *     dz_j = 1/T [ g (1[j = t] - p_j) - h p_j (log p_j + entropy) ]
 *   dlogits : rows x vocab dense of `dtype`; may be the logits if ld == vocab.
 *   A row with a NaN or +inf has a gradient of NaN, unless nothing reaches it:
 *   with h = 0, and g = 0 or no target, a row's gradient is 0 whatever it holds.
 * ------------------------------------------------------------------------- */
size_t qhead_logprobs_fwd_workspace_size(const qhead_rows_desc *desc);
ql_status qhead_logprobs_fwd(const qhead_rows_desc *desc, const void *logits, const int64_t *target, float *logp,
                             float *entropy, float *lse, float *top_logp, int64_t *top_ids, float *stats,
                             void *workspace, size_t workspace_bytes, void *stream);
ql_status qhead_logprobs_bwd(const qhead_rows_desc *desc, const void *logits, const int64_t *target,
                             const float *stats, const float *entropy, const float *g, const float *h, void *dlogits,
                             void *stream);

/* ---------------------------------------------------------------------------
 * Distillation from a teacher's top logits.  With K = desc->top places a row,
 *     q = softmax of the teacher's logits / T over the row's places,
 *     p^T = softmax(logits / T),   p^1 = softmax(logits),
 *     loss = alpha T^2 sum_k q_k (log q_k - log p^T[id_k])
 *            + (1 - alpha) (-log p^1[label])
 *   t_ids    : rows x K int64.  A negative id is an empty place; a row with
 *              only empty places has no teacher's term.  An id at or above
 *              vocab makes the loss NaN (and takes no part in the gradient).
 *              With alpha = 0 neither ids nor t_logits are looked at.
 *              An id may occur more than once in a row: each place counts.
 *   t_logits : rows x K of `dtype`, or float32 (teacher_f32; the alternatives of
 *              qhead_logprobs_fwd are).  -inf is a place of probability 0.
 *   label    : rows int64, or NULL (no label's term).  Negative: a row without
 *              one.  At or above vocab: the loss is NaN, no gradient from it.
 *              With alpha = 1 labels are not looked at.
 *              The label's term has the weight 1 - alpha also where a row has
 *              no teacher's places, and the teacher's alpha where it has no label.
 *   loss     : rows float32.
 *   K may be 0 with NULL t_ids and t_logits (cross entropy alone).
 * Gradient, with the rows' upstream gradients (or weights) g (float32):
 *     dz_j = g [ alpha T (Q p^T_j - q_j) + (1 - alpha) C (p^1_j - 1[j = label]) ]
 *   Q = 1 if the row has a teacher's term, C = 1 if it has a label, else 0;
 *   q_j is the sum over the places with id j.  dlogits : rows x vocab dense of
 *   `dtype`; may be the logits if ld == vocab.
 * _fwd : the loss, and `stats` (rows x 4 float32, or NULL) for _bwd.
 * _bwd : the gradient.
 * _step: both in one call, for a g that is known beforehand: the logits are
 *        read from memory once.
 * A row whose logits are all -inf has p = 0: loss +inf if it has a teacher's
 * place of positive probability or a label, else 0.  A NaN or +inf among the
 * logits of a row with a term makes its loss NaN, and its gradient unless g = 0;
 * a row without a term has a loss and a gradient of 0, and one with g = 0 a
 * gradient of 0, whatever they hold.
 * ------------------------------------------------------------------------- */
size_t qhead_distill_workspace_size(const qhead_rows_desc *desc);
ql_status qhead_distill_fwd(const qhead_rows_desc *desc, const void *logits, const int64_t *t_ids, const void *t_logits,
                            const int64_t *label, float *loss, float *stats, void *workspace, size_t workspace_bytes,
                            void *stream);
ql_status qhead_distill_bwd(const qhead_rows_desc *desc, const void *logits, const int64_t *t_ids, const void *t_logits,
                            const int64_t *label, const float *stats, const float *g, void *dlogits, void *stream);
ql_status qhead_distill_step(const qhead_rows_desc *desc, const void *logits, const int64_t *t_ids,
                             const void *t_logits, const int64_t *label, const float *g, float *loss, void *dlogits,
                             void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* QHEAD_H */
