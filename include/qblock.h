/*
 * qblock.h -- C ABI of the operators of a block that is trained with its
 * activations kept in 8 bits, beside the quadratic layers of qlayer.h, the batch
 * normalization of qnet.h and the first-order layer of qhead.h: checkpoints of
 * activations in 8 bits, group normalization with an activation over channels-last
 * maps, and the gated layer (two projections, an activation, their product).  The
 * memory modes of arXiv 2204.01701, section 4.3, are to save what the backward
 * reads or to recompute it; a checkpoint is the third: saved at half (bf16) or a
 * quarter (float32) of its bytes.
 *
 * Conventions: as in qhead.h (device pointers owned by the caller, work enqueued on
 * `stream`, arguments validated before the first launch, status codes,
 * caller-allocated workspaces whose contents on entry are irrelevant and which two
 * calls under way must not share, no device memory allocated, nothing kept between
 * calls, 64-bit offsets, pointers aligned to their elements only, workspaces to 16
 * bytes, results independent of the order of execution).  Matrices and maps are
 * dense unless a row stride is named.
 */
#ifndef QBLOCK_H
#define QBLOCK_H

#include <stddef.h>
#include <stdint.h>

#include "qhead.h"
#include "qlayer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------
 * Checkpoint of a matrix in 8 bits.  The `cols` values of a row are cut into blocks
 * of QBLOCK_KEEP neighbours (the last one may be shorter).  With amax the largest
 * magnitude in a block,
 *     E = the least integer >= -126 with amax <= 127 * 2^E,
 *     q = x / 2^E rounded to the nearest integer (halves to even),   x8 = q 2^E.
 * |x - x8| <= 2^E / 2 <= amax / 127 (for 2^E from 2^-125 to 2^121).  x8 is exact in
 * bfloat16 and float32: reading a checkpoint rounds nothing.  At the very end of the
 * range (E = 122) |q| is at most 63, so that x8 is finite: magnitudes above 63.5 2^122
 * read back as 63 2^122, up to a whole 2^122 less.
 *   q : rows x cols int8, dense.   e : rows x ceil(cols / 32) uint8, dense: E + 127.
 * A block with a NaN or an infinity has e = 255 and reads back as NaN throughout.
 * An e that no pack writes (0, 250 .. 254) reads as the power of two e - 127, 0 as 0.
 * x : rows x cols of `dtype`, row stride ld.  rows >= 0 (below 2^47 values in all),
 * 1 <= cols <= 2^31 - 65536.
 * ------------------------------------------------------------------------- */
#define QBLOCK_KEEP 32

typedef struct {
    long long rows;
    int cols;
    long long ld;
    ql_dtype dtype;
} qblock_keep_desc;

ql_status qblock_pack8(const qblock_keep_desc *desc, const void *x, int8_t *q, uint8_t *e, void *stream);
ql_status qblock_unpack8(const qblock_keep_desc *desc, const int8_t *q, const uint8_t *e, void *x, void *stream);

/* ---------------------------------------------------------------------------
 * Group normalization with an activation.  x and y: n x hw x c (channels last: an
 * N x H x W x C map, or rows with hw = 1); group g has the channels g c / groups ..
 * (g + 1) c / groups - 1.  Over the hw pixels and the channels of a group of a sample
 *     mean, var (divided by the count),   rstd = 1 / sqrt(var + eps),
 *     xh = (x - mean) rstd,   z = gamma xh + beta,   y = act(z)
 *   gamma, beta : c float32, or NULL (1 and 0).
 *   mean, rstd  : n x groups float32, for the backward; either may be NULL.
 *   q, e        : NULL, or the checkpoint of x as (n hw) x c, written on the way.
 * y may be x.  Statistics are float32, from sums of differences to a mean (large
 * offsets of a group cancel before they are squared); where a sum of (x - mean)^2
 * overflows, rstd is 0, and where a sum of x does, NaN.  A NaN or infinity reaches its group of its sample and nothing else.
 *
 * Backward, with dy = dl/dy:
 *     dz = dy act'(z),   dbeta = sum dz,   dgamma = sum dz xh   (over samples and pixels)
 *     t = gamma dz,   dx = rstd (t - avg(t) - xh avg(t xh))     (averages over the group)
 * x is given as it was, or (x NULL) as its checkpoint q, e: xh and z are then formed
 * from x8 with the mean and rstd of the forward.  dx : of `dtype`, may be dy or x;
 * dgamma, dbeta : c float32; each of the three may be NULL (not all, but for n = 0).
 * relu'(0) = 0.  n >= 0 (with n = 0 dgamma and dbeta are 0); hw, c >= 1; groups divides c;
 * eps > 0 and finite.  QL_EUNSUPPORTED: n or hw above 2^31 - 65536, c above 2^20,
 * 2^47 values or more.
 * ------------------------------------------------------------------------- */
typedef struct {
    int n, hw, c, groups;
    ql_dtype dtype;
    ql_act act;
    float eps; /* (the backward does not look at it) */
} qblock_norm_desc;

size_t qblock_norm_fwd_workspace_size(const qblock_norm_desc *desc);
ql_status qblock_norm_fwd(const qblock_norm_desc *desc, const void *x, const float *gamma, const float *beta, void *y,
                          float *mean, float *rstd, int8_t *q, uint8_t *e, void *workspace, size_t workspace_bytes,
                          void *stream);
size_t qblock_norm_bwd_workspace_size(const qblock_norm_desc *desc);
ql_status qblock_norm_bwd(const qblock_norm_desc *desc, const void *dy, const void *x, const int8_t *q, const uint8_t *e,
                          const float *gamma, const float *beta, const float *mean, const float *rstd, void *dx,
                          float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * Gated layer:
 *     g = x wg^T + bg,   u = x wu^T + bu,   h = act(g) o u
 *   x : m x k (ldx);  wg, wu : n x k, both with the row stride ldw;  h : m x n (ldh);
 *   all of `dtype`.  bg, bu : n float32, each may be NULL.
 *   z : NULL, or 2 x m x n of `dtype`: g and behind it u, for the backward.
 *   q, e : NULL, or the checkpoint of z as (2 m) x n, from the unrounded g and u.
 * Products are accumulated, and the rest computed, in float32; h is rounded once
 * (from the unrounded g and u), and so is z.
 *
 * Backward, with dh = dl/dh (m x n, ldh), from z or (z NULL) its checkpoint:
 *     dg = dh o u o act'(g),   du = dh o act(g)
 *     dx = dg wg + du wu,   dwg = dg^T x,   dwu = du^T x,   dbg, dbu = column sums
 *   dx : m x k dense of `dtype`; dwg, dwu : n x k dense of `dtype`, or float32
 *   (dw_f32), both or neither; dbg, dbu : n float32, each may be NULL.  Not all of
 *   them NULL (but for m = 0).  x is needed for the weights' gradients, wg and wu for dx.  In bf16, dg
 *   and du are rounded once to bf16 as operands of the products; the column sums take
 *   them unrounded.  relu'(0) = 0.
 * Operands whose rows are not whole, aligned 16-byte vectors are copied into the
 * workspace; the query covers what the descriptor shows, and misaligned pointers if
 * `unaligned` is set.  A misaligned pointer among x, wg, wu without it: QL_EINVAL,
 * but where k is not whole 16-byte vectors (which are copied in any case), and for the
 * forward of up to QBLOCK_FEW_ROWS rows without a checkpoint, which reads
 * any layout and needs no workspace, whatever the query (which does not know of the
 * checkpoint) returns.
 * Sizes: m >= 0 (m = 0: zeros in the weights' and bias gradients), k, n >= 1;
 * QL_EUNSUPPORTED for m above 2^31 - 65536, or k or n above 2^19.
 * ------------------------------------------------------------------------- */
#define QBLOCK_FEW_ROWS 16

typedef struct {
    int m, k, n;
    long long ldx, ldw, ldh;
    ql_dtype dtype;
    ql_act act;
    int unaligned; /* nonzero: one of x, wg, wu may not be 16-byte aligned (sizes the workspace for copies) */
    int dw_f32;    /* backward, nonzero: dwg and dwu are float32 though the rest is bf16 */
} qblock_gated_desc;

size_t qblock_gated_fwd_workspace_size(const qblock_gated_desc *desc);
ql_status qblock_gated_fwd(const qblock_gated_desc *desc, const void *x, const void *wg, const void *wu, const float *bg,
                           const float *bu, void *h, void *z, int8_t *q, uint8_t *e, void *workspace,
                           size_t workspace_bytes, void *stream);
size_t qblock_gated_bwd_workspace_size(const qblock_gated_desc *desc);
ql_status qblock_gated_bwd(const qblock_gated_desc *desc, const void *x, const void *wg, const void *wu, const void *dh,
                           const void *z, const int8_t *q, const uint8_t *e, void *dx, void *dwg, void *dwu, float *dbg,
                           float *dbu, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* QBLOCK_H */
