/*
 * llmoe -- expert-layer operators for one MI355X (gfx950): C ABI, same library
 * and status codes as llcoll.h.
 *
 * What an expert-parallel layer computes between its AllGather and its
 * ReduceScatter, one rank at a time: top-k routing, tokens sorted by expert
 * (dispatch) and summed back with their weights (combine), and the experts'
 * matrix products with bias, activation and residual in their epilogue.  One
 * group makes the same product an ordinary dense layer (the column- and
 * row-parallel layers around an AllReduce).  Every operator has its gradient.
 *
 * Conventions, where a function does not say otherwise:
 *   - Pointers are device pointers, aligned to their element; `stream` is a
 *     hipStream_t passed as void* (NULL = the null stream).  Leading
 *     dimensions (ld*) are in elements and at least the row's length.  Rows
 *     at 16-byte-aligned addresses run on the vector path; every other
 *     alignment and length is served too.
 *   - `dt` (LL_F32 or LL_BF16) is the type of matrices and rows.  Routing
 *     weights and biases on keys are binary32, indices are int32.
 *   - Sums, softmax statistics and activations are computed in binary32 and
 *     rounded once to the output's type (round to nearest even).  Results do
 *     not depend on timing: no output is accumulated with atomics.
 *   - Outputs must not overlap inputs unless stated.  Nothing is allocated,
 *     synchronised or kept between calls; arguments are checked before any
 *     HIP call.
 *   - An extent of zero (tokens, rows) is LL_OK and writes what is left to
 *     write: offsets, zero gradients.  Pointers to nothing may be NULL then.
 *
 * Errors: LL_ERR_INVALID (a null or misaligned pointer, a leading dimension
 * below the row's length, a bad enum value, k outside [1, 32] or above
 * experts), LL_ERR_UNSUPPORTED (unknown dtype, experts or groups above 1024,
 * 2^24 tokens or more, features of a product above 2^20, its leading dimensions
 * above 2^21, a gated ll_linear with a weight of more than 0xF0000000 bytes
 * (out * ldw) a group, other extents past 2^31 - 1), LL_ERR_SCRATCH (workspace
 * too small), LL_ERR_HIP.
 */
#ifndef LLMOE_H
#define LLMOE_H

#include <stddef.h>
#include <stdint.h>

#include "llcoll.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LL_MOE_MAX_EXPERTS 1024
#define LL_MOE_MAX_K 32

/* ---- routing ---- */
typedef enum { LL_SCORE_SOFTMAX = 0, LL_SCORE_SIGMOID = 1 } ll_score;

/* Top-k routing.  The key of expert e is logits[t, e] (+ bias[e] when bias is
 * not NULL), a binary32 sum; the k largest keys are chosen in descending
 * order, ties to the lowest index.  A key of -Infinity or NaN is never
 * chosen: where fewer than k remain, ids ends in -1 with weight 0.  The score
 * of an expert is the softmax of the logits over all experts, or their
 * sigmoid (without the bias; a NaN logit counts as -Infinity).  weights[t, j]
 * = scale * score, divided by the sum of the row's chosen scores when
 * normalise is not 0 (0 if that sum is 0; scores too small for binary32 but
 * not for binary64 have their shares).  ids, weights: [tokens, k].
 *
 * The bias moves the logit.  Routers that balance their experts by a selection
 * bias on the score choose other experts, since the scores are not linear in
 * the logits: for those pass the scores (binary32) as logits, which makes the
 * key score + bias, take the ids from that call and the weights from the
 * scores; ll_moe_route_grad takes these ids with the logits as it does any. */
int ll_moe_route(const void *logits, size_t ld, size_t tokens, int experts, int k, ll_dtype dt, const float *bias,
                 ll_score score, int normalise, float scale, int32_t *ids, float *weights, void *stream);

/* Gradient of the weights of ll_moe_route (same arguments, its ids) with
 * respect to the logits: dlogits[t, e] in dt, every element written.  An id
 * outside [0, experts) contributes nothing; the ids of a row are distinct. */
int ll_moe_route_grad(const void *logits, size_t ld, size_t tokens, int experts, int k, ll_dtype dt, ll_score score,
                      int normalise, float scale, const int32_t *ids, const float *dweights, void *dlogits,
                      size_t ldd, void *stream);

/* ---- dispatch and combine ---- */

/* Workspace of ll_moe_dispatch, in bytes (4-byte aligned; may be 0). */
int ll_moe_dispatch_bytes(size_t tokens, int k, int experts, size_t *bytes);

/* Sort the tokens*k (token, choice) pairs whose id lies in [first, first +
 * experts) by expert, stable in (token, choice) order, and copy the tokens'
 * rows into that order.  offsets[0..experts]: rows of local expert e are
 * [offsets[e], offsets[e+1]).  slots[i] = token*k + choice of sorted row i,
 * -1 for i >= offsets[experts]; rows[token*k + choice] = the sorted row, or
 * -1 if the choice is not local.  y[i] = x[slots[i] / k] for i <
 * offsets[experts]; the remaining rows of y (it has tokens*k) are left as
 * they are.  x NULL (then y NULL): sort only.  No array may overlap another
 * (LL_ERR_INVALID).  The gradient of y with respect to x is ll_moe_combine
 * with weights NULL. */
int ll_moe_dispatch(const int32_t *ids, size_t tokens, int k, int first, int experts, const void *x, size_t ldx,
                    size_t features, ll_dtype dt, int32_t *offsets, int32_t *slots, int32_t *rows, void *y, size_t ldy,
                    void *workspace, size_t workspace_bytes, void *stream);

/* out[t] = residual[t] + sum over j of weights[t, j] * y[rows[t, j]], in
 * ascending j, the residual last; choices whose row is outside [0, nrows) are
 * left out, so a token without any gets its residual, or 0.  weights NULL:
 * all 1.  residual NULL: none; it may be out itself. */
int ll_moe_combine(const void *y, size_t ldy, size_t nrows, const int32_t *rows, const float *weights,
                   const void *residual, size_t ldr, size_t tokens, int k, size_t features, ll_dtype dt, void *out,
                   size_t ldo, void *stream);

/* Gradient of ll_moe_combine: dy[rows[t, j]] = weights[t, j] * dout[t] and
 * dweights[t, j] = <dout[t], y[rows[t, j]]> (0 where the row is left out).
 * Rows of dy that no choice names are left as they are; no row is named
 * twice.  weights NULL: all 1; dweights NULL (then y may be NULL): not
 * wanted.  The gradient with respect to the residual is dout. */
int ll_moe_combine_grad(const void *dout, size_t ldd, const void *y, size_t ldy, size_t nrows, const int32_t *rows,
                        const float *weights, size_t tokens, int k, size_t features, ll_dtype dt, void *dy,
                        size_t lddy, float *dweights, void *stream);

/* ---- grouped matrix products ---- */

/* Activations.  GELU is the exact one, x Phi(x), relatively accurate far below
 * zero too.  The gated ones take pre-activations of two halves [a, u] and
 * return silu(a) * u, gelu(a) * u. */
typedef enum {
  LL_ACT_NONE = 0,
  LL_ACT_RELU = 1,
  LL_ACT_GELU = 2,
  LL_ACT_SILU = 3,
  LL_ACT_SWIGLU = 4,
  LL_ACT_GEGLU = 5
} ll_act;

/* A product's shape.  Row r of x belongs to group g where offsets[g] <= r <
 * offsets[g+1] (device memory, ascending from 0, offsets[groups] <= rows, as
 * ll_moe_dispatch writes them); rows from offsets[groups] on belong to none
 * and their results are left as they are.  offsets NULL: one group of all
 * rows (groups must be 1).  Group g's weight is [out, in] at w + g*wstride,
 * its bias `out` elements at bias + g*out.  Fill with ll_linear_desc_init
 * (contiguous rows), then change leading dimensions. */
typedef struct {
  uint32_t size;   /* sizeof(ll_linear_desc), set by ll_linear_desc_init */
  ll_dtype dt;
  ll_act act;
  int32_t groups;
  size_t rows, in, out;
  const int32_t *offsets;
  size_t ldx;      /* x: in elements a row */
  size_t ldw;      /* weight rows: in elements */
  size_t wstride;  /* between groups' weights */
  size_t ldy;      /* y, and dz / dy of the gradients */
  size_t ldz;      /* z */
  size_t ldr;      /* residual */
} ll_linear_desc;

/* Sets every field: contiguous rows, offsets NULL.  ldy is `out`, half of it
 * for a gated activation (of ll_linear); ldz is `out`. */
int ll_linear_desc_init(ll_linear_desc *d, ll_dtype dt, ll_act act, int groups, size_t rows, size_t in, size_t out);

/* Which product a workspace is for. */
typedef enum { LL_LINEAR_FORWARD = 0, LL_LINEAR_GRAD_X = 1, LL_LINEAR_GRAD_W = 2 } ll_linear_pass;

/* Workspace (bytes, 16-byte aligned) with which the product runs as fast as it
 * can; 0 where it needs none.  Every product also runs without one. */
int ll_linear_bytes(const ll_linear_desc *d, ll_linear_pass pass, size_t *bytes);

/* y[r] = act(x[r] w[g]^T + bias[g]) + residual[r].  With a gated activation
 * `out` is even and y and residual have out/2 columns.  z (may be NULL)
 * receives the pre-activations x w^T + bias, [rows, out], for the backward
 * pass.  bias, residual may be NULL; residual may be y itself. */
int ll_linear(const ll_linear_desc *d, const void *x, const void *w, const void *bias, const void *residual, void *y,
              void *z, void *workspace, size_t workspace_bytes, void *stream);

/* dx[r] = dz[r] w[g], for dz [rows, out] (ldy) and dx [rows, in] (ldx).  With
 * act != LL_ACT_NONE the result is taken on through that activation, the one
 * of the layer below whose output is x: z (ldz) holds its pre-activations
 * [rows, in], or [rows, 2*in] for a gated one, and dx their gradient in the
 * same shape (ldx at least its width).  z NULL only with LL_ACT_NONE. */
int ll_linear_grad_x(const ll_linear_desc *d, const void *dz, const void *w, const void *z, void *dx, void *workspace,
                     size_t workspace_bytes, void *stream);

/* dw[g] = dz[rows of g]^T x[rows of g], [out, in] at ldw and wstride, and
 * dbias[g] = the sum of dz over those rows ([groups, out]; NULL: not wanted).
 * A group without rows gets zeros.  d->act is not used.  flags:
 * LL_GRAD_F32: dw and dbias are binary32 whatever dt is; LL_GRAD_ADD: the
 * gradients are added to what dw and dbias hold. */
#define LL_GRAD_F32 0x1u
#define LL_GRAD_ADD 0x2u
int ll_linear_grad_w(const ll_linear_desc *d, const void *dz, const void *x, void *dw, void *dbias, uint32_t flags,
                     void *workspace, size_t workspace_bytes, void *stream);

/* dz = dy * act'(z), elementwise over [rows, features] (dy), for an
 * activation whose layer above is not a product.  Gated: z and dz have
 * 2*features columns.  dz may be dy (ungated) or z. */
int ll_act_grad(const void *dy, size_t lddy, const void *z, size_t ldz, size_t rows, size_t features, ll_dtype dt,
                ll_act act, void *dz, size_t lddz, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* LLMOE_H */
