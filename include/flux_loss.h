/*
 * flux_loss.h - C ABI of the MI355X (gfx950) softmax cross entropy of a vocabulary projection, with its backward pass.  The logits
 * Z = X W^T are never kept: the forward pass leaves three numbers a row, the backward pass takes Z anew, a piece of the vocabulary at a time.
 * A rank of a tensor-parallel group may hold some columns of the vocabulary: flux_loss_join puts the ranks' numbers together.
 *
 *   flux_loss            lse = log sum_v exp(Z_v),  logit = Z_target,  loss = lse - logit        Z = X W^T, X [M,K], W [V,K]
 *   flux_loss_join       the same over the columns of R ranks, out of each rank's lse and logit
 *   flux_loss_backward   dZ = dloss (exp(Z - lse) - [v = target]),  dX = dZ W,  dW = dZ^T X
 *
 * Conventions: those of flux_ffn.h (the same library).
 */
#ifndef FLUX_LOSS_MI355_H_
#define FLUX_LOSS_MI355_H_

#include <stddef.h>
#include <stdint.h>
#include "flux_ffn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { FLUX_LOSS_FORWARD = 0, FLUX_LOSS_BACKWARD = 1 } flux_loss_op_t;
typedef enum { FLUX_TARGET_I32 = 0, FLUX_TARGET_I64 = 1 } flux_target_t;

/* M, V >= 1; M <= 2^27, M V <= 2^36; K % 8 == 0, K <= 2^28 for gradients; pitches multiples of 8, at least a row long; X, W, dX and dW 16-byte aligned; every matrix below 2^31
 * elements.
 * A row whose target is not in [0, vocab) does not count: its loss is 0 and it adds nothing to a gradient, whatever its lse and dloss are (but X and W have to be finite: dW is
 * a sum over all rows of X, dX over all of W, and 0 times infinity is none).  So is a row whose dloss is 0.  A target of another rank's columns gives a logit of 0 here. */
typedef struct flux_loss {
  int32_t M, V, K;          /* tokens, this rank's columns of the vocabulary, model width       */
  int32_t target_dtype;     /* flux_target_t                                                    */
  int64_t v0, vocab;        /* first of this rank's columns; columns of all ranks (0: v0 + V)   */
  int32_t dloss_one;        /* 1: dloss is one number, for every row; 0: a number a row         */
  int32_t dx_dtype;         /* of dX (flux_dtype_t)                                             */
  int32_t dw_dtype;         /* of dW                                                            */
  int32_t dw_accumulate;    /* 1: dW is added to what the buffer holds (micro-batches)          */
  int64_t ldx, ldw;         /* pitches in elements, 0 = K: X and dX; W and dW                   */
  int32_t piece;            /* columns of the vocabulary that the backward pass takes at a time: 0 = library picks (up to 256 MiB of dZ); else a
                               multiple of 64, more than V counts as V.  M times a piece, below 2^31, is what the workspace holds of dZ */
  int32_t tile_config;      /* of the forward pass and of Z in the backward pass, as in flux_glu_t (flux_ffn_tile_config_info) */
  int32_t split_k;          /* as in flux_glu_t                                                 */
  int32_t reserved;         /* must be 0                                                        */
} flux_loss_t;

/* As flux_glu_workspace_bytes; one workspace serves the operators of flux_ffn.h and of this header alike. */
size_t flux_loss_workspace_bytes(int op, const flux_loss_t* p);

/* Products accumulate in fp32, and everything behind them is fp32.
 *   X [M,K], W [V,K]  bf16
 *   target [M]        target_dtype, numbers of the whole vocabulary
 *   lse, logit [M]    fp32, over this rank's columns
 *   loss [M]          fp32; may be NULL, as on a rank that holds some of the columns (what it gets there is lse - logit of its own) */
int flux_loss(const flux_loss_t* p, const void* X, const void* W, const void* target, float* lse, float* logit, float* loss,
              void* workspace, size_t workspace_bytes, void* stream);

/* The whole vocabulary's lse, logit and loss out of those of R ranks, 1 <= R <= FLUX_MAX_RANKS.  lses, logits: HOST arrays of R device pointers,
 * read during the call only.  Any of the results may be NULL; one may be one of the inputs.  Of the problem M, target_dtype and vocab
 * (v0 + V) are read. */
int flux_loss_join(const flux_loss_t* p, int32_t R, const float* const* lses, const float* const* logits, const void* target,
                   float* lse, float* logit, float* loss, void* stream);

/* Gradients of sum over rows of dloss * loss.  lse is that of the whole vocabulary.  dZ / D, D the largest |dloss| of the rows that count, is taken in fp32 and
 * rounded to bf16 once, as operand of the two products, which accumulate in fp32, take the factor D, and are rounded once at the end.  (Rows whose |dloss|
 * is below 2^-100 of the largest lose digits.)  So dX and dW in fp32 hold dZ's rounding, up to half a step of bf16 (2^-8) of every term: fp32 spares them a rounding of their own, and
 * adds up micro-batches without one.  Off by, in parts of their norm: 2e-4 to 8e-4 with one dloss for all rows, 1.4e-3 to 1.7e-3 with one a row; in bf16 1.7e-3 and 2.3e-3.
 *   dloss             fp32, [M] or one number
 *   dX [M,K]          dx_dtype: this rank's part of the sum over ranks.  May be NULL
 *   dW [V,K]          dw_dtype.  May be NULL
 *   workspace         >= flux_loss_workspace_bytes(FLUX_LOSS_BACKWARD, p) bytes */
int flux_loss_backward(const flux_loss_t* p, const void* X, const void* W, const void* target, const float* lse, const float* dloss,
                       void* dX, void* dW, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FLUX_LOSS_MI355_H_ */
