/*
 * flux_norm.h - C ABI of the MI355X (gfx950) root-mean-square norm of a transformer's residual stream, with the addition in front of it
 * and its backward pass.  It stands between the two fused GEMMs of flux.h: X is a slice that flux_gemm_rs left, Y a chunk that
 * flux_ag_gemm gathers; and in front of the 4-bit operators of flux_ffn.h, which read Y in blocks.
 *
 *   flux_norm            S = X + R,  r = 1 / sqrt(mean(S^2) + eps),  Y = S r W         per row of K numbers
 *   flux_norm_backward   dR = r (dY W - S r^2 mean(dY W S)) + dS,   dW = sum over rows of dY S r
 *   flux_mx8_dequantize  what blocks of 8-bit numbers stand for
 *
 * Conventions: those of flux_ffn.h (the same library).  Rows need no alignment beyond their type's, K and pitches may be odd.
 */
#ifndef FLUX_NORM_MI355_H_
#define FLUX_NORM_MI355_H_

#include <stddef.h>
#include <stdint.h>
#include "flux_ffn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What Y is: numbers, or blocks of 32 along a row (OCP Microscaling Formats 1.0, "MXFP4" and "MXFP8") laid out as flux_mx4_quantize lays them out.
 * 8 bits (E4M3): the largest magnitude's exponent less 8 is the block's, numbers are held at 448, and a row of numbers takes 32 bytes per
 * block: flux_mx8_row_bytes.  Scales as with 4 bits (flux_mx4_scale_row_bytes).  (8 bits are for a caller who moves Y: the products of flux_ffn.h read 4 bits.) */
typedef enum { FLUX_NORM_BF16 = 0, FLUX_NORM_F32 = 1, FLUX_NORM_MX4 = 2, FLUX_NORM_MX8 = 3 } flux_norm_out_t;

/* M >= 1; 1 <= K <= 2^30; pitches at least a row long; every matrix below 2^31 elements. */
typedef struct flux_norm {
  int32_t M, K;             /* rows (tokens), their width                                       */
  int32_t x_dtype;          /* of X and dX (flux_dtype_t)                                       */
  int32_t s_dtype;          /* of the stream: R, S, dS, dR                                      */
  int32_t w_dtype;          /* of W                                                             */
  int32_t out;              /* of Y (flux_norm_out_t), and of dY, which is in numbers           */
  int32_t dw_dtype;         /* of dW                                                            */
  int32_t dw_accumulate;    /* 1: dW is added to what the buffer holds (micro-batches)          */
  float eps;                /* >= 0, finite                                                     */
  int32_t reserved;         /* must be 0                                                        */
  int64_t ldx, lds, ldy;    /* pitches in elements, 0 = K: X and dX; R, S, dS and dR; Y and dY (in numbers) */
} flux_norm_t;

/* The sum is taken in fp32 and rounded to s_dtype once; the norm is that of S as it is stored, in fp32, rounded once.
 *   X [M,K]           x_dtype
 *   R, S [M,K]        s_dtype; S may be R itself.  Both or neither (NULL): without them S is X, and nothing but Y is written
 *   W [K]             w_dtype
 *   Y                 [M,K] with pitch ldy; or blocks (16-byte aligned), then with
 *   scales            their scales (16-byte aligned; NULL otherwise).  Numbers are in blocks what they are in fp32, rounded once
 *   rstd [M]          fp32: r of every row, for the backward pass; may be NULL */
int flux_norm(const flux_norm_t* p, const void* X, const void* R, const void* W, void* S, void* Y, void* scales, float* rstd, void* stream);

/* Bytes of workspace of the backward pass (0 for a problem that is refused).  It may be shared with the operators of flux_ffn.h, as they share theirs. */
size_t flux_norm_workspace_bytes(const flux_norm_t* p);

/* Gradients of flux_norm, whose S and rstd are read.  (Where there was no R, S is X, and s_dtype and lds have to be X's.)
 *   dY [M,K]          gradient of Y, bf16 or fp32 as `out` says; FLUX_ERR_UNSUPPORTED where Y is in blocks
 *   dS [M,K]          s_dtype: the gradient of S from what else reads it, or NULL for none
 *   dR [M,K]          s_dtype: the gradient of R, and of X; may be dS itself.  May be NULL
 *   dX [M,K]          x_dtype: the same numbers in X's type.  May be NULL
 *   dW [K]            dw_dtype, summed over rows in fp32, in an order that depends on M and K alone.  May be NULL
 *   workspace         >= flux_norm_workspace_bytes(p) bytes; NULL if dW is NULL */
int flux_norm_backward(const flux_norm_t* p, const void* dY, const void* S, const void* W, const float* rstd, const void* dS,
                       void* dR, void* dX, void* dW, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of a row of K 8-bit numbers in blocks of 32. */
size_t flux_mx8_row_bytes(int32_t K);

/* dst [rows,K] bf16 or fp32 with pitch `ld`, any alignment that its type has: what the blocks stand for, rounded once.  K up to 2^30. */
int flux_mx8_dequantize(int32_t rows, int32_t K, const void* q, const void* scales, int32_t dst_dtype, void* dst, int64_t ld, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FLUX_NORM_MI355_H_ */
