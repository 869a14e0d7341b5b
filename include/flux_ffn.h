/*
 * flux_ffn.h - C ABI of the MI355X (gfx950) operators of a gated feed-forward block, in bf16 with its backward pass and on
 * 4-bit microscaled operands.  They are what stands between and beside the two fused GEMMs of flux.h: the up
 * projections of a tensor-parallel rank with activation and product in one kernel (its result is the A of flux_gemm_rs), the
 * gradients of the rank's shards, and the same block for serving with weights of 4.25 bits.
 *
 *   flux_glu            H = act(X Wg) * (X Wu)                         X [M,K], H [M,N]
 *   flux_glu_backward   dG = dH * U * act'(G),  dU = dH * act(G)
 *                       dX = dG Wg^T + dU Wu^T,  dWg = X^T dG,  dWu = X^T dU
 *   flux_mx4_quantize / flux_mx4_dequantize    a matrix to 4-bit blocks and back
 *   flux_mx4_gemm       C = A B^T                                      A [M,K], B [N,K] in 4-bit blocks
 *   flux_mx4_glu        H = act(X Wg^T) * (X Wu^T)                     X [M,K], Wg, Wu [N,K] in 4-bit blocks
 *
 * Conventions: those of flux.h.  Matrices are row-major, pitches in elements (0 = packed); every pointer is device memory of
 * the current device that the caller owns; calls validate, enqueue on `stream` (hipStream_t as void*, NULL = the default
 * stream) and return a flux_status_t; nothing is enqueued unless it is FLUX_OK; nothing throws or aborts; no device memory
 * is allocated.  Every call is plain kernel launches on the one stream and may be recorded in a HIP graph.  Outputs must not
 * overlap inputs or each other.  What lies between the end of a row and the next row is neither read nor written.
 * Same inputs, same problem: same bits.
 */
#ifndef FLUX_FFN_MI355_H_
#define FLUX_FFN_MI355_H_

#include <stddef.h>
#include <stdint.h>
#include "flux.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  FLUX_ACT_SILU = 0,        /* g / (1 + exp(-g))                                              */
  FLUX_ACT_GELU = 1,        /* g Phi(g), Phi the normal distribution function                 */
  FLUX_ACT_GELU_TANH = 2    /* g/2 (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3)))                  */
} flux_act_t;

typedef enum { FLUX_GLU_FORWARD = 0, FLUX_GLU_BACKWARD = 1 } flux_glu_op_t;
typedef enum { FLUX_MX4_GEMM = 0, FLUX_MX4_GLU = 1 } flux_mx4_op_t;

/* Problem of flux_glu and flux_glu_backward.  M >= 1; N % 8 == 0; K % 8 == 0; pitches multiples of 8, at least a row long;
 * base pointers 16-byte aligned; every matrix below 2^31 elements. */
typedef struct flux_glu {
  int32_t M, N, K;          /* tokens, hidden columns of this rank, model width                 */
  int32_t act;              /* flux_act_t                                                       */
  int32_t w_is_nk;          /* Wg, Wu (and their gradients) are [N,K], as a linear layer stores them; 0: [K,N] */
  int32_t out_dtype;        /* of H and dX (flux_dtype_t)                                       */
  int32_t dw_dtype;         /* of dWg and dWu                                                   */
  int32_t dw_accumulate;    /* 1: dWg and dWu are added to what the buffers hold (micro-batches) */
  int64_t ldx, ldw, ldh;    /* pitches: X and dX; Wg, Wu, dWg and dWu; H, G, U and dH           */
  int32_t tile_config;      /* 0 = library picks; else an id from flux_ffn_tile_config_info     */
  int32_t split_k;          /* 0 = library picks; else the most parts (1..64, more than 16 count as 16) that the contraction of the
                               tiles of a partly filled last round may be cut into; 1 = no cut.  2 and more ask for tiles:
                               the kernel for few rows, which cuts nothing, is not picked then */
} flux_glu_t;

/* Bytes of workspace that `op` wants (0 for a problem that is refused).  A workspace has to go through flux_ffn_init (or be
 * filled with zeros) before its first call; a call leaves it fit for the next one, whatever its problem or op.  Calls
 * that share a workspace must not overlap in time. */
size_t flux_glu_workspace_bytes(int op, const flux_glu_t* p);

/* Makes a workspace ready for its first call: clears what has to be zero in it. */
int flux_ffn_init(void* workspace, size_t workspace_bytes, void* stream);

/* H = act(X Wg) * (X Wu).  Products accumulate in fp32; activation and product are taken in fp32, rounded once.
 *   X [M,K], Wg, Wu   bf16
 *   H [M,N]           out_dtype
 *   G, U [M,N]        bf16: X Wg and X Wu for the backward pass; both or neither (NULL)
 *   workspace         >= flux_glu_workspace_bytes(FLUX_GLU_FORWARD, p) bytes (NULL if that is 0) */
int flux_glu(const flux_glu_t* p, const void* X, const void* Wg, const void* Wu, void* H, void* G, void* U,
             void* workspace, size_t workspace_bytes, void* stream);

/* Gradients of flux_glu.  G and U are the forward call's; dH [M,N] bf16.  dG and dU are taken in fp32 and rounded to bf16
 * once, as operands of the three products, which accumulate in fp32 and are rounded once at the end (a gradient in fp32 is
 * therefore as exact as bf16 dG and dU make it).  dX, or the pair dWg and dWu, may be NULL and is then not computed;
 * Wg and Wu are read for dX alone, X for dWg and dWu alone, and may be NULL without it.
 *   workspace         >= flux_glu_workspace_bytes(FLUX_GLU_BACKWARD, p) bytes */
int flux_glu_backward(const flux_glu_t* p, const void* X, const void* Wg, const void* Wu, const void* G, const void* U,
                      const void* dH, void* dX, void* dWg, void* dWu, void* workspace, size_t workspace_bytes, void* stream);

/*
 * 4-bit microscaled matrices (OCP Microscaling Formats 1.0, "MXFP4").
 * A row of K numbers is cut into blocks of 32; the last one is filled up with zeros.  A block is 32 numbers of 4 bits (E2M1: sign,
 * 0, 0.5, 1, 1.5, 2, 3, 4 or 6) and one byte e (E8M0) that multiplies them by 2^(e - 127); e = 255 makes the whole block
 * NaN.
 *   q        row r at q + r * flux_mx4_row_bytes(K): 16 bytes per block, number 2i in the low and 2i + 1 in the
 *            high four bits of byte i.
 *   scales   row r at scales + r * flux_mx4_scale_row_bytes(K): one byte per block, then zeros up to a
 *            multiple of 16 bytes.  (The products read those zeros.)
 * Quantising: e - 127 = floor(log2(largest magnitude of the block)) - 2, no less than -127; every number is divided by
 * 2^(e - 127), rounded to the nearest of the values above (ties to the even code) and held at 6 beyond it.  A block with
 * a NaN or an infinity gets e = 255; a block of zeros e = 0.
 */
size_t flux_mx4_row_bytes(int32_t K);
size_t flux_mx4_scale_row_bytes(int32_t K);

/* src [rows,K] bf16 or fp32 with pitch `ld`, any alignment that its type has; q and scales 16-byte aligned.  K up to 2^30; src spans fewer
 * than 2^31 elements. */
int flux_mx4_quantize(int32_t rows, int32_t K, int32_t src_dtype, const void* src, int64_t ld, void* q, void* scales, void* stream);
/* dst [rows,K] bf16 or fp32 with pitch `ld`: what the blocks stand for. */
int flux_mx4_dequantize(int32_t rows, int32_t K, const void* q, const void* scales, int32_t dst_dtype, void* dst, int64_t ld, void* stream);

/* Problem of flux_mx4_gemm and flux_mx4_glu.  M >= 1; N % 8 == 0; K >= 1; q and scales 16-byte aligned; each below 2^31 bytes. */
typedef struct flux_mx4 {
  int32_t M, N, K;
  int32_t out_dtype;        /* of C and H                                                       */
  int32_t act;              /* flux_mx4_glu: flux_act_t                                         */
  int32_t reserved;         /* must be 0                                                        */
  int64_t ldc;              /* pitch of C and H: a multiple of 8, at least N; 0 = N             */
  int32_t tile_config;      /* as in flux_glu_t                                                 */
  int32_t split_k;
} flux_mx4_t;

/* As flux_glu_workspace_bytes; one workspace serves the operators of this header alike. */
size_t flux_mx4_workspace_bytes(int op, const flux_mx4_t* p);

/* C = A B^T, accumulated in fp32, rounded once. */
int flux_mx4_gemm(const flux_mx4_t* p, const void* Aq, const void* As, const void* Bq, const void* Bs, void* C,
                  void* workspace, size_t workspace_bytes, void* stream);
/* H = act(X Wg^T) * (X Wu^T). */
int flux_mx4_glu(const flux_mx4_t* p, const void* Xq, const void* Xs, const void* Wgq, const void* Wgs, const void* Wuq,
                 const void* Wus, void* H, void* workspace, size_t workspace_bytes, void* stream);

/* Tile configurations, ids 1 .. count: rows by columns of products (of a gated product half are gate's and half up's), and one,
 * 0 by 0, for products of at most 64 rows and 2^28 - 16 columns whose weights lie along the contraction (4 bits, or [N,K] in flux_glu): it
 * reads the weights once, and the library picks it there unless it expects cut tiles to be well ahead (few columns over a long
 * contraction).  FLUX_ERR_UNSUPPORTED where a problem asks for that one and is not of its kind. */
int flux_ffn_tile_config_count(void);
int flux_ffn_tile_config_info(int32_t id, int32_t* tile_m, int32_t* tile_n);

/* hipError_t of the calling thread's last FLUX_ERR_HIP from this header's calls. */
int flux_ffn_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FLUX_FFN_MI355_H_ */
