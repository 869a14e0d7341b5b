// Root-mean-square norm with the residual's addition, and its backward pass.
//
//   forward    S = X + R,  r = 1 / sqrt(mean(S^2) + eps),  Y = S r W
//   backward   with h = S r:  dR = r (dY W - h mean(dY W h)) + dS,  dW = sum over rows of dY h
//
// Sums are fp32, a lane's own first and then over lanes in a fixed order.  r is taken with the square root and the division that round
// correctly: one a row.
#include <algorithm>
#include "flux_ffn_internal.h"
#include "flux_mx_blocks.h"
#include "flux_norm.h"

namespace flux_ffn {

struct NormArgs {
  const void *x, *r, *w;
  void *s, *y;
  uint8_t* scales;
  float* rstd;
  long long ldx, lds, ldy;
  int32_t M, K;
  float eps;
  int32_t out, w_f32;
};

struct NormGradArgs {
  const void *dy, *s, *w, *ds;
  const float* rstd;
  void *dr, *dx;
  float* partial;                // [row groups][K]
  long long ldx, lds, ldy;
  int32_t M, K;
  int32_t w_f32, x_f32;
};

// ---- numbers of a lane ----------------------------------------------------------------------------------------
__device__ __forceinline__ void load8_of(const void* p, int f32, long long at, int left, float (&x)[PER_LANE]) {
  if (f32) load8(static_cast<const float*>(p) + at, left, x);
  else load8(static_cast<const uint16_t*>(p) + at, left, x);
}
template <class T>
__device__ __forceinline__ void round8(const float (&x)[PER_LANE], T (&v)[PER_LANE]) {
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = x[i];
    else v[i] = __builtin_bit_cast(uint16_t, (__bf16)x[i]);
  }
}
template <class T>
__device__ __forceinline__ void write8(void* p, long long at, int left, const float (&x)[PER_LANE]) {
  T v[PER_LANE];
  round8(x, v);
  store8<false>(static_cast<T*>(p) + at, left, v);
}

// Sum over the workgroup's 256 lanes, everybody's.
__device__ __forceinline__ float sum_of_256(float v) {
  __shared__ float part[4];
#pragma unroll
  for (int n = 1; n < 64; n *= 2) v += __shfl_xor(v, n);
  __syncthreads();               // (of the sum before)
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
  __syncthreads();
  return part[0] + part[1] + part[2] + part[3];
}

// Y of a lane: numbers, or its part of a block of 32; k may lie past the row's end, where blocks' padding is.
__device__ __forceinline__ void write_y(const NormArgs& a, int row, int k, const float (&y)[PER_LANE]) {
  if (a.out == FLUX_NORM_BF16) {
    if (k < a.K) write8<uint16_t>(a.y, row * a.ldy + k, a.K - k, y);
  } else if (a.out == FLUX_NORM_F32) {
    if (k < a.K) write8<float>(a.y, row * a.ldy + k, a.K - k, y);
  } else {
    const int blocks = (a.K + 31) / 32, row_scales = (blocks + 15) / 16 * 16;
    uint32_t byte;
    if (a.out == FLUX_NORM_MX4) {
      const uint32_t codes = encode4(y, byte);
      if (k < blocks * 32) *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.y) + (long long)row * (blocks * 16ll) + k / 2) = codes;
    } else {
      const uint2 codes = encode8(y, byte);
      if (k < blocks * 32) *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.y) + (long long)row * (blocks * 32ll) + k) = codes;
    }
    if (k % 32 == 0 && k / 32 < row_scales) a.scales[(long long)row * row_scales + k / 32] = (uint8_t)byte;
  }
}

// ---- kernels --------------------------------------------------------------------------------------------------
// A workgroup a row; the row is read twice.
template <class TX, class TS, bool RESIDUAL>
__global__ void __launch_bounds__(256) norm_kernel(const NormArgs a) {
  const int row = blockIdx.x;
  const TX* const x = static_cast<const TX*>(a.x) + row * a.ldx;
  const TS* const r = static_cast<const TS*>(a.r) + row * a.lds;
  TS* const s = static_cast<TS*>(a.s) + row * a.lds;
  float sum = 0.f;
  for (int k = threadIdx.x * PER_LANE; k < a.K; k += 256 * PER_LANE) {
    float v[PER_LANE];
    load8(x + k, a.K - k, v);
    if (RESIDUAL) {
      float u[PER_LANE];
      load8(r + k, a.K - k, u);
      TS w[PER_LANE];
#pragma unroll
      for (int i = 0; i < PER_LANE; ++i) v[i] += u[i];
      round8(v, w);
#pragma unroll
      for (int i = 0; i < PER_LANE; ++i) {
        if constexpr (sizeof(TS) == 2) v[i] = from_bf16(w[i]);
      }
      store8<false>(s + k, a.K - k, w);
    }
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) sum += v[i] * v[i];
  }
  const float rstd = 1.f / sqrtf(sum_of_256(sum) / (float)a.K + a.eps);
  if (threadIdx.x == 0 && a.rstd != nullptr) a.rstd[row] = rstd;
  const int end = a.out >= FLUX_NORM_MX4 ? (a.K + 511) / 512 * 512 : a.K;
  for (int k0 = 0; k0 < end; k0 += 256 * PER_LANE) {
    const int k = k0 + threadIdx.x * PER_LANE;
    float v[PER_LANE] = {}, w[PER_LANE] = {};
    if (k < a.K) {
      if constexpr (RESIDUAL) load8(s + k, a.K - k, v);
      else load8(x + k, a.K - k, v);
      load8_of(a.w, a.w_f32, k, a.K - k, w);
    }
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) v[i] = v[i] * rstd * w[i];
    write_y(a, row, k, v);
  }
}

// A workgroup a row; the row is read twice.
template <class TY, class TS>
__global__ void __launch_bounds__(256) norm_grad_kernel(const NormGradArgs a) {
  const int row = blockIdx.x;
  const TY* const dy = static_cast<const TY*>(a.dy) + row * a.ldy;
  const TS* const s = static_cast<const TS*>(a.s) + row * a.lds;
  const float rstd = a.rstd[row];
  float sum = 0.f;
  for (int k = threadIdx.x * PER_LANE; k < a.K; k += 256 * PER_LANE) {
    float g[PER_LANE], h[PER_LANE], w[PER_LANE];
    load8(dy + k, a.K - k, g);
    load8(s + k, a.K - k, h);
    load8_of(a.w, a.w_f32, k, a.K - k, w);
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) sum += g[i] * w[i] * (h[i] * rstd);
  }
  const float mean = sum_of_256(sum) / (float)a.K;
  for (int k = threadIdx.x * PER_LANE; k < a.K; k += 256 * PER_LANE) {
    float g[PER_LANE], h[PER_LANE], w[PER_LANE], d[PER_LANE] = {};
    load8(dy + k, a.K - k, g);
    load8(s + k, a.K - k, h);
    load8_of(a.w, a.w_f32, k, a.K - k, w);
    if (a.ds != nullptr) load8(static_cast<const TS*>(a.ds) + row * a.lds + k, a.K - k, d);
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) d[i] += rstd * (g[i] * w[i] - h[i] * rstd * mean);
    if (a.dr != nullptr) write8<TS>(a.dr, row * a.lds + k, a.K - k, d);
    if (a.dx != nullptr) {
      if (a.x_f32) write8<float>(a.dx, row * a.ldx + k, a.K - k, d);
      else write8<uint16_t>(a.dx, row * a.ldx + k, a.K - k, d);
    }
  }
}

// dW of a group of rows: a lane has eight columns.
template <class TY, class TS>
__global__ void __launch_bounds__(256) norm_dw_kernel(const NormGradArgs a, int rows_each) {
  const int k = (blockIdx.x * 256 + threadIdx.x) * PER_LANE;
  if (k >= a.K) return;
  const int first = blockIdx.y * rows_each, last = min(first + rows_each, a.M);
  float sum[PER_LANE] = {};
  for (int row = first; row < last; ++row) {
    float g[PER_LANE], h[PER_LANE];
    load8(static_cast<const TY*>(a.dy) + row * a.ldy + k, a.K - k, g);
    load8(static_cast<const TS*>(a.s) + row * a.lds + k, a.K - k, h);
    const float rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) sum[i] += g[i] * (h[i] * rstd);
  }
  store8<false>(a.partial + (long long)blockIdx.y * a.K + k, a.K - k, sum);
}

// dW out of the groups' sums, in their order.
__global__ void __launch_bounds__(256) norm_dw_join_kernel(const float* partial, int groups, int K, void* dw, int f32, int accumulate) {
  const int k = blockIdx.x * 256 + threadIdx.x;
  if (k >= K) return;
  float sum = 0.f;
  for (int g = 0; g < groups; ++g) sum += partial[(long long)g * K + k];
  if (f32) {
    float* const p = static_cast<float*>(dw) + k;
    *p = accumulate ? *p + sum : sum;
  } else {
    __bf16* const p = static_cast<__bf16*>(dw) + k;
    *p = (__bf16)(accumulate ? (float)*p + sum : sum);
  }
}

// ---- checks ---------------------------------------------------------------------------------------------------
static long long pitch(long long ld, int K) { return ld ? ld : K; }
static bool in_blocks(int out) { return out == FLUX_NORM_MX4 || out == FLUX_NORM_MX8; }
static int size_of(int dtype) { return dtype == FLUX_F32 ? 4 : 2; }

static int validate(const flux_norm_t* p) {
  if (p == nullptr || !dtype_ok(p->x_dtype) || !dtype_ok(p->s_dtype) || !dtype_ok(p->w_dtype) || !dtype_ok(p->dw_dtype)) return FLUX_ERR_INVALID_ARG;
  if (p->out < FLUX_NORM_BF16 || p->out > FLUX_NORM_MX8 || (p->dw_accumulate | 1) != 1 || p->reserved != 0) return FLUX_ERR_INVALID_ARG;
  if (!(p->eps >= 0.f) || __builtin_isinf(p->eps) || p->ldx < 0 || p->lds < 0 || p->ldy < 0) return FLUX_ERR_INVALID_ARG;
  if (p->M < 1 || p->K < 1 || p->K > (1 << 30)) return FLUX_ERR_SHAPE;
  for (long long ld : {pitch(p->ldx, p->K), pitch(p->lds, p->K), pitch(p->ldy, p->K)})
    if (ld < p->K || !below_limit(p->M, ld, p->K)) return FLUX_ERR_SHAPE;
  return FLUX_OK;
}

// Groups of rows whose part of dW is summed by itself.
static int row_groups(const flux_norm_t* p) { return std::min(p->M, 64); }

}  // namespace flux_ffn

using namespace flux_ffn;

extern "C" {

int flux_norm(const flux_norm_t* p, const void* X, const void* R, const void* W, void* S, void* Y, void* scales, float* rstd, void* stream) {
  const int st = validate(p);
  if (st != FLUX_OK) return st;
  if (X == nullptr || W == nullptr || Y == nullptr || (R == nullptr) != (S == nullptr)) return FLUX_ERR_INVALID_ARG;
  if (!aligned(X, size_of(p->x_dtype)) || !aligned(R, size_of(p->s_dtype)) || !aligned(S, size_of(p->s_dtype)) || !aligned(W, size_of(p->w_dtype))) return FLUX_ERR_INVALID_ARG;
  if (in_blocks(p->out) ? scales == nullptr || !aligned(scales, 16) || !aligned(Y, 16) : scales != nullptr || !aligned(Y, size_of(p->out))) return FLUX_ERR_INVALID_ARG;
  if (!aligned(rstd, 4)) return FLUX_ERR_INVALID_ARG;
  NormArgs a = {};
  a.x = X;
  a.r = R;
  a.w = W;
  a.s = S;
  a.y = Y;
  a.scales = static_cast<uint8_t*>(scales);
  a.rstd = rstd;
  a.ldx = pitch(p->ldx, p->K);
  a.lds = pitch(p->lds, p->K);
  a.ldy = pitch(p->ldy, p->K);
  a.M = p->M;
  a.K = p->K;
  a.eps = p->eps;
  a.out = p->out;
  a.w_f32 = p->w_dtype == FLUX_F32;
  const bool xf = p->x_dtype == FLUX_F32, sf = p->s_dtype == FLUX_F32;
  void (*const kernel)(NormArgs) =
      R == nullptr ? (xf ? norm_kernel<float, float, false> : norm_kernel<uint16_t, uint16_t, false>)
      : xf ? (sf ? norm_kernel<float, float, true> : norm_kernel<float, uint16_t, true>)
           : (sf ? norm_kernel<uint16_t, float, true> : norm_kernel<uint16_t, uint16_t, true>);
  FFN_HIP(start(kernel, dim3(p->M), static_cast<hipStream_t>(stream), a));
  return FLUX_OK;
}

size_t flux_norm_workspace_bytes(const flux_norm_t* p) {
  if (validate(p) != FLUX_OK || in_blocks(p->out)) return 0;
  return WS_HEADER + 4ull * row_groups(p) * p->K;
}

int flux_norm_backward(const flux_norm_t* p, const void* dY, const void* S, const void* W, const float* rstd, const void* dS, void* dR, void* dX,
                       void* dW, void* workspace, size_t workspace_bytes, void* stream) {
  int st = validate(p);
  if (st != FLUX_OK) return st;
  if (in_blocks(p->out)) return FLUX_ERR_UNSUPPORTED;
  if (dY == nullptr || S == nullptr || W == nullptr || rstd == nullptr) return FLUX_ERR_INVALID_ARG;
  if (!aligned(dY, size_of(p->out)) || !aligned(S, size_of(p->s_dtype)) || !aligned(W, size_of(p->w_dtype)) || !aligned(rstd, 4)) return FLUX_ERR_INVALID_ARG;
  if (!aligned(dS, size_of(p->s_dtype)) || !aligned(dR, size_of(p->s_dtype)) || !aligned(dX, size_of(p->x_dtype)) || !aligned(dW, size_of(p->dw_dtype))) return FLUX_ERR_INVALID_ARG;
  if (dW != nullptr && (st = workspace_ok(flux_norm_workspace_bytes(p), workspace, workspace_bytes)) != FLUX_OK) return st;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  NormGradArgs a = {};
  a.dy = dY;
  a.s = S;
  a.w = W;
  a.ds = dS;
  a.rstd = rstd;
  a.dr = dR;
  a.dx = dX;
  a.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + WS_HEADER);
  a.ldx = pitch(p->ldx, p->K);
  a.lds = pitch(p->lds, p->K);
  a.ldy = pitch(p->ldy, p->K);
  a.M = p->M;
  a.K = p->K;
  a.w_f32 = p->w_dtype == FLUX_F32;
  a.x_f32 = p->x_dtype == FLUX_F32;
  const bool yf = p->out == FLUX_NORM_F32, sf = p->s_dtype == FLUX_F32;
  if (dW != nullptr) {
    // (ahead of dR, which may take dS's place, but not S's)
    const int groups = row_groups(p), each = ceil_div(p->M, groups);
    const dim3 grid(ceil_div(p->K, 256 * PER_LANE), groups);
    void (*const kernel)(NormGradArgs, int) = yf ? (sf ? norm_dw_kernel<float, float> : norm_dw_kernel<float, uint16_t>) : (sf ? norm_dw_kernel<uint16_t, float> : norm_dw_kernel<uint16_t, uint16_t>);
    FFN_HIP(start(kernel, grid, s, a, each));
    FFN_HIP(start(norm_dw_join_kernel, dim3(ceil_div(p->K, 256)), s, (const float*)a.partial, groups, (int)p->K, dW, (int)(p->dw_dtype == FLUX_F32), (int)p->dw_accumulate));
  }
  if (dR != nullptr || dX != nullptr) {
    void (*const kernel)(NormGradArgs) = yf ? (sf ? norm_grad_kernel<float, float> : norm_grad_kernel<float, uint16_t>) : (sf ? norm_grad_kernel<uint16_t, float> : norm_grad_kernel<uint16_t, uint16_t>);
    FFN_HIP(start(kernel, dim3(p->M), s, a));
  }
  return FLUX_OK;
}

}  // extern "C"
