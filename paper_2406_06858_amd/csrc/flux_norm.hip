// Root-mean-square norm with the residual's addition, and its backward pass.
//
//   forward    S = X + R,  r = 1 / sqrt(mean(S^2) + eps),  Y = S r W
//   backward   with h = S r:  dR = r (dY W - h mean(dY W h)) + dS,  dW = sum over rows of dY h
//
// Sums are fp32, a lane's own first and then over lanes in a fixed order.  r is taken with the square root and the division that round
// correctly: one a row.
//
// Memory bounds both: each number is read once and each result written once.  us (TB/s): forward in bf16 8192x12288 135 (6.0), 8192x8192 91 (5.9), into 4 bits 83
// (5.3); backward with dS 8192x8192 100 (5.6, and 4 for the join of dW), 8192x12288 151 (5.3); a pass that scales 1 GiB reaches 6.25.  Up to some hundred rows it is
// the launch.
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
  float* partial;                // [groups of rows], pitch `pitch`; or null
  void* dw;                      // where one group has all rows: dW itself; or null
  int32_t dw_f32, dw_accumulate;
  long long ldx, lds, ldy, pitch;
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
template <class T, bool PAST, bool WHOLE = false>
__device__ __forceinline__ void write8(void* p, long long at, int left, const float (&x)[PER_LANE]) {
  T v[PER_LANE];
  round8(x, v);
  store8<PAST, WHOLE>(static_cast<T*>(p) + at, left, v);
}

// Sum over a row's LANES lanes, everybody's: in a wave by exchange, over waves through LDS, `turn` telling one sum's place from the next one's.
template <int LANES>
__device__ __forceinline__ float sum_of(float v, int turn = 0) {
#pragma unroll
  for (int n = 1; n < (LANES < 64 ? LANES : 64); n *= 2) v += __shfl_xor(v, n);
  if constexpr (LANES > 64) {
    __shared__ float part[2][LANES / 64];
    if (threadIdx.x % 64 == 0) part[turn][threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < LANES / 64; ++i) v += part[turn][i];
  }
  return v;
}

// Y of a lane: numbers, or its part of a block of 32; k may lie past the row's end, where blocks' padding is.
template <bool PAST, bool WHOLE>
__device__ __forceinline__ void write_y(const NormArgs& a, int row, int k, int left, const float (&y)[PER_LANE]) {
  if (a.out == FLUX_NORM_BF16) {
    write8<uint16_t, PAST, WHOLE>(a.y, row * a.ldy + k, left, y);
  } else if (a.out == FLUX_NORM_F32) {
    write8<float, false, WHOLE>(a.y, row * a.ldy + k, left, y);
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
    if (k % 32 == 0 && k / 32 < row_scales) a.scales[(long long)row * row_scales + k / 32] = (uint8_t)(k / 32 < blocks ? byte : 0u);      // (a row of NaN has padding too)
  }
}

// ---- kernels --------------------------------------------------------------------------------------------------
// The row in registers, so that memory is read once: LANES lanes a row, VECS pieces of 8 numbers a lane, 256 / LANES rows a workgroup where LANES is less.  WHOLE: K
// is a multiple of 8, a piece is in the row or is not.  All pieces of the row and of W are asked for before the first is used.  Results in bf16 go past the caches
// (8192x8192 91 us, through them 95); fp32 ones, of which a lane's two stores are half lines, do not (1496x5112 12.2, past them 14.3).
template <class TX, class TS, bool RESIDUAL, int LANES, int VECS, bool WHOLE>
__global__ void __launch_bounds__(LANES < 256 ? 256 : LANES) norm_row_kernel(const NormArgs a) {
  constexpr int ROWS = LANES < 256 ? 256 / LANES : 1;
  const int lane = threadIdx.x % LANES;
  const long long r64 = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * ROWS + threadIdx.x / LANES;
  if (r64 >= a.M) return;                        // (with more than one row a workgroup there is no barrier)
  const int row = (int)r64;
  const TX* const x = static_cast<const TX*>(a.x) + row * a.ldx;
  const TS* const r = static_cast<const TS*>(a.r) + row * a.lds;
  TS* const s = static_cast<TS*>(a.s) + row * a.lds;
  const auto left = [&](int k) { return WHOLE ? (k < a.K ? PER_LANE : 0) : a.K - k; };
  Raw8<TX> raw_x[VECS];
  Raw8<TS> raw_r[VECS];
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int k = (i * LANES + lane) * PER_LANE;
    raw_x[i].template ask<WHOLE>(x, k, a.K);
    if constexpr (RESIDUAL) raw_r[i].template ask<WHOLE>(r, k, a.K);
  }
  Raw8<float> raw_w[VECS];
  Raw8<uint16_t> raw_w16[VECS];
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int k = (i * LANES + lane) * PER_LANE;
    if (a.w_f32) raw_w[i].template ask<WHOLE>(static_cast<const float*>(a.w), k, a.K);
    else raw_w16[i].template ask<WHOLE>(static_cast<const uint16_t*>(a.w), k, a.K);
  }
  float v[VECS][PER_LANE];
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int k = (i * LANES + lane) * PER_LANE;
    raw_x[i].template settle<WHOLE>(k, a.K);
#pragma unroll
    for (int e = 0; e < PER_LANE; ++e) v[i][e] = raw_x[i].at(e);
    if constexpr (RESIDUAL) {
      raw_r[i].template settle<WHOLE>(k, a.K);
      TS t[PER_LANE];
#pragma unroll
      for (int e = 0; e < PER_LANE; ++e) v[i][e] += raw_r[i].at(e);
      round8(v[i], t);
#pragma unroll
      for (int e = 0; e < PER_LANE; ++e) {
        if constexpr (sizeof(TS) == 2) v[i][e] = from_bf16(t[e]);
      }
      store8<sizeof(TS) == 2, WHOLE>(s + k, left(k), t);
    }
  }
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < VECS; ++i)
#pragma unroll
    for (int e = 0; e < PER_LANE; ++e) sum += v[i][e] * v[i][e];
  const float rstd = 1.f / sqrtf(sum_of<LANES>(sum) / (float)a.K + a.eps);
  if (lane == 0 && a.rstd != nullptr) a.rstd[row] = rstd;
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int k = (i * LANES + lane) * PER_LANE;
    float w[PER_LANE];
    if (a.w_f32) {
      raw_w[i].template settle<WHOLE>(k, a.K);
#pragma unroll
      for (int e = 0; e < PER_LANE; ++e) w[e] = raw_w[i].at(e);
    } else {
      raw_w16[i].template settle<WHOLE>(k, a.K);
#pragma unroll
      for (int e = 0; e < PER_LANE; ++e) w[e] = raw_w16[i].at(e);
    }
#pragma unroll
    for (int e = 0; e < PER_LANE; ++e) v[i][e] = v[i][e] * rstd * w[e];
    write_y<true, WHOLE>(a, row, k, left(k), v[i]);
  }
}

// Rows too long for registers: a workgroup a row, which is read twice (the second time mostly out of the caches).
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
  const float rstd = 1.f / sqrtf(sum_of<256>(sum) / (float)a.K + a.eps);
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
    write_y<false, false>(a, row, k, a.K - k, v);
  }
}

__device__ __forceinline__ void write_dw(void* dw, int k, float v, int f32, int accumulate) {
  if (f32) {
    float* const p = static_cast<float*>(dw) + k;
    *p = accumulate ? *p + v : v;
  } else {
    __bf16* const p = static_cast<__bf16*>(dw) + k;
    *p = (__bf16)(accumulate ? (float)*p + v : v);
  }
}

// The row in registers, as norm_row_kernel has it; a workgroup takes rows from its first one on in steps of all workgroups' rows, keeps its lanes' part of dW
// beside them, and leaves it as one row of `partial`: one pass over dY, S and dS for all three results.  AHEAD: the next row's numbers are asked for ahead of this one's sum.
template <class TY, class TS, int LANES, int VECS, bool AHEAD, bool WHOLE>
__global__ void __launch_bounds__(LANES < 256 ? 256 : LANES) norm_grad_row_kernel(const NormGradArgs a) {
  constexpr int NT = LANES < 256 ? 256 : LANES, ROWS = NT / LANES;
  const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES, step = gridDim.x * ROWS;
  const auto left = [&](int k) { return WHOLE ? (k < a.K ? PER_LANE : 0) : a.K - k; };
  struct Row {
    Raw8<TY> g[VECS];
    Raw8<TS> h[VECS], d[VECS];
    float rstd = 0.f;
  };
  const auto ask = [&](Row& x, long long row) {
    if (row >= a.M) return;
    x.rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const int k = (i * LANES + lane) * PER_LANE;
      x.g[i].template ask<WHOLE>(static_cast<const TY*>(a.dy) + row * a.ldy, k, a.K);
      x.h[i].template ask<WHOLE>(static_cast<const TS*>(a.s) + row * a.lds, k, a.K);
      if (a.ds != nullptr) x.d[i].template ask<WHOLE>(static_cast<const TS*>(a.ds) + row * a.lds, k, a.K);
    }
  };
  long long row = (long long)blockIdx.x * ROWS + slot;
  Row next;
  if (AHEAD) ask(next, row);
  float w[VECS][PER_LANE], dw[VECS][PER_LANE];
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int k = (i * LANES + lane) * PER_LANE;
    if (a.w_f32) load8<WHOLE>(static_cast<const float*>(a.w) + k, left(k), w[i]);
    else load8<WHOLE>(static_cast<const uint16_t*>(a.w) + k, left(k), w[i]);
#pragma unroll
    for (int e = 0; e < PER_LANE; ++e) dw[i][e] = 0.f;
  }
  // (every slot of a workgroup takes as many turns as its first)
  for (int turn = 0; row - slot < a.M; ++turn, row += step) {
    Row x;
    if (AHEAD) {
      x = next;
      ask(next, row + step);
    } else {
      ask(x, row);
    }
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const int k = (i * LANES + lane) * PER_LANE;
      x.g[i].template settle<WHOLE>(k, a.K);
      x.h[i].template settle<WHOLE>(k, a.K);
      if (a.ds != nullptr) x.d[i].template settle<WHOLE>(k, a.K);
    }
    const float r = x.rstd;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
      for (int e = 0; e < PER_LANE; ++e) {
        const float t = x.g[i].at(e) * (x.h[i].at(e) * r);
        if (row < a.M) dw[i][e] += t;
        sum += t * w[i][e];
      }
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      x.g[i].fold();
      x.h[i].fold();
      x.d[i].fold();
    }
    const float mean = sum_of<LANES>(sum, turn & 1) / (float)a.K;
    if (row < a.M) {
#pragma unroll
      for (int i = 0; i < VECS; ++i) {
        const int k = (i * LANES + lane) * PER_LANE;
        float v[PER_LANE];
#pragma unroll
        for (int e = 0; e < PER_LANE; ++e) {
          v[e] = r * (x.g[i].at(e) * w[i][e] - x.h[i].at(e) * r * mean);
          if (a.ds != nullptr) v[e] += x.d[i].at(e);
        }
        if (a.dr != nullptr) write8<TS, sizeof(TS) == 2, WHOLE>(a.dr, row * a.lds + k, left(k), v);
        if (a.dx != nullptr) {
          if (a.x_f32) write8<float, false, WHOLE>(a.dx, row * a.ldx + k, left(k), v);
          else write8<uint16_t, true, WHOLE>(a.dx, row * a.ldx + k, left(k), v);
        }
      }
    }
  }
  if (a.partial == nullptr && a.dw == nullptr) return;
  // the slots' sums, in their order
  if constexpr (ROWS > 1) {
    __shared__ float part[ROWS][LANES * VECS * PER_LANE];
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
      for (int e = 0; e < PER_LANE; ++e) part[slot][(i * LANES + lane) * PER_LANE + e] = dw[i][e];
    __syncthreads();
    for (int k = threadIdx.x; k < a.K; k += NT) {
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < ROWS; ++j) sum += part[j][k];
      if (a.dw != nullptr) write_dw(a.dw, k, sum, a.dw_f32, a.dw_accumulate);
      else a.partial[blockIdx.x * a.pitch + k] = sum;
    }
  } else {
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const int k = (i * LANES + lane) * PER_LANE;
      if (VECS == 1 && a.dw != nullptr) {          // (with two pieces a lane there are no registers for it)
#pragma unroll
        for (int e = 0; e < PER_LANE; ++e)
          if (k + e < a.K) write_dw(a.dw, k + e, dw[i][e], a.dw_f32, a.dw_accumulate);
      } else {
        store8<false, WHOLE>(a.partial + blockIdx.x * a.pitch + k, left(k), dw[i]);
      }
    }
  }
}

// Rows too long for registers: a workgroup a row, which is read twice; dW in a launch of its own.
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
  const float mean = sum_of<256>(sum) / (float)a.K;
  for (int k = threadIdx.x * PER_LANE; k < a.K; k += 256 * PER_LANE) {
    float g[PER_LANE], h[PER_LANE], w[PER_LANE], d[PER_LANE] = {};
    load8(dy + k, a.K - k, g);
    load8(s + k, a.K - k, h);
    load8_of(a.w, a.w_f32, k, a.K - k, w);
    if (a.ds != nullptr) load8(static_cast<const TS*>(a.ds) + row * a.lds + k, a.K - k, d);
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) d[i] += rstd * (g[i] * w[i] - h[i] * rstd * mean);
    if (a.dr != nullptr) write8<TS, false>(a.dr, row * a.lds + k, a.K - k, d);
    if (a.dx != nullptr) {
      if (a.x_f32) write8<float, false>(a.dx, row * a.ldx + k, a.K - k, d);
      else write8<uint16_t, false>(a.dx, row * a.ldx + k, a.K - k, d);
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
  store8<false>(a.partial + blockIdx.y * a.pitch + k, a.K - k, sum);
}

// dW out of the groups' sums.  A workgroup has 32 columns, a line of every group's; 32 lanes a column, each a run of groups in their order, then the
// runs in theirs.
__global__ void __launch_bounds__(256) norm_dw_join_kernel(const float* partial, long long pitch, int groups, int K, void* dw, int f32, int accumulate) {
  __shared__ float part[32][33];
  const int c = threadIdx.x % 8 * 4, run = threadIdx.x / 8, each = (groups + 31) / 32, first = run * each, last = min(first + each, groups);
  const long long k0 = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 32;
  if (k0 >= K) return;                           // (the whole workgroup)
  flux::f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  const float* const from = partial + k0 + c;
#pragma unroll 8
  for (int g = first; g < last; ++g) sum += *reinterpret_cast<const flux::f32x4*>(from + g * pitch);
#pragma unroll
  for (int e = 0; e < 4; ++e) part[run][c + e] = sum[e];
  __syncthreads();
  const int k = (int)k0 + threadIdx.x;
  if (threadIdx.x >= 32 || k >= K) return;
  float v = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) v += part[i][threadIdx.x];
  write_dw(dw, k, v, f32, accumulate);
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

// (a grid is at most 2^23 workgroups wide: see flux_mx4.hip)
static dim3 grid_of(long long n) {
  const long long x = std::min(n, 1ll << 23);
  return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}

template <class TX, class TS, bool RESIDUAL, int LANES, int VECS>
static hipError_t go_row(const NormArgs& a, hipStream_t s) {
  constexpr int NT = LANES < 256 ? 256 : LANES, ROWS = NT / LANES;
  return start_with(a.K % PER_LANE == 0 ? norm_row_kernel<TX, TS, RESIDUAL, LANES, VECS, true> : norm_row_kernel<TX, TS, RESIDUAL, LANES, VECS, false>,
                    grid_of(ceil_div(a.M, ROWS)), NT, s, a);
}
// Lanes and pieces by a row's length.  A piece a lane asks for most at once with the fewest registers, as long as a workgroup's lanes are not idle: us of 8192x8192
// 1024 lanes x 1 piece / 256 x 4: 92 / 98; 1496x5112, of which 1024 x 1 leaves a third of the lanes idle, 256 x 3 / 768 x 1: 11.5 / 13.3.
template <class TX, class TS, bool RESIDUAL>
static hipError_t go(const NormArgs& a, hipStream_t s) {
  const int K = in_blocks(a.out) ? (a.K + 511) / 512 * 512 : a.K;          // (the padding of a row's scales is written too)
  if (K <= 128) return go_row<TX, TS, RESIDUAL, 16, 1>(a, s);
  if (K <= 512) return go_row<TX, TS, RESIDUAL, 64, 1>(a, s);
  if (K <= 1024) return go_row<TX, TS, RESIDUAL, 64, 2>(a, s);
  if (K <= 2048) return go_row<TX, TS, RESIDUAL, 256, 1>(a, s);
  if (K <= 4096) return go_row<TX, TS, RESIDUAL, 512, 1>(a, s);
  if (K <= 6144) return go_row<TX, TS, RESIDUAL, 256, 3>(a, s);
  if (K <= 8192) return go_row<TX, TS, RESIDUAL, 1024, 1>(a, s);
  if (K <= 12288) return go_row<TX, TS, RESIDUAL, 768, 2>(a, s);
  if (K <= 16384) return go_row<TX, TS, RESIDUAL, 1024, 2>(a, s);
  // (registers: a row in 32 bits whose end needs putting in place has no room for four pieces)
  constexpr bool WIDE = RESIDUAL && sizeof(TX) + sizeof(TS) == 8;
  if constexpr (WIDE) {
    if (K <= 32768 && a.K % PER_LANE == 0) return start_with(norm_row_kernel<TX, TS, RESIDUAL, 1024, 4, true>, dim3(a.M), 1024, s, a);
  } else {
    if (K <= 32768) return go_row<TX, TS, RESIDUAL, 1024, 4>(a, s);
  }
  return start(norm_kernel<TX, TS, RESIDUAL>, dim3(a.M), s, a);
}
static hipError_t launch_norm(const flux_norm_t* p, const NormArgs& a, bool residual, hipStream_t s) {
  const bool xf = p->x_dtype == FLUX_F32, sf = p->s_dtype == FLUX_F32;
  if (!residual) return xf ? go<float, float, false>(a, s) : go<uint16_t, uint16_t, false>(a, s);
  if (xf) return sf ? go<float, float, true>(a, s) : go<float, uint16_t, true>(a, s);
  return sf ? go<uint16_t, float, true>(a, s) : go<uint16_t, uint16_t, true>(a, s);
}

// How the backward pass runs: lanes and pieces of norm_grad_row_kernel (0: rows too long for it), and groups of rows whose part of dW is summed by itself. One
// workgroup a unit where it has 768 lanes or more, two or three of the smaller: us of 8192x8192 with 256 / 512 groups 99.8 / 101.8, of 1024x8192 17.3 / 21.5, whose
// parts of dW are the more to join the more groups there are.
struct GradPlan { int lanes, vecs, groups; };
static GradPlan grad_plan(const flux_norm_t* p) {
  static constexpr GradPlan plans[] = {{16, 1, 512}, {64, 1, 512}, {64, 2, 512}, {256, 1, 768}, {512, 1, 512}, {768, 1, 256}, {1024, 1, 256}, {768, 2, 256}, {1024, 2, 256}};
  for (GradPlan g : plans)
    if (p->K <= g.lanes * g.vecs * PER_LANE && (g.lanes * g.vecs <= 1536 || p->K % PER_LANE == 0)) {
      const int slots = std::max(1, 256 / g.lanes);
      // (up to four turns of one workgroup are over before a second launch would be: us of 1x8192 4.9 and not 8.5)
      g.groups = p->M <= 4 * slots && (g.vecs == 1 || g.lanes == 64) ? 1 : std::min(g.groups, ceil_div(p->M, slots));
      return g;
    }
  return GradPlan{0, 0, std::min(p->M, 64)};
}
static long long partial_pitch(const flux_norm_t* p) { return (p->K + 31ll) / 32 * 32; }

template <class TY, class TS>
static hipError_t go_grad(const GradPlan& g, const NormGradArgs& a, hipStream_t s) {
#define GO(LANES, VECS, AHEAD, AHEAD_ODD) \
  if (g.lanes == LANES && g.vecs == VECS) \
    return start_with(a.K % PER_LANE == 0 ? norm_grad_row_kernel<TY, TS, LANES, VECS, AHEAD, true> : norm_grad_row_kernel<TY, TS, LANES, VECS, AHEAD_ODD, false>, \
                      dim3(g.groups), LANES < 256 ? 256 : LANES, s, a)
  GO(16, 1, true, true);
  GO(64, 1, true, true);
  GO(64, 2, true, true);
  GO(256, 1, true, true);
  GO(512, 1, true, true);
  GO(768, 1, true, true);
  GO(1024, 1, true, true);
  GO(768, 2, sizeof(TS) == 2, sizeof(TS) == 2 && sizeof(TY) == 2);          // (beside a stream in 32 bits there are no registers for the next row; with a row's odd end beside dY in 32 bits neither)
  if (g.lanes == 1024 && g.vecs == 2) return start_with(norm_grad_row_kernel<TY, TS, 1024, 2, false, true>, dim3(g.groups), 1024, s, a);
#undef GO
  if (a.partial != nullptr) {
    // (ahead of dR, which may take dS's place)
    const hipError_t e = start(norm_dw_kernel<TY, TS>, dim3(ceil_div(a.K, 256 * PER_LANE), g.groups), s, a, ceil_div(a.M, g.groups));
    if (e != hipSuccess) return e;
  }
  return a.dr != nullptr || a.dx != nullptr ? start(norm_grad_kernel<TY, TS>, dim3(a.M), s, a) : hipSuccess;
}

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
  FFN_HIP(launch_norm(p, a, R != nullptr, static_cast<hipStream_t>(stream)));
  return FLUX_OK;
}

size_t flux_norm_workspace_bytes(const flux_norm_t* p) {
  if (validate(p) != FLUX_OK || in_blocks(p->out)) return 0;
  return WS_HEADER + 4ull * grad_plan(p).groups * partial_pitch(p);
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
  const GradPlan g = grad_plan(p);
  const bool direct = g.groups == 1 && (g.vecs == 1 || g.lanes == 64);
  a.dw = direct ? dW : nullptr;
  a.dw_f32 = p->dw_dtype == FLUX_F32;
  a.dw_accumulate = p->dw_accumulate;
  a.partial = dW != nullptr && !direct ? reinterpret_cast<float*>(static_cast<char*>(workspace) + WS_HEADER) : nullptr;
  a.pitch = partial_pitch(p);
  a.ldx = pitch(p->ldx, p->K);
  a.lds = pitch(p->lds, p->K);
  a.ldy = pitch(p->ldy, p->K);
  a.M = p->M;
  a.K = p->K;
  a.w_f32 = p->w_dtype == FLUX_F32;
  a.x_f32 = p->x_dtype == FLUX_F32;
  if (dR == nullptr && dX == nullptr && dW == nullptr) return FLUX_OK;
  const bool yf = p->out == FLUX_NORM_F32, sf = p->s_dtype == FLUX_F32;
  FFN_HIP(yf ? (sf ? go_grad<float, float>(g, a, s) : go_grad<float, uint16_t>(g, a, s)) : (sf ? go_grad<uint16_t, float>(g, a, s) : go_grad<uint16_t, uint16_t>(g, a, s)));
  if (a.partial != nullptr)
    FFN_HIP(start(norm_dw_join_kernel, grid_of(ceil_div(p->K, 32)), s, (const float*)a.partial, a.pitch, g.groups, (int)p->K, dW, (int)(p->dw_dtype == FLUX_F32), (int)p->dw_accumulate));
  return FLUX_OK;
}

}  // extern "C"
