// What becomes of a tile of logits Z = X W^T, which nobody keeps (gfx950): out of the accumulators of the tile kernel's main loop either
//
//   statistics   of every row and each wave's run of columns the largest logit m and the sum of exp(Z - m), and the target's logit; or
//   dZ           dloss (exp(Z - lse) - [v = target]) in bf16, operand of the two products of the backward pass.
#pragma once
#include "flux_ffn_tile.h"

namespace flux_ffn {

struct LossArgs {
  const void* target;            // [rows], 32 or 64 bits
  int32_t target_i64, dloss_one;
  long long v0, vocab;           // number of the product's first column; columns of the whole vocabulary
  // statistics
  float2* stats;                 // [runs of columns][rows]: m, sum
  float* logit;                  // written where the target is a column here
  // dZ
  const float *lse, *dloss;
  __bf16* dz;                    // pitch TileArgs::ld
};


// exp(x), within |x| 2^-24 of itself: what that is off by matters for logits that count for nothing.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(LOG2E * x); }

// The row's target as a column of this product, -1 where it is none; counts: whether the row counts at all.
__device__ __forceinline__ int target_column(const LossArgs& l, int row, int cols, bool& counts) {
  const long long t = l.target_i64 ? static_cast<const long long*>(l.target)[row] : static_cast<const int32_t*>(l.target)[row];
  counts = t >= 0 && t < l.vocab;
  const long long c = t - l.v0;
  return counts && c >= 0 && c < cols ? (int)c : -1;
}

// (m, s) and (m2, s2) of two sets of logits as of one.  An infinite m leaves exp its argument as it is: no infinity is taken from another.
__device__ __forceinline__ void join_stats(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2), at = __builtin_fabsf(top) == __builtin_inff() ? 0.f : top;
  s = s * exp_of(m - at) + s2 * exp_of(m2 - at);
  m = top;
}

// 16 rows of a wave's part of the tile: a lane holds columns 16 n + 4 (lane / 16) .. + 3 of row lane % 16.
template <class C>
__device__ __forceinline__ void finish_stats16(const TileArgs& t, const LossArgs& l, const f32x4 (&acc)[C::NI], int row0, int col0, int lane) {
  const int g = lane >> 4, row = row0 + (lane & 15);
  const bool in_row = !C::EDGE || row < t.rows;
  bool counts;
  const int target = in_row ? target_column(l, row, t.cols, counts) : -1;
  float m = -__builtin_inff();
#pragma unroll
  for (int n = 0; n < C::NI; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (!C::EDGE || col0 + n * 16 + 4 * g + e < t.cols) m = fmaxf(m, acc[n][e]);
  m = fmaxf(m, __shfl_xor(m, 16));
  m = fmaxf(m, __shfl_xor(m, 32));
  const float at = __builtin_fabsf(m) == __builtin_inff() ? 0.f : m;
  float s = 0.f, z = 0.f;
#pragma unroll
  for (int n = 0; n < C::NI; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int col = col0 + n * 16 + 4 * g + e;
      if (!C::EDGE || col < t.cols) s += exp_of(acc[n][e] - at);
      if (col == target) z = acc[n][e];
    }
  s += __shfl_xor(s, 16);
  s += __shfl_xor(s, 32);
  if (!in_row) return;
  if (g == 0) l.stats[(long long)(col0 / C::WTN) * t.rows + row] = make_float2(m, s);
  const int off = target - col0;
  if (target >= 0 && off >= 0 && off < C::WTN && (off >> 2 & 3) == g) l.logit[row] = z;
}

// Columns past the last one are zeros as far as the 16 bytes that hold it reach: the products read them.
template <class C>
__device__ __forceinline__ void finish_dz16(const TileArgs& t, const LossArgs& l, const f32x4 (&acc)[C::NI], int row0, int col0, int lane) {
  const int g = lane >> 4, row = row0 + (lane & 15), in_bf16 = (g & 1) * 32 + (g >> 1) * 16;
  int target = -1;
  float lse = 0.f, d = 0.f;
  if (!C::EDGE || row < t.rows) {
    bool counts;
    target = target_column(l, row, t.cols, counts);
    lse = l.lse[row];
    d = counts ? l.dloss[l.dloss_one ? 0 : row] : 0.f;
  }
  u32x4 p[C::NI / 2];
#pragma unroll
  for (int n = 0; n < C::NI; n += 2) {
    float v[8];
    eight_columns(acc[n], acc[n + 1], v);
    const int col = col0 + n * 16 + 16 * (g & 1) + 8 * (g >> 1);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float dz = d * (exp_of(v[e] - lse) - (col + e == target ? 1.f : 0.f));
      v[e] = d == 0.f || (C::EDGE && col + e >= t.cols) ? 0.f : dz;      // (a row that does not count, whatever its logits are)
    }
    p[n / 2] = pack8(v);
  }
  if constexpr (C::NI == 2) {
    store_piece<C::EDGE>(t, l.dz, 2, p[0], row0, col0, lane, in_bf16);
  } else {
#pragma unroll
    for (int n = 0; n < C::NI / 2; n += 2) store_pair<C::EDGE>(t, l.dz, 2, p[n], p[n + 1], row0, col0 + n * 32, lane, in_bf16);
  }
}

template <class C, bool GRADIENT>
__global__ void __launch_bounds__(C::NT, C::OCC) logits_kernel(const TileArgs t, const LossArgs l) {
  __shared__ __attribute__((aligned(1024))) unsigned char pool[C::POOL_BYTES];
  tile_body<C>(t, pool, [&](int, const f32x4 (&x)[C::NI], int row0, int col0, int lane) {
    if constexpr (GRADIENT) finish_dz16<C>(t, l, x, row0, col0, lane);
    else finish_stats16<C>(t, l, x, row0, col0, lane);
  });
}

}  // namespace flux_ffn
