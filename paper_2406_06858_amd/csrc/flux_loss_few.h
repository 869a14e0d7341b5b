// Logits of few rows: the statistics of a workgroup's columns, or dZ (see flux_loss_tile.h), out of the kernel that reads the weights once.
#pragma once
#include "flux_ffn_few.h"
#include "flux_loss_tile.h"

namespace flux_ffn {

template <class C, bool GRADIENT>
__global__ void __launch_bounds__(C::NT) few_logits_kernel(const FewArgs t, const LossArgs l) {
  __shared__ __attribute__((aligned(1024))) unsigned char pool[C::POOL_BYTES];
  const int run = by_die((int)blockIdx.x, (int)gridDim.x), n0 = run * C::COLS;
  const float* const red = few_body<C>(t, pool, n0);
  float most = 1.f;
  if (GRADIENT && !l.dloss_one) {
    // (a lane a row)
    const int row = threadIdx.x & 63;
    float d = 0.f;
    if (row < t.rows) {
      bool counts;
      (void)target_column(l, row, t.cols, counts);
      d = row_dloss(l, row, counts);
    }
    most = sane_most(wave_max(__builtin_fabsf(d)));
    if (blockIdx.x == 0 && threadIdx.x == 0) *l.most = most;
  }
  // COLS neighbouring lanes a row
  for (int e = threadIdx.x; e < C::MB * 16 * C::COLS; e += C::NT) {
    const int c = e % C::COLS, row = e / C::COLS, col = n0 + c;
    if (row >= t.rows) continue;
    const float z = few_sum<C>(red, row, c);
    bool counts;
    const int target = target_column(l, row, t.cols, counts);
    if constexpr (GRADIENT) {
      const float d = row_factor(l, row_dloss(l, row, counts), most);
      const float dz = d * (exp_of(z - l.lse[row]) - (col == target ? 1.f : 0.f));
      if (col < (t.cols + 7) / 8 * 8) l.dz[row * t.ld + col] = (__bf16)(d == 0.f || col >= t.cols ? 0.f : dz);
    } else {
      float m = col < t.cols ? z : -__builtin_inff();
#pragma unroll
      for (int n = 1; n < C::COLS; n *= 2) m = fmaxf(m, __shfl_xor(m, n));
      const float at = __builtin_fabsf(m) == __builtin_inff() ? 0.f : m;
      float s = col < t.cols ? exp_of(z - at) : 0.f;
#pragma unroll
      for (int n = 1; n < C::COLS; n *= 2) s += __shfl_xor(s, n);
      if (c == 0) l.stats[(long long)run * t.rows + row] = make_float2(m, s);
      if (col == target) l.logit[row] = z;
    }
  }
}

}  // namespace flux_ffn
