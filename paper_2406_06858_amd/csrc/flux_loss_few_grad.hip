// Gradients of the loss for few rows, where the weights are everything: dX reads them once, dW writes their gradient once.
#include <algorithm>
#include "flux_ffn_internal.h"
#include "flux_loss_tile.h"

namespace flux_ffn {

// ---- dX -------------------------------------------------------------------------------------------------------
// The tile kernel with the weights past the caches.
template <class C>
__global__ void __launch_bounds__(C::NT, C::OCC) streamed_kernel(const TileArgs t) {
  __shared__ __attribute__((aligned(1024))) unsigned char pool[C::POOL_BYTES];
  Results<C, true> results{t};
  tile_body<C>(t, pool, results);
}

hipError_t launch_dx_few(int shape, const TileArgs& a, int grid, hipStream_t s) {
  if (shape == 2) return start(streamed_kernel<Cfg<DX_KN, 128, 128, 2, 2, 2, true, true>>, dim3(grid), s, a);
  if (shape == 3) return start(streamed_kernel<Cfg<DX_KN, 128, 128, 4, 4, 1, true, true>>, dim3(grid), s, a);
  if (shape == 4) return start(streamed_kernel<Cfg<DX_KN, 64, 128, 3, 3, 2, true, true>>, dim3(grid), s, a);
  return start(streamed_kernel<Cfg<DX_KN, 64, 128, 6, 6, 1, true, true>>, dim3(grid), s, a);
}

// ---- dW -------------------------------------------------------------------------------------------------------
// dW = dZ^T X is an outer product of few terms: nothing but its stores counts.  A workgroup keeps its 256 columns of X in registers, 64 a wave, as
// the matrix units want them (a lane has 8 rows' numbers of one column, so X is transposed first: a line a column), and goes through rows of dW,
// 16 at a time: dZ transposed, a line a row as well.
struct OuterArgs {
  TileArgs t;                    // rows, cols, ld, out[0], out_f32, accumulate, stream
  const __bf16* zt;              // [rows][32 KS]
  const __bf16* xt;              // [cols][32 KS]
  int32_t rows_each;             // of a workgroup, a multiple of 16
};
template <int KS>
__global__ void __launch_bounds__(256) outer_kernel(const OuterArgs o) {
  typedef Cfg<DW, 128, 128, 2, 2, 2, true> C;         // (its four column blocks of a wave, and nothing else of it)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int col0 = blockIdx.x * 256 + wave * 64, first = blockIdx.y * o.rows_each, last = min(first + o.rows_each, o.t.rows);
  if (col0 >= o.t.cols) return;
  bf16x8 x[KS][4], z[2][KS];
#pragma unroll
  for (int k = 0; k < KS; ++k)
#pragma unroll
    for (int n = 0; n < 4; ++n) x[k][n] = *reinterpret_cast<const bf16x8*>(o.xt + min(col0 + n * 16 + i, o.t.cols - 1) * (32ll * KS) + k * 32 + g * 8);
  const auto ask = [&](bf16x8 (&to)[KS], int row) {
#pragma unroll
    for (int k = 0; k < KS; ++k) to[k] = *reinterpret_cast<const bf16x8*>(o.zt + min(row + i, o.t.rows - 1) * (32ll * KS) + k * 32 + g * 8);
  };
  const auto rows16 = [&](const bf16x8 (&a)[KS], int row) {
    f32x4 acc[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[k][n], a[k], acc[n], 0, 0, 0);
    }
    finish_rows16<C, true>(o.t, 0, acc, row, col0, lane);
  };
  ask(z[0], first);
  for (int row = first; row < last; row += 32) {
    ask(z[1], row + 16);
    rows16(z[0], row);
    ask(z[0], row + 32);
    if (row + 16 < last) rows16(z[1], row + 16);
  }
}

// [rows of `from`][cols] to [cols][held], zeros in the place of rows that are not there.  A lane takes eight rows' numbers of one column.
struct TransposeArgs {
  const __bf16* from[2];
  __bf16* to[2];
  long long pitch[2];
  int32_t rows, held, cols[2], groups;         // groups: workgroups of the first matrix
};
__global__ void __launch_bounds__(256) transpose_kernel(const TransposeArgs a) {
  const int which = (int)blockIdx.x >= a.groups ? 1 : 0, col = ((int)blockIdx.x - which * a.groups) * 256 + threadIdx.x, r = blockIdx.y * 8;
  if (col >= a.cols[which]) return;
  const __bf16* const from = a.from[which] + col;
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = r + e < a.rows ? from[(r + e) * a.pitch[which]] : (__bf16)0.f;
  *reinterpret_cast<bf16x8*>(a.to[which] + col * (long long)a.held + r) = v;
}

int outer_terms(int M) { return M <= 32 ? 32 : M <= 64 ? 64 : 128; }

hipError_t launch_dw_few(const TileArgs& t, const void* dz, long long ldz, const void* X, long long ldx, void* scratch, int M, hipStream_t s) {
  OuterArgs o = {};
  o.t = t;
  __bf16* const zt = static_cast<__bf16*>(scratch);
  o.zt = zt;
  const int held = outer_terms(M);
  o.xt = zt + t.rows * (long long)held;
  TransposeArgs a = {{static_cast<const __bf16*>(dz), static_cast<const __bf16*>(X)}, {zt, zt + t.rows * (long long)held}, {ldz, ldx}, M, held, {t.rows, t.cols}, ceil_div(t.rows, 256)};
  const hipError_t e = start(transpose_kernel, dim3(a.groups + ceil_div(t.cols, 256), held / 8), s, a);
  if (e != hipSuccess) return e;
  const int strips = ceil_div(t.cols, 256), groups = std::max(1, std::min(ceil_div(t.rows, 16), (held == 128 ? 768 : 1024) / strips));          // (as many workgroups as run at once)
  o.rows_each = ceil_div(ceil_div(t.rows, groups), 16) * 16;
  return start(held == 32 ? outer_kernel<1> : held == 64 ? outer_kernel<2> : outer_kernel<4>, dim3(strips, ceil_div(t.rows, o.rows_each)), s, o);
}

}  // namespace flux_ffn
