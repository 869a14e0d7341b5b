// Instantiates the kernel for few rows.
#include <algorithm>
#include "flux_ffn_internal.h"
#include "flux_loss_few.h"

namespace flux_ffn {

// Calls f with the configuration for a product, an empty FewCfg.
template <bool MX, int HALVES, int BLOCKS, class F>
static auto by_rows(int rows, int row_vecs, F f) {
  // Rows of up to 512 bytes are one turn of one slab a wave, of up to 1 KB two: nothing to look further ahead for, and with less LDS two to
  // four workgroups share a unit.  us, 4-bit gated 5x10328x544: 4.5 so, 8.8 with a ring for long rows.
  const bool one = row_vecs <= 32, two = row_vecs <= 64;
  if (rows <= 16) {
    if (one) return f(FewCfg<MX, HALVES, BLOCKS, 1, 1, 1>());
    if (two) return f(FewCfg<MX, HALVES, BLOCKS, 1, 1, 2>());
    if constexpr (MX) return f(FewCfg<MX, HALVES, BLOCKS, 1, 1, 5>());
    else return f(FewCfg<MX, HALVES, BLOCKS, 1, 2, 3>());
  }
  if (rows <= 32) {
    if (one) return f(FewCfg<MX, HALVES, BLOCKS, 2, 1, 1>());
    return two ? f(FewCfg<MX, HALVES, BLOCKS, 2, 1, 2>()) : f(FewCfg<MX, HALVES, BLOCKS, 2, 1, 4>());
  }
  return f(FewCfg<MX, HALVES, BLOCKS, 4, 1, MX ? 2 : 3>());
}

template <class F>
static auto with_config(int kind, int rows, int cols, int row_vecs, F f) {
  // Plain 4-bit products: 16 columns a workgroup while that gives every unit at most one, 32 beyond.  us, 16 / 32 columns at K = 3584: 8x2048
  // 3.9 / 4.6, 8x4096 4.1 / 4.9, 8x4104 5.5 / 4.8, 8x8192 6.6 / 5.3, 64x4104 8.5 / 6.6, 8x28672 18.8 / 16.5; at K = 512, where workgroups share a
  // unit, 8x8192 3.1 / 3.3, 64x8192 6.1 / 4.8.
  if (kind == MX_GEMM) return cols > 256 * 16 ? by_rows<true, 1, 2>(rows, row_vecs, f) : by_rows<true, 1, 1>(rows, row_vecs, f);
  if (kind == LOGITS) return cols > 256 * 16 ? by_rows<false, 1, 2>(rows, row_vecs, f) : by_rows<false, 1, 1>(rows, row_vecs, f);
  if (kind == MX_GLU) return by_rows<true, 2, 2>(rows, row_vecs, f);
  return by_rows<false, 2, 2>(rows, row_vecs, f);
}

hipError_t launch_few(int kind, const FewArgs& a, hipStream_t s) {
  return with_config(kind, a.rows, a.cols, a.row_vecs, [&](auto c) {
    typedef decltype(c) C;
    static_assert(C::NT == 256, "start");
    if constexpr (!C::MX && C::HALVES == 1) return hipErrorInvalidValue;          // (logits: launch_few_logits)
    else return start(few_kernel<C>, dim3((a.cols + C::COLS - 1) / C::COLS), s, a);
  });
}

int few_columns(int kind, int rows, int cols, int row_vecs) {
  return with_config(kind, rows, cols, row_vecs, [](auto c) { return decltype(c)::COLS; });
}

hipError_t launch_few_logits(bool gradient, const FewArgs& a, const LossArgs& l, hipStream_t s) {
  return with_config(LOGITS, a.rows, a.cols, a.row_vecs, [&](auto c) {
    typedef decltype(c) C;
    // (one of with_config's kinds is meant; the others are not built for it)
    if constexpr (!C::MX && C::HALVES == 1) return start(gradient ? few_logits_kernel<C, true> : few_logits_kernel<C, false>, dim3(ceil_div(a.cols, C::COLS)), s, a, l);
    else return hipErrorInvalidValue;
  });
}

// A round of workgroups: its ends, then the weights, as fast as a unit or the memory gives them, and the rows out of the L2.  us and bytes a
// us, fitted to 1190 products of 1 to 64 rows, 64 to 28672 columns and 128 to 28672 numbers: off by 15 % (bf16) and 11 % (4 bits) in the
// mean square, and no more on 597 others.
double few_us(int kind, int rows, int cols, int row_vecs) {
  struct Pace { double ends_us, round_us, weights, rows, all; };
  static constexpr Pace paces[2] = {{1.4, 2.1, 43e3, 57e3, 7.0e6}, {1.2, 2.4, 42e3, 46e3, 7.0e6}};
  const Pace& p = paces[kind >= MX_GEMM];
  struct Shape { int cols, blocks, per_unit; };
  const Shape sh = with_config(kind, rows, cols, row_vecs, [](auto c) {
    typedef decltype(c) C;
    return Shape{C::COLS, C::BLOCKS, std::min(160 * 1024 / C::POOL_BYTES, 8)};
  });
  const double row = row_vecs * 16.0, weights = 16 * sh.blocks * row, all_rows = rows * row;
  const int groups = (cols + sh.cols - 1) / sh.cols, at_once = 256 * sh.per_unit;
  const auto round = [&](int n) {
    const int a_unit = (n + 255) / 256;
    return p.round_us + std::max(a_unit * weights / p.weights, n * weights / p.all) + a_unit * all_rows / p.rows;
  };
  return p.ends_us + groups / at_once * round(at_once) + (groups % at_once ? round(groups % at_once) : 0.0);
}

}  // namespace flux_ffn
