// Instantiates the kernel for few rows.
#include "flux_ffn_internal.h"

namespace flux_ffn {

template <bool MX, int HALVES, int BLOCKS, int MB, int SLABS, int RING>
static hipError_t go(const FewArgs& a, hipStream_t s) {
  typedef FewCfg<MX, HALVES, BLOCKS, MB, SLABS, RING> C;
  static_assert(C::NT == 256, "start");
  return start(few_kernel<C>, dim3((a.cols + C::COLS - 1) / C::COLS), s, a);
}

template <bool MX, int HALVES, int BLOCKS>
static hipError_t by_rows(const FewArgs& a, hipStream_t s) {
  // Rows of up to 512 bytes are one turn of one slab a wave, of up to 1 KB two: nothing to look further ahead for, and with less LDS two to
  // four workgroups share a unit.  us, 4-bit gated 5x10328x544: 4.5 so, 8.8 with a ring for long rows.
  const bool one = a.row_vecs <= 32, two = a.row_vecs <= 64;
  if (a.rows <= 16) {
    if (one) return go<MX, HALVES, BLOCKS, 1, 1, 1>(a, s);
    if (two) return go<MX, HALVES, BLOCKS, 1, 1, 2>(a, s);
    if constexpr (MX) return go<MX, HALVES, BLOCKS, 1, 1, 5>(a, s);
    else return go<MX, HALVES, BLOCKS, 1, 2, 3>(a, s);
  }
  if (a.rows <= 32) {
    if (one) return go<MX, HALVES, BLOCKS, 2, 1, 1>(a, s);
    return two ? go<MX, HALVES, BLOCKS, 2, 1, 2>(a, s) : go<MX, HALVES, BLOCKS, 2, 1, 4>(a, s);
  }
  return go<MX, HALVES, BLOCKS, 4, 1, MX ? 2 : 3>(a, s);
}

hipError_t launch_few(int kind, const FewArgs& a, hipStream_t s) {
  if (kind == MX_GEMM) return a.cols > 256 * 16 ? by_rows<true, 1, 2>(a, s) : by_rows<true, 1, 1>(a, s);
  if (kind == MX_GLU) return by_rows<true, 2, 2>(a, s);
  return by_rows<false, 2, 2>(a, s);
}

}  // namespace flux_ffn
