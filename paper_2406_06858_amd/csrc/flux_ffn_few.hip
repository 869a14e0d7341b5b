// Instantiates the kernel for few rows.
#include "flux_ffn_internal.h"

namespace flux_ffn {

template <bool MX, int HALVES, int BLOCKS, int MB, int SLABS, int RING>
static hipError_t go(const FewArgs& a, hipStream_t s) {
  typedef FewCfg<MX, HALVES, BLOCKS, MB, SLABS, RING> C;
  hipLaunchKernelGGL(few_kernel<C>, dim3((a.cols + C::COLS - 1) / C::COLS), dim3(C::NT), 0, s, a);
  return hipGetLastError();
}

template <bool MX, int HALVES, int BLOCKS>
static hipError_t by_rows(const FewArgs& a, hipStream_t s) {
  // Rows of up to 1 KB are two turns of one slab a wave: nothing to look further ahead for, and with half of the LDS two
  // workgroups share a unit.
  const bool is_short = a.row_vecs <= 64;
  if (a.rows <= 16) return is_short ? go<MX, HALVES, BLOCKS, 1, 1, 2>(a, s) : go<MX, HALVES, BLOCKS, 1, 2, 3>(a, s);
  if (a.rows <= 32) return is_short ? go<MX, HALVES, BLOCKS, 2, 1, 2>(a, s) : go<MX, HALVES, BLOCKS, 2, 1, 4>(a, s);
  return go<MX, HALVES, BLOCKS, 4, 1, 3>(a, s);
}

hipError_t launch_few(int kind, const FewArgs& a, hipStream_t s) {
  if (kind == MX_GEMM) return a.cols > 256 * 16 ? by_rows<true, 1, 2>(a, s) : by_rows<true, 1, 1>(a, s);
  if (kind == MX_GLU) return by_rows<true, 2, 2>(a, s);
  return by_rows<false, 2, 2>(a, s);
}

}  // namespace flux_ffn
