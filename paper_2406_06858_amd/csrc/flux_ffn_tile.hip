// Instantiates the tile kernel for ONE kind of product; compiled once for each with -DFLUX_FFN_KIND=<Kind> so that they build in
// parallel.
#include "flux_ffn_internal.h"

namespace flux_ffn {

template <int BM, int BN, int NA, int NB, int OCC>
static hipError_t go(const TileArgs& a, bool edge, int grid, hipStream_t s) {
  if (edge) hipLaunchKernelGGL((tile_kernel<Cfg<FLUX_FFN_KIND, BM, BN, NA, NB, OCC, true>>), dim3(grid), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((tile_kernel<Cfg<FLUX_FFN_KIND, BM, BN, NA, NB, OCC, false>>), dim3(grid), dim3(256), 0, s, a);
  return hipGetLastError();
}

#define FFN_CAT2(a, b) a##b
#define FFN_CAT(a, b) FFN_CAT2(a, b)

hipError_t FFN_CAT(launch_tile, FLUX_FFN_KIND)(int shape, const TileArgs& a, bool edge, int grid, hipStream_t s) {
  constexpr int NA = FLUX_FFN_KIND == MX_GEMM || FLUX_FFN_KIND == MX_GLU ? 2 : 3;
  if (shape == 0) return go<256, 256, NA, 2, 1>(a, edge, grid, s);
  return go<128, 128, 2, 2, 2>(a, edge, grid, s);
}

}  // namespace flux_ffn
