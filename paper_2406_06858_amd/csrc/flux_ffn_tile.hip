// Instantiates the tile kernel for ONE kind of product; compiled once for each with -DFLUX_FFN_KIND=<Kind> so that they build in
// parallel.
#include "flux_ffn_internal.h"

namespace flux_ffn {

template <int BM, int BN, int NA, int NB, int OCC>
static hipError_t go(const TileArgs& a, bool edge, int grid, hipStream_t s) {
  return start(edge ? tile_kernel<Cfg<FLUX_FFN_KIND, BM, BN, NA, NB, OCC, true>> : tile_kernel<Cfg<FLUX_FFN_KIND, BM, BN, NA, NB, OCC, false>>, dim3(grid), s, a);
}

#define FFN_CAT2(a, b) a##b
#define FFN_CAT(a, b) FFN_CAT2(a, b)

hipError_t FFN_CAT(launch_tile, FLUX_FFN_KIND)(int shape, const TileArgs& a, bool edge, int grid, hipStream_t s) {
  constexpr bool MX = FLUX_FFN_KIND == MX_GEMM || FLUX_FFN_KIND == MX_GLU;
  switch (shape) {                     // (SHAPES)
    case 0: return go<256, 256, MX ? 2 : 3, 2, 1>(a, edge, grid, s);
    case 1: return go<256, 128, MX ? 2 : 3, MX ? 2 : 3, 1>(a, edge, grid, s);
    case 2: return go<128, 128, 2, 2, 2>(a, edge, grid, s);
    case 3: return go<128, 128, 4, 4, 1>(a, edge, grid, s);
    case 4: return go<64, 128, MX ? 2 : 3, MX ? 2 : 3, 2>(a, edge, grid, s);
    default: return go<64, 128, 6, 6, 1>(a, edge, grid, s);
  }
}

}  // namespace flux_ffn
