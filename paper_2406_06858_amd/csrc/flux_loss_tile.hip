// Instantiates the tile kernel of logits; compiled once for each of -DFLUX_LOSS_GRADIENT=0 (statistics) and =1 (dZ).
#include "flux_ffn_internal.h"
#include "flux_loss_tile.h"

namespace flux_ffn {

// One row of tiles reads the weights once: past the caches, unless they may be there from the call before, or lines are read in two pieces.
// us, through the caches / past them: 64x128256x4096 222 / 189, 16x128256x4096 178 / 160, 64x32000x2048 44.5 / 41.3; 16x4000x8192 (66 MB) 18.4 / 20.2.
// (The backward pass reads them twice, and the Infinity Cache keeps what is below its 256 MiB: 128x50257x1024, 103 MB, 115 / 124 for the whole pass.)
static bool streams_weights(const TileArgs& a) { return a.tiles_m == 1 && a.bytes_b >= (FLUX_LOSS_GRADIENT ? 192u : 96u) << 20 && a.pitch_b % 128 == 0 && aligned(a.b[0], 128); }

template <int BM, int BN, int NA, int NB, int OCC>
static hipError_t go(const TileArgs& a, const LossArgs& l, bool edge, int grid, hipStream_t s) {
  constexpr bool G = FLUX_LOSS_GRADIENT;
  if constexpr (BM <= 128) {
    if (streams_weights(a))
      return start(edge ? logits_kernel<Cfg<DX_NK, BM, BN, NA, NB, OCC, true, true, true>, G> : logits_kernel<Cfg<DX_NK, BM, BN, NA, NB, OCC, false, true, true>, G>, dim3(grid), s, a, l);
  }
  return start(edge ? logits_kernel<Cfg<DX_NK, BM, BN, NA, NB, OCC, true, false, true>, G> : logits_kernel<Cfg<DX_NK, BM, BN, NA, NB, OCC, false, false, true>, G>, dim3(grid), s, a, l);
}

#if FLUX_LOSS_GRADIENT
#define LAUNCH launch_dz
#else
#define LAUNCH launch_stats
#endif
hipError_t LAUNCH(int shape, const TileArgs& a, const LossArgs& l, bool edge, int grid, hipStream_t s);

hipError_t LAUNCH(int shape, const TileArgs& a, const LossArgs& l, bool edge, int grid, hipStream_t s) {
  switch (shape) {                     // (SHAPES)
    case 0: return go<256, 256, 3, 2, 1>(a, l, edge, grid, s);
    case 1: return go<256, 128, 3, 3, 1>(a, l, edge, grid, s);
    case 2: return go<128, 128, 2, 2, 2>(a, l, edge, grid, s);
    case 3: return go<128, 128, 4, 4, 1>(a, l, edge, grid, s);
    case 4: return go<64, 128, 3, 3, 2>(a, l, edge, grid, s);
    default: return go<64, 128, 6, 6, 1>(a, l, edge, grid, s);
  }
}

}  // namespace flux_ffn
