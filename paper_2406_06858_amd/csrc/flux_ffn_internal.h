// Declarations shared by the translation units of libflux_ffn_mi355.so.
#pragma once
#include <hip/hip_runtime.h>
#include "flux_ffn.h"
#include "flux_ffn_tile.h"
#include "flux_ffn_few.h"

namespace flux_ffn {

// Tiles of the tile kernel: rows, columns of products, workgroups per compute unit; and in us, what a slab takes where every unit
// has that many, what it takes with one a unit, a workgroup's two ends, and what joining the parts of a cut tile adds.
struct Shape { int bm, bn, per_unit; double slab_us, alone_us, ends_us, join_us; };
constexpr Shape SHAPES[] = {{256, 256, 1, 1.35, 1.28, 8.0, 10.0}, {256, 128, 1, 0.8, 0.8, 5.0, 5.0}, {128, 128, 2, 1.05, 0.85, 5.0, 4.0},
                            {128, 128, 1, 0.57, 0.55, 5.0, 3.0},  {64, 128, 2, 0.75, 0.48, 4.0, 3.0}, {64, 128, 1, 0.43, 0.43, 4.0, 2.0}};
constexpr int N_SHAPES = 6;

#define FFN_DECLARE(KIND) hipError_t launch_tile##KIND(int shape, const TileArgs& a, bool edge, int grid, hipStream_t s);
FFN_DECLARE(0)
FFN_DECLARE(1)
FFN_DECLARE(2)
FFN_DECLARE(3)
FFN_DECLARE(4)
FFN_DECLARE(5)
FFN_DECLARE(6)
#undef FFN_DECLARE

// Products of at most this many rows whose weights lie along the contraction (GLU_NK and the 4-bit kinds).
constexpr int FEW_ROWS = 64;
hipError_t launch_few(int kind, const FewArgs& a, hipStream_t s);

// Remembers a failed runtime call for flux_ffn_last_hip_error and returns the status for it.
int hip_failed(hipError_t e);
#define FFN_HIP(call) do { const hipError_t e_ = (call); if (e_ != hipSuccess) return ::flux_ffn::hip_failed(e_); } while (0)

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline long long row_bytes(long long K) { return (K + 31) / 32 * 16; }
inline long long scale_row_bytes(long long K) { return ((K + 31) / 32 + 15) / 16 * 16; }

}  // namespace flux_ffn
