// Declarations shared by the translation units of libflux_ffn_mi355.so.
#pragma once
#include <hip/hip_runtime.h>
#include "flux_ffn.h"
#include "flux_ffn_tile.h"
#include "flux_ffn_few.h"

namespace flux_ffn {

// Tiles of the tile kernel: rows, columns of products, workgroups per compute unit; and in us (of bf16 operands, of 4-bit ones) what a
// slab takes where every unit has that many workgroups, what it takes with few of them, a workgroup's two ends, and what joining
// the parts of a cut tile adds.  Fitted to 220 problems of random sizes, all tiles whole and cut (within 12 to 22 % each; the tile that
// is picked so takes 4 % longer than the best of them in the mean).
struct Pace { double slab_us, alone_us, ends_us, join_us; };
struct Shape { int bm, bn, per_unit; Pace pace[2]; };
constexpr Shape SHAPES[] = {
    {256, 256, 1, {{1.46, 1.10, 8.6, 6.3}, {2.20, 1.10, 8.3, 6.1}}}, {256, 128, 1, {{0.82, 0.52, 6.5, 4.2}, {1.29, 0.70, 6.0, 4.7}}},
    {128, 128, 2, {{1.03, 0.49, 3.8, 4.7}, {1.38, 0.44, 4.6, 4.2}}}, {128, 128, 1, {{0.49, 0.35, 4.2, 4.3}, {0.65, 0.47, 5.2, 3.9}}},
    {64, 128, 2, {{0.69, 0.25, 3.1, 4.8}, {0.88, 0.36, 3.9, 3.7}}},  {64, 128, 1, {{0.35, 0.29, 3.2, 4.4}, {0.41, 0.39, 4.5, 3.7}}}};
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
