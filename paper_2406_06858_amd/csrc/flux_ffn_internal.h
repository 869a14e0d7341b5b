// Declarations shared by the translation units of libflux_ffn_mi355.so.
#pragma once
#include <hip/hip_runtime.h>
#include "flux_ffn.h"
#include "flux_ffn_tile.h"
#include "flux_ffn_few.h"

namespace flux_ffn {

// Tiles of the tile kernel: rows, columns of products, workgroups per compute unit; and in us (of bf16 operands, of 4-bit ones) what a
// slab takes where every unit has that many workgroups, what it takes with few of them, a workgroup's two ends, and what joining
// the parts of cut tiles adds where they are few and, on top, where every unit has some.  Fitted to 220 problems of random sizes, all
// tiles whole and cut (within 10 to 18 % each in the mean; large 4-bit products on 256x256 tiles are faster than their estimate: 8192x12288x6144 285 us
// for 332, gated 4096x3584x8192 110 for 136).
struct Pace { double slab_us, alone_us, ends_us, join_us, join_all_us; };
struct Shape { int bm, bn, per_unit; Pace pace[2]; };
constexpr Shape SHAPES[] = {
    {256, 256, 1, {{1.34, 1.15, 8.7, 3.7, 8.5}, {1.95, 1.17, 8.5, 4.3, 8.0}}}, {256, 128, 1, {{0.78, 0.55, 6.5, 2.3, 5.5}, {1.21, 0.75, 5.9, 3.2, 5.5}}},
    {128, 128, 2, {{0.93, 0.53, 3.9, 1.8, 9.9}, {1.25, 0.49, 4.6, 2.6, 7.7}}}, {128, 128, 1, {{0.47, 0.37, 4.2, 2.4, 5.2}, {0.63, 0.50, 5.2, 2.8, 4.0}}},
    {64, 128, 2, {{0.63, 0.28, 3.1, 2.1, 9.0}, {0.83, 0.40, 3.9, 2.3, 6.4}}},  {64, 128, 1, {{0.34, 0.30, 3.2, 2.5, 4.8}, {0.41, 0.40, 4.5, 3.0, 2.6}}}};
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
double few_us(int kind, int rows, int cols, int row_vecs);          // estimate of what that kernel takes

// Remembers a failed runtime call for flux_ffn_last_hip_error and returns the status for it.
int hip_failed(hipError_t e);
#define FFN_HIP(call) do { const hipError_t e_ = (call); if (e_ != hipSuccess) return ::flux_ffn::hip_failed(e_); } while (0)

// A launch of 256 threads a workgroup, with the status of this very launch: the runtime's last error may be an earlier one of the caller's
// own, which stays the caller's to fetch.
template <class... A>
inline hipError_t start(void (*kernel)(A...), dim3 grid, hipStream_t s, A... args) {
  void* p[] = {static_cast<void*>(&args)...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(256), p, 0, s);
}

// A matrix spans fewer elements than this.
constexpr long long LIMIT = 1ll << 31;
inline bool below_limit(long long rows, long long pitch, long long cols) {
  return rows == 1 ? cols < LIMIT : pitch < LIMIT && (rows - 1) * pitch + cols < LIMIT;          // (a pitch of any size: no overflow)
}
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline long long row_bytes(long long K) { return (K + 31) / 32 * 16; }
inline long long scale_row_bytes(long long K) { return ((K + 31) / 32 + 15) / 16 * 16; }

}  // namespace flux_ffn
