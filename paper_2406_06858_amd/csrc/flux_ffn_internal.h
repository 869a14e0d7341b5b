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

#define FFN_DECLARE(NAME) hipError_t launch_##NAME(int shape, const TileArgs& a, bool edge, int grid, hipStream_t s);
FFN_DECLARE(tile0)
FFN_DECLARE(tile1)
FFN_DECLARE(tile2)
FFN_DECLARE(tile3)
FFN_DECLARE(tile4)
FFN_DECLARE(tile5)
FFN_DECLARE(tile6)
FFN_DECLARE(scaled3)
FFN_DECLARE(scaled4)
#undef FFN_DECLARE

// How a product is run.
struct Plan {
  int shape = 0, full = 0, cut = 0, parts = 1, part_slabs = 0, slabs = 0, tiles_m = 0, tiles_n = 0;
  bool edge = false, few = false;
  size_t partial_bytes = 0;
};
// depth: pieces of two bytes of (a segment of) the contraction; config, want_parts: the caller's choice, 0 for the library's; segs: segments of the
// contraction (dX); jobs: products in one grid (dW).
Plan plan_tiles(int kind, int rows, int cols, int depth, int config, int want_parts, int segs = 1, int jobs = 1);
int launch(int kind, const Plan& pl, TileArgs& t, void* ws, size_t partial_at, hipStream_t s);

// The workspace begins with a word a cut tile, zero between calls.
constexpr size_t WS_HEADER = 512 * COUNTER_STRIDE * 4;
inline void set_tiles(TileArgs& t, const Plan& pl, void* ws, size_t partial_at) {
  t.slabs = pl.slabs;
  t.seg_slabs = (t.depth + 63) / 64;
  t.full_tiles = pl.full;
  t.cut_tiles = pl.cut;
  t.parts = pl.parts;
  t.part_slabs = pl.part_slabs;
  t.tiles_m = pl.tiles_m;
  t.tiles_n = pl.tiles_n;
  t.band = pl.tiles_m < 8 ? pl.tiles_m : 8;
  t.counters = static_cast<uint32_t*>(ws);
  t.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + partial_at);
}

constexpr int FEW_CONFIG = N_SHAPES + 1;        // id of the kernel for few rows
inline bool choice_ok(int config, int parts) { return config >= 0 && config <= FEW_CONFIG && parts >= 0 && parts <= 64; }
bool few_fits(int kind, int rows, int cols);

// Products of at most this many rows whose weights lie along the contraction (GLU_NK and the 4-bit kinds).
constexpr int FEW_ROWS = 64;
hipError_t launch_few(int kind, const FewArgs& a, hipStream_t s);
int few_columns(int kind, int rows, int cols, int row_vecs);         // of a workgroup
struct LossArgs;
hipError_t launch_few_logits(bool gradient, const FewArgs& a, const LossArgs& l, hipStream_t s);
double few_us(int kind, int rows, int cols, int row_vecs);          // estimate of what that kernel takes

// Remembers a failed runtime call for flux_ffn_last_hip_error and returns the status for it.
int hip_failed(hipError_t e);
#define FFN_HIP(call) do { const hipError_t e_ = (call); if (e_ != hipSuccess) return ::flux_ffn::hip_failed(e_); } while (0)

// A launch of 256 threads a workgroup (or `threads`), with the status of this very launch: the runtime's last error may be an earlier one of the caller's
// own, which stays the caller's to fetch.
template <class... A>
inline hipError_t start_with(void (*kernel)(A...), dim3 grid, int threads, hipStream_t s, A... args) {
  void* p[] = {static_cast<void*>(&args)...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), p, 0, s);
}
template <class... A>
inline hipError_t start(void (*kernel)(A...), dim3 grid, hipStream_t s, A... args) { return start_with(kernel, grid, 256, s, args...); }

// A matrix spans fewer elements than this.
constexpr long long LIMIT = 1ll << 31;
inline bool below_limit(long long rows, long long pitch, long long cols) {
  return rows == 1 ? cols < LIMIT : pitch < LIMIT && (rows - 1) * pitch + cols < LIMIT;          // (a pitch of any size: no overflow)
}
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool pitch_ok(long long pitch, long long rows, long long cols) { return pitch >= cols && pitch % 8 == 0 && below_limit(rows, pitch, cols); }
inline bool dtype_ok(int d) { return d == FLUX_BF16 || d == FLUX_F32; }
inline int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
inline uint32_t extent(long long rows, long long pitch, long long row) { return (uint32_t)((rows - 1) * pitch + row); }
inline int workspace_ok(size_t need, const void* ws, size_t bytes) {
  if (need == 0) return FLUX_OK;
  return ws != nullptr && aligned(ws, 16) && bytes >= need ? FLUX_OK : FLUX_ERR_WORKSPACE;
}
inline long long row_bytes(long long K) { return (K + 31) / 32 * 16; }
inline long long scale_row_bytes(long long K) { return ((K + 31) / 32 + 15) / 16 * 16; }

}  // namespace flux_ffn
