// Softmax cross entropy of a vocabulary projection: checks of arguments, the join of statistics, dispatch.
#include <algorithm>
#include "flux_ffn_internal.h"
#include "flux_loss.h"
#include "flux_loss_tile.h"

namespace flux_ffn {

hipError_t launch_stats(int shape, const TileArgs& a, const LossArgs& l, bool edge, int grid, hipStream_t s);
hipError_t launch_dz(int shape, const TileArgs& a, const LossArgs& l, bool edge, int grid, hipStream_t s);

hipError_t launch_dx_few(int shape, const TileArgs& a, int grid, hipStream_t s);
int outer_terms(int M);
hipError_t launch_dw_few(const TileArgs& t, const void* dz, long long ldz, const void* X, long long ldx, void* scratch, int M, hipStream_t s);

// ---- joins ----------------------------------------------------------------------------------------------------
// lse = m + log(s) over all runs of columns of a row; then the loss.  A workgroup takes ROWS rows, whose statistics lie side by side, and shares out the runs among
// 256 / ROWS lanes a row; these meet in LDS, in ascending order.  (Of few rows with many runs a workgroup takes few: 1496 rows of 394 runs 6.3 us with four, 12.4
// with sixteen.)
struct StatsArgs {
  const float2* stats;           // [runs][rows]
  int32_t runs, rows, cols;
  LossArgs loss;
  float *lse, *logit, *value;
};
template <int ROWS>
__global__ void __launch_bounds__(256) stats_kernel(const StatsArgs a) {
  constexpr int LANES = 256 / ROWS;
  __shared__ float2 part[LANES][ROWS];
  const int r = threadIdx.x % ROWS, lane = threadIdx.x / ROWS, row = blockIdx.x * ROWS + r;
  float m = -__builtin_inff(), s = 0.f;
  if (row < a.rows) {
#pragma unroll 4
    for (int i = lane; i < a.runs; i += LANES) {
      const float2 v = a.stats[(long long)i * a.rows + row];
      join_stats(m, s, v.x, v.y);
    }
  }
  part[lane][r] = make_float2(m, s);
  for (int n = LANES / 2; n > 0; n /= 2) {
    __syncthreads();
    if (lane < n) {
      join_stats(m, s, part[lane + n][r].x, part[lane + n][r].y);
      part[lane][r] = make_float2(m, s);
    }
  }
  if (lane != 0 || row >= a.rows) return;
  const float lse = (__builtin_fabsf(m) == __builtin_inff() ? 0.f : m) + logf(s);
  bool counts;
  const int target = target_column(a.loss, row, a.cols, counts);
  const float z = target >= 0 ? a.logit[row] : 0.f;
  a.lse[row] = lse;
  if (target < 0) a.logit[row] = 0.f;
  if (a.value != nullptr) a.value[row] = counts ? lse - z : 0.f;
}

// D, the largest |dloss| of the rows that count, where a tile has not all rows.  One workgroup of NT lanes; eight rows a lane are asked for together.
template <class T, int NT>
__device__ __forceinline__ void find_most(const LossArgs& l, int rows, float* most) {
  __shared__ float part[NT / 64];
  const T* const target = static_cast<const T*>(l.target);
  float m = 0.f;
  for (int from = threadIdx.x; from < rows; from += 8 * NT) {
    T t[8];
    float d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = min(from + i * NT, rows - 1);          // (past the end: the last again)
      t[i] = target[row];
      d[i] = l.dloss[row];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, t[i] >= 0 && (long long)t[i] < l.vocab ? __builtin_fabsf(d[i]) : 0.f);
  }
  m = wave_max(m);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = m;
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) m = fmaxf(m, part[i]);
  *most = sane_most(m);
}
template <int NT>
__device__ __forceinline__ void find_most_of(const LossArgs& l, int rows, float* most) {
  if (l.target_i64) find_most<long long, NT>(l, rows, most);
  else find_most<int32_t, NT>(l, rows, most);
}
__global__ void __launch_bounds__(1024) most_kernel(const LossArgs l, int rows, float* most) { find_most_of<1024>(l, rows, most); }

// X in rows of whole lines, for products that read it many times.  A workgroup takes rows in steps of all workgroups.  Where `most` is asked for, one workgroup more
// finds it: a launch of its own takes 5 us.
__global__ void __launch_bounds__(256) whole_rows_kernel(const uint4* from, uint4* to, long long pitch, long long to_pitch, int rows, int row_vecs, const LossArgs l, float* most) {
  const int step = gridDim.x - (most != nullptr);
  if ((int)blockIdx.x == step) {
    find_most_of<256>(l, rows, most);
    return;
  }
  for (int row = blockIdx.x; row < rows; row += step)
    for (int i = threadIdx.x; i < row_vecs; i += 256) to[row * to_pitch + i] = from[row * pitch + i];
}

struct RanksArgs {
  const float* lse[FLUX_MAX_RANKS];
  const float* logit[FLUX_MAX_RANKS];
  int32_t ranks, rows;
  LossArgs loss;
  float *to_lse, *to_logit, *value;
};
__global__ void __launch_bounds__(256) ranks_kernel(const RanksArgs a) {
  const int row = blockIdx.x * 256 + threadIdx.x;
  if (row >= a.rows) return;
  float m = -__builtin_inff(), s = 0.f, z = 0.f;
  for (int r = 0; r < a.ranks; ++r) {
    join_stats(m, s, a.lse[r][row], 1.f);
    z += a.logit[r][row];
  }
  const float lse = (__builtin_fabsf(m) == __builtin_inff() ? 0.f : m) + logf(s);
  bool counts;
  (void)target_column(a.loss, row, 0, counts);
  if (a.to_lse != nullptr) a.to_lse[row] = lse;
  if (a.to_logit != nullptr) a.to_logit[row] = z;
  if (a.value != nullptr) a.value[row] = counts ? lse - z : 0.f;
}

// ---- checks ----------------------------------------------------------------------------------------------------
static long long pitch_x(const flux_loss_t* p) { return p->ldx ? p->ldx : p->K; }
static long long pitch_w(const flux_loss_t* p) { return p->ldw ? p->ldw : p->K; }
static long long vocab_of(const flux_loss_t* p) { return p->vocab ? p->vocab : p->v0 + p->V; }
constexpr long long MAX_VOCAB = 1ll << 62, MAX_LOGITS = 1ll << 36;          // (with V <= 2^28 below 2^24 workgroups of the smallest tile, both sides rounded up: 2^32 threads)
constexpr int MAX_ROWS = 1 << 27;
constexpr int MAX_WIDTH = 1 << 28;          // of gradients: a result's place in its row is counted in bytes, in 32 bits (store_pair)

static int validate(int op, const flux_loss_t* p) {
  if (p == nullptr || (op != FLUX_LOSS_FORWARD && op != FLUX_LOSS_BACKWARD)) return FLUX_ERR_INVALID_ARG;
  if ((p->target_dtype != FLUX_TARGET_I32 && p->target_dtype != FLUX_TARGET_I64) || !dtype_ok(p->dx_dtype) || !dtype_ok(p->dw_dtype)) return FLUX_ERR_INVALID_ARG;
  if ((p->dloss_one | 1) != 1 || (p->dw_accumulate | 1) != 1 || p->reserved != 0 || !choice_ok(p->tile_config, p->split_k)) return FLUX_ERR_INVALID_ARG;
  if (p->ldx < 0 || p->ldw < 0 || p->v0 < 0 || p->vocab < 0 || p->piece < 0) return FLUX_ERR_INVALID_ARG;
  if (p->M < 1 || p->V < 1 || p->K < 1 || p->K % 8 != 0 || p->piece % 64 != 0) return FLUX_ERR_SHAPE;
  if (p->v0 > MAX_VOCAB || p->vocab > MAX_VOCAB || vocab_of(p) < p->v0 + p->V) return FLUX_ERR_SHAPE;
  if (!pitch_ok(pitch_x(p), p->M, p->K) || !pitch_ok(pitch_w(p), p->V, p->K)) return FLUX_ERR_SHAPE;
  if (op == FLUX_LOSS_BACKWARD && p->K > MAX_WIDTH) return FLUX_ERR_SHAPE;
  if (p->M > MAX_ROWS || (long long)p->M * p->V > MAX_LOGITS) return FLUX_ERR_SHAPE;
  if (p->tile_config == FEW_CONFIG && !few_fits(LOGITS, p->M, p->V)) return FLUX_ERR_UNSUPPORTED;
  return FLUX_OK;
}

// ---- plans -----------------------------------------------------------------------------------------------------
static Plan plan_z(const flux_loss_t* p, int cols) { return plan_tiles(LOGITS, p->M, cols, p->K, p->tile_config, p->split_k); }
// (dX runs over the weights' rows, cols of them, though dZ is in whole vectors of 8: of 57 to 63 the masked kernel has to be the one, since the other would read up to seven
// rows more than there are, for dZ's zeros)
static Plan plan_dx(const flux_loss_t* p, int cols) { return plan_tiles(DX_KN, p->M, p->K, cols, 0, 0); }
static Plan plan_dw(const flux_loss_t* p, int cols) { return plan_tiles(DW, cols, p->K, p->M, 0, 0); }

// Columns of the backward pass's pieces, the last one's apart.  dZ of a piece takes 256 MiB, what the Infinity Cache holds: in smaller ones dX is added to the more
// often, larger ones take memory and give nothing.  (Of few rows it is the whole vocabulary: W is read from memory twice, for Z and for dX.)  us of 8192x32000x8192 by columns a piece: 2048 10650, 4096 9530, 8192 9050, 16384 8960, 32768 8990.
static long long whole_lines(long long n) { return (n + 63) / 64 * 64; }
static int piece_of(const flux_loss_t* p) {
  const long long all = whole_lines(p->V);
  if (p->piece) return (int)std::min<long long>(p->piece, all);
  long long most = std::max(2048ll, (256ll << 20) / 2 / std::max(p->M, FEW_ROWS) / 256 * 256);
  while (most > 64 && p->M * most >= LIMIT) most /= 2;
  return (int)std::min(all, most);
}
static bool dz_fits(const flux_loss_t* p) { return p->M * (long long)piece_of(p) < LIMIT; }
static size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Whether X is laid out anew: a slab's loads, 128 bytes a row, are two lines each where rows are no whole lines, and every column tile reads X.  us, X as it is / laid
// out anew by the caller: statistics of 1496x50257x5112 (256x256 tiles) 729 / 678, 8192x4000x5112 252 / 244, 2328x4096x7640 (256x128) 175 / 135, 512x8000x5112
// (128x128) 58.6 / 49.2; gradients of 1496x6283x5112 279 / 262: 5 to 7 % of the products that read X on the largest tiles, 12 to 23 % on the others, which read X
// for fewer columns each.  Against that, a launch and a pass of 4.5 TB/s.  The copy's rows are longer than X's: it is a matrix below 2^31 elements too, or is not made.
static bool lays_out_x(int op, const flux_loss_t* p, const Plan& z) {
  if (pitch_x(p) % 64 == 0 || z.few || !below_limit(p->M, whole_lines(p->K), p->K)) return false;
  const double gflop = 2e-9 * p->M * p->V * p->K, gain_us = z.shape == 0 ? 0.046 * gflop : 0.15 * gflop;
  return gain_us * (op == FLUX_LOSS_BACKWARD ? 2 : 1) > 2.0 + 4.0 * p->M * p->K / 4.5e6;
}
static size_t x_bytes(int op, const flux_loss_t* p, const Plan& z) { return lays_out_x(op, p, z) ? up256(2ull * p->M * whole_lines(p->K)) : 0; }

// Whether dW is taken as an outer product, and not on tiles.  us of the whole call, so / on tiles: 1x32000x8192 288 / 320, 100x32000x8192 392 / 454, 100x4000x8192
// 70 / 73; 200x4000x8192 107 / 90 (its registers leave room for two workgroups a unit then), 100x1000x1000 25.4 / 21.7 (two launches).
static bool outer(const flux_loss_t* p) { return p->M <= 128 && (long long)p->V * p->K >= 1 << 23; }

// The backward pass's workspace: the header, D, X in whole lines, dZ of a piece, dX in fp32 where its pieces are summed for a result in bf16, the cut tiles' sums.
constexpr size_t MOST_BYTES = 256;
struct Layout {
  size_t dz, sums, partial, all;
  bool lays_out;
  Plan z[2], dx[2], dw[2];           // of the pieces before the last one, and of the last
};
static Layout layout(const flux_loss_t* p) {
  const int piece = piece_of(p), last = p->V - (p->V - 1) / piece * piece;
  Layout y;
  size_t most = outer(p) ? 2ull * outer_terms(p->M) * (piece + (size_t)p->K) : 0;          // (dW of few rows: dZ and X transposed)
  for (int i = 0; i < 2; ++i) {
    const int cols = i ? last : std::min(piece, p->V);
    if (i && cols == std::min(piece, p->V)) {
      y.z[1] = y.z[0];
      y.dx[1] = y.dx[0];
      y.dw[1] = y.dw[0];
      break;
    }
    y.z[i] = plan_z(p, cols);
    y.dx[i] = plan_dx(p, cols);
    if (!outer(p)) y.dw[i] = plan_dw(p, cols);
    for (const Plan* pl : {&y.z[i], &y.dx[i], &y.dw[i]}) most = std::max(most, pl->partial_bytes);
  }
  const size_t x = x_bytes(FLUX_LOSS_BACKWARD, p, y.z[0]);
  y.lays_out = x != 0;
  y.dz = WS_HEADER + MOST_BYTES + x;
  y.sums = y.dz + up256(2ull * p->M * piece);
  y.partial = y.sums + (p->V > piece && p->dx_dtype == FLUX_BF16 ? up256(4ull * ((p->M - 1ull) * pitch_x(p) + p->K)) : 0);
  y.all = y.partial + most;
  return y;
}

// A forward pass's: the header, X in whole lines, the statistics, the cut tiles' sums.
static int runs_of(const flux_loss_t* p, const Plan& pl) { return pl.few ? ceil_div(p->V, few_columns(LOGITS, p->M, p->V, p->K / 8)) : 2 * pl.tiles_n; }
static size_t stats_bytes(const flux_loss_t* p, const Plan& pl) { return up256(8ull * p->M * runs_of(p, pl)); }

static LossArgs loss_args(const flux_loss_t* p, const void* target) {
  LossArgs l = {};
  l.target = target;
  l.target_i64 = p->target_dtype == FLUX_TARGET_I64;
  l.dloss_one = p->dloss_one;
  l.v0 = p->v0;
  l.vocab = vocab_of(p);
  return l;
}

static TileArgs logits_args(const flux_loss_t* p, const void* X, long long lx, const void* W, int v, int cols) {
  TileArgs t = {};
  const long long lw = pitch_w(p);
  t.a[0] = X;
  t.b[0] = static_cast<const __bf16*>(W) + v * lw;
  t.pitch_a = (uint32_t)(lx * 2);
  t.pitch_b = (uint32_t)(lw * 2);
  t.bytes_a = extent(p->M, lx * 2, p->K * 2ll);
  t.bytes_b = extent(cols, lw * 2, p->K * 2ll);
  t.rows = p->M;
  t.cols = cols;
  t.depth = p->K;
  return t;
}

// From here on X and its pitch are those of the copy.
static int lay_out_x(const flux_loss_t* p, const void*& X, long long& lx, char* to, const LossArgs& l, float* most, hipStream_t s) {
  const long long pitch = whole_lines(p->K);
  FFN_HIP(start(whole_rows_kernel, dim3(std::min(p->M, 1 << 16) + (most != nullptr)), s, static_cast<const uint4*>(X), reinterpret_cast<uint4*>(to), lx / 8, pitch / 8, (int)p->M, p->K / 8, l, most));
  X = to;
  lx = pitch;
  return FLUX_OK;
}

static int launch_logits(bool gradient, const Plan& pl, TileArgs& t, const LossArgs& l, void* ws, size_t partial_at, hipStream_t s) {
  if (pl.few) {
    FewArgs f = {};
    f.a = t.a[0];
    f.b[0] = f.b[1] = t.b[0];
    f.pitch_a = t.pitch_a;
    f.pitch_b = t.pitch_b;
    f.bytes_a = t.bytes_a;
    f.bytes_b = t.bytes_b;
    f.rows = t.rows;
    f.cols = t.cols;
    f.row_vecs = t.depth / 8;
    f.ld = t.ld;
    FFN_HIP(launch_few_logits(gradient, f, l, s));
    return FLUX_OK;
  }
  set_tiles(t, pl, ws, partial_at);
  FFN_HIP((gradient ? launch_dz : launch_stats)(pl.shape, t, l, pl.edge, pl.full + pl.cut * pl.parts, s));
  return FLUX_OK;
}

}  // namespace flux_ffn

using namespace flux_ffn;

extern "C" {

size_t flux_loss_workspace_bytes(int op, const flux_loss_t* p) {
  if (validate(op, p) != FLUX_OK) return 0;
  if (op == FLUX_LOSS_BACKWARD) return dz_fits(p) ? layout(p).all : 0;
  const Plan pl = plan_z(p, p->V);
  return WS_HEADER + x_bytes(op, p, pl) + stats_bytes(p, pl) + pl.partial_bytes;
}

int flux_loss(const flux_loss_t* p, const void* X, const void* W, const void* target, float* lse, float* logit, float* loss, void* workspace,
              size_t workspace_bytes, void* stream) {
  int st = validate(FLUX_LOSS_FORWARD, p);
  if (st != FLUX_OK) return st;
  const int target_bytes = p->target_dtype == FLUX_TARGET_I64 ? 8 : 4;
  if (X == nullptr || W == nullptr || !aligned(X, 16) || !aligned(W, 16) || target == nullptr || !aligned(target, target_bytes)) return FLUX_ERR_INVALID_ARG;
  if (lse == nullptr || logit == nullptr || !aligned(lse, 4) || !aligned(logit, 4) || !aligned(loss, 4)) return FLUX_ERR_INVALID_ARG;
  const Plan pl = plan_z(p, p->V);
  const size_t stats_at = WS_HEADER + x_bytes(FLUX_LOSS_FORWARD, p, pl), partial_at = stats_at + stats_bytes(p, pl);
  st = workspace_ok(partial_at + pl.partial_bytes, workspace, workspace_bytes);
  if (st != FLUX_OK) return st;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  StatsArgs a = {};
  a.loss = loss_args(p, target);
  a.loss.stats = reinterpret_cast<float2*>(static_cast<char*>(workspace) + stats_at);
  a.loss.logit = logit;
  long long lx = pitch_x(p);
  if (stats_at != WS_HEADER) {
    st = lay_out_x(p, X, lx, static_cast<char*>(workspace) + WS_HEADER, a.loss, nullptr, s);
    if (st != FLUX_OK) return st;
  }
  TileArgs t = logits_args(p, X, lx, W, 0, p->V);
  st = launch_logits(false, pl, t, a.loss, workspace, partial_at, s);
  if (st != FLUX_OK) return st;
  a.stats = a.loss.stats;
  a.runs = runs_of(p, pl);
  a.rows = p->M;
  a.cols = p->V;
  a.lse = lse;
  a.logit = logit;
  a.value = loss;
  if (p->M > 4096) FFN_HIP(start(stats_kernel<16>, dim3(ceil_div(p->M, 16)), s, a));
  else if (p->M > 256) FFN_HIP(start(stats_kernel<4>, dim3(ceil_div(p->M, 4)), s, a));
  else FFN_HIP(start(stats_kernel<1>, dim3(p->M), s, a));
  return FLUX_OK;
}

int flux_loss_join(const flux_loss_t* p, int32_t R, const float* const* lses, const float* const* logits, const void* target, float* lse,
                   float* logit, float* loss, void* stream) {
  if (p == nullptr || R < 1 || R > FLUX_MAX_RANKS || lses == nullptr || logits == nullptr || target == nullptr) return FLUX_ERR_INVALID_ARG;
  if ((p->target_dtype != FLUX_TARGET_I32 && p->target_dtype != FLUX_TARGET_I64) || p->v0 < 0 || p->vocab < 0) return FLUX_ERR_INVALID_ARG;
  if (p->M < 1 || p->V < 1 || p->v0 > MAX_VOCAB || p->vocab > MAX_VOCAB) return FLUX_ERR_SHAPE;
  if (!aligned(target, p->target_dtype == FLUX_TARGET_I64 ? 8 : 4)) return FLUX_ERR_INVALID_ARG;
  RanksArgs a = {};
  for (int r = 0; r < R; ++r) {
    if (lses[r] == nullptr || logits[r] == nullptr || !aligned(lses[r], 4) || !aligned(logits[r], 4)) return FLUX_ERR_INVALID_ARG;
    a.lse[r] = lses[r];
    a.logit[r] = logits[r];
  }
  if (!aligned(lse, 4) || !aligned(logit, 4) || !aligned(loss, 4)) return FLUX_ERR_INVALID_ARG;
  a.ranks = R;
  a.rows = p->M;
  a.loss = loss_args(p, target);
  a.to_lse = lse;
  a.to_logit = logit;
  a.value = loss;
  FFN_HIP(start(ranks_kernel, dim3(ceil_div(p->M, 256)), static_cast<hipStream_t>(stream), a));
  return FLUX_OK;
}

int flux_loss_backward(const flux_loss_t* p, const void* X, const void* W, const void* target, const float* lse, const float* dloss, void* dX,
                       void* dW, void* workspace, size_t workspace_bytes, void* stream) {
  int st = validate(FLUX_LOSS_BACKWARD, p);
  if (st != FLUX_OK) return st;
  if (!dz_fits(p)) return FLUX_ERR_SHAPE;
  const int target_bytes = p->target_dtype == FLUX_TARGET_I64 ? 8 : 4;
  if (X == nullptr || W == nullptr || !aligned(X, 16) || !aligned(W, 16) || target == nullptr || !aligned(target, target_bytes)) return FLUX_ERR_INVALID_ARG;
  if (lse == nullptr || dloss == nullptr || !aligned(lse, 4) || !aligned(dloss, 4) || !aligned(dX, 16) || !aligned(dW, 16)) return FLUX_ERR_INVALID_ARG;
  const Layout y = layout(p);
  st = workspace_ok(y.all, workspace, workspace_bytes);
  if (st != FLUX_OK) return st;
  if (dX == nullptr && dW == nullptr) return FLUX_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  char* const ws = static_cast<char*>(workspace);
  __bf16* const dz = reinterpret_cast<__bf16*>(ws + y.dz);
  float* const sums = reinterpret_cast<float*>(ws + y.sums);
  long long lx = pitch_x(p);
  const long long lw = pitch_w(p);
  const int piece = piece_of(p);
  float* const most = reinterpret_cast<float*>(ws + WS_HEADER);
  const float* const factor = p->dloss_one ? dloss : most;
  const auto finds = [&](const Plan& pl) { return !p->dloss_one && (pl.few || pl.tiles_m == 1); };
  const bool wants_most = !p->dloss_one && !finds(y.z[0]);
  LossArgs of_rows = loss_args(p, target);
  of_rows.dloss = dloss;
  if (y.lays_out) {
    st = lay_out_x(p, X, lx, ws + WS_HEADER + MOST_BYTES, of_rows, wants_most ? most : nullptr, s);
    if (st != FLUX_OK) return st;
  } else if (wants_most) {
    FFN_HIP(start_with(most_kernel, dim3(1), 1024, s, of_rows, (int)p->M, most));
  }
  for (int v = 0; v < p->V; v += piece) {
    const int of = p->V - v <= piece, cols = std::min(piece, p->V - v), held = (cols + 7) / 8 * 8;
    const long long ldz = whole_lines(cols);
    const uint32_t bytes_z = extent(p->M, ldz * 2, held * 2ll);
    {
      const Plan& pl = y.z[of];
      TileArgs t = logits_args(p, X, lx, W, v, cols);
      t.ld = ldz;
      LossArgs l = loss_args(p, target);
      l.v0 += v;
      l.lse = lse;
      l.dloss = dloss;
      l.most = most;
      l.finds_most = finds(pl);
      l.dz = dz;
      st = launch_logits(true, pl, t, l, ws, y.partial, s);
      if (st != FLUX_OK) return st;
    }
    if (dX != nullptr) {
      const bool first = v == 0, last = p->V - v <= piece, f32 = p->dx_dtype == FLUX_F32;
      TileArgs t = {};
      t.a[0] = dz;
      t.b[0] = static_cast<const __bf16*>(W) + v * lw;
      t.pitch_a = (uint32_t)(ldz * 2);
      t.pitch_b = (uint32_t)(lw * 2);
      t.bytes_a = bytes_z;
      t.bytes_b = extent(cols, lw * 2, p->K * 2ll);
      t.rows = p->M;
      t.cols = p->K;
      t.depth = cols;
      t.ld = pitch_x(p);
      // sums of pieces stay in fp32: in dX, or in the workspace until the last piece rounds them
      t.out_f32 = f32 || !last;
      t.out[0] = f32 || last ? dX : sums;
      t.addend = first ? nullptr : f32 ? static_cast<const float*>(dX) : sums;
      t.factor = factor;
      const Plan& pl = y.dx[of];
      if (pl.tiles_m == 1 && pl.shape >= 2 && t.bytes_b >= 192u << 20 && lw % 64 == 0) {
        set_tiles(t, pl, ws, y.partial);
        FFN_HIP(launch_dx_few(pl.shape, t, pl.full + pl.cut * pl.parts, s));
      } else {
        st = launch(DX_KN, pl, t, ws, y.partial, s);
      }
      if (st != FLUX_OK) return st;
    }
    if (dW != nullptr) {
      TileArgs t = {};
      t.a[0] = dz;
      t.b[0] = X;
      t.pitch_a = (uint32_t)(ldz * 2);
      t.pitch_b = (uint32_t)(lx * 2);
      t.bytes_a = bytes_z;
      t.bytes_b = extent(p->M, lx * 2, p->K * 2ll);
      t.rows = cols;
      t.cols = p->K;
      t.depth = p->M;
      t.out_f32 = p->dw_dtype == FLUX_F32;
      t.accumulate = p->dw_accumulate;
      t.factor = factor;
      t.ld = lw;
      t.out[0] = static_cast<char*>(dW) + v * lw * (t.out_f32 ? 4 : 2);
      if (outer(p)) {
        t.stream = lw * (t.out_f32 ? 4 : 2) % 128 == 0 && aligned(t.out[0], 128);          // (parts of lines stay in the caches: us, so / past them, 31x35072x840 19 / 33, 7x2665x11624 17 / 31)
        FFN_HIP(launch_dw_few(t, dz, ldz, X, lx, ws + y.partial, p->M, s));
      } else {
        st = launch(DW, y.dw[of], t, ws, y.partial, s);
      }
      if (st != FLUX_OK) return st;
    }
  }
  return FLUX_OK;
}

}  // extern "C"
