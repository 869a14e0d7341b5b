// The gated feed-forward block and the products of 4-bit matrices: checks of arguments, kernels, dispatch.
#include <algorithm>
#include "flux_ffn_internal.h"
#include "flux_ffn_act.h"

namespace flux_ffn {

static thread_local int g_last_hip_error = 0;
int hip_failed(hipError_t e) {
  g_last_hip_error = (int)e;
  (void)hipGetLastError();              // (reported here, not again by the caller's next call)
  return FLUX_ERR_HIP;
}

// ---- kernels -------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) zero_kernel(uint4* p, long long n) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) p[i] = make_uint4(0u, 0u, 0u, 0u);
}

// dG = dH U act'(G), dU = dH act(G), taken in 32 bits and rounded to bf16 once, since they are operands of the three products: a second
// MFMA for what the rounding leaves would double the products' work.  It costs the gradients, of either type, 2.3e-3 of their norm
// against 64 bits, where dG and dU in 32 bits and a gradient in bf16 have 1.7e-3.  Memory-bound: 8192x3584 46 us (three reads and two
// writes, 6.3 TB/s), 1496x3400 15.6 us.
struct SlopeArgs {
  const __bf16 *G, *U, *dH;
  __bf16 *dG, *dU;
  long long ldh, ldd;
  int32_t M, N;
};
template <int ACT>
__global__ void __launch_bounds__(256) slope_kernel(const SlopeArgs s) {
  const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 8;
  const int row = (int)(i / s.N), col = (int)(i % s.N);            // (N % 8 == 0)
  if (row >= s.M) return;
  const long long in = row * s.ldh + col, out = row * s.ldd + col;
  const bf16x8 g = *reinterpret_cast<const bf16x8*>(s.G + in), u = *reinterpret_cast<const bf16x8*>(s.U + in);
  const bf16x8 d = *reinterpret_cast<const bf16x8*>(s.dH + in);
  bf16x8 dg, du;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float a, slope;
    act_and_slope<ACT>((float)g[e], a, slope);
    dg[e] = (__bf16)((float)d[e] * (float)u[e] * slope);
    du[e] = (__bf16)((float)d[e] * a);
  }
  *reinterpret_cast<bf16x8*>(s.dG + out) = dg;
  *reinterpret_cast<bf16x8*>(s.dU + out) = du;
}

// ---- checks --------------------------------------------------------------------------------------------------
static long long pitch_x(const flux_glu_t* p) { return p->ldx ? p->ldx : p->K; }
static long long pitch_w(const flux_glu_t* p) { return p->ldw ? p->ldw : p->w_is_nk ? p->K : p->N; }
static long long pitch_h(const flux_glu_t* p) { return p->ldh ? p->ldh : p->N; }

static bool pitch_ok(long long pitch, long long rows, long long cols) {
  return pitch >= cols && pitch % 8 == 0 && below_limit(rows, pitch, cols);
}
static bool dtype_ok(int d) { return d == FLUX_BF16 || d == FLUX_F32; }
static bool act_ok(int a) { return a >= FLUX_ACT_SILU && a <= FLUX_ACT_GELU_TANH; }

constexpr int FEW_CONFIG = N_SHAPES + 1;        // id of the kernel for few rows
static bool choice_ok(int config, int parts) { return config >= 0 && config <= FEW_CONFIG && parts >= 0 && parts <= 64; }
// (a workgroup of 256 threads has at least 16 columns, and 2^32 threads are too many for a launch)
static bool few_fits(int kind, int rows, int cols) {
  return rows <= FEW_ROWS && cols <= (1 << 28) - 16 && (kind == GLU_NK || kind == MX_GEMM || kind == MX_GLU);
}

static int validate(int op, const flux_glu_t* p) {
  if (p == nullptr || (op != FLUX_GLU_FORWARD && op != FLUX_GLU_BACKWARD)) return FLUX_ERR_INVALID_ARG;
  if (!act_ok(p->act) || !dtype_ok(p->out_dtype) || !dtype_ok(p->dw_dtype)) return FLUX_ERR_INVALID_ARG;
  if ((p->w_is_nk | 1) != 1 || (p->dw_accumulate | 1) != 1 || !choice_ok(p->tile_config, p->split_k)) return FLUX_ERR_INVALID_ARG;
  if (p->ldx < 0 || p->ldw < 0 || p->ldh < 0) return FLUX_ERR_INVALID_ARG;
  if (p->M < 1 || p->N < 1 || p->K < 1 || p->N % 8 != 0 || p->K % 8 != 0) return FLUX_ERR_SHAPE;
  const long long w_rows = p->w_is_nk ? p->N : p->K, w_cols = p->w_is_nk ? p->K : p->N;
  if (!pitch_ok(pitch_x(p), p->M, p->K) || !pitch_ok(pitch_w(p), w_rows, w_cols) || !pitch_ok(pitch_h(p), p->M, p->N)) return FLUX_ERR_SHAPE;
  if (p->tile_config == FEW_CONFIG && (op != FLUX_GLU_FORWARD || !few_fits(p->w_is_nk ? GLU_NK : GLU_KN, p->M, p->N))) return FLUX_ERR_UNSUPPORTED;
  return FLUX_OK;
}

static int validate(int op, const flux_mx4_t* p) {
  if (p == nullptr || (op != FLUX_MX4_GEMM && op != FLUX_MX4_GLU)) return FLUX_ERR_INVALID_ARG;
  if (!dtype_ok(p->out_dtype) || (op == FLUX_MX4_GLU && !act_ok(p->act)) || p->reserved != 0 || p->ldc < 0) return FLUX_ERR_INVALID_ARG;
  if (!choice_ok(p->tile_config, p->split_k)) return FLUX_ERR_INVALID_ARG;
  if (p->M < 1 || p->N < 1 || p->K < 1 || p->N % 8 != 0) return FLUX_ERR_SHAPE;
  if (p->M * row_bytes(p->K) >= LIMIT || p->N * row_bytes(p->K) >= LIMIT) return FLUX_ERR_SHAPE;
  if (!pitch_ok(p->ldc ? p->ldc : p->N, p->M, p->N)) return FLUX_ERR_SHAPE;
  if (p->tile_config == FEW_CONFIG && !few_fits(MX_GEMM, p->M, p->N)) return FLUX_ERR_UNSUPPORTED;
  return FLUX_OK;
}

// ---- how a product is run --------------------------------------------------------------------------------------
struct Plan {
  int shape = 0, full = 0, cut = 0, parts = 1, part_slabs = 0, slabs = 0, tiles_m = 0, tiles_n = 0;
  bool edge = false, few = false;
  size_t partial_bytes = 0;
};

static int halves_of(int kind) { return kind == GLU_NK || kind == GLU_KN || kind == MX_GLU ? 2 : 1; }
static int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

// Estimated us of a product: whole rounds of workgroups, a last one that is not full, the cut tiles.
static double tile_us(const Shape& sh, const Pace& p, int full, int cut, int parts, int slabs, int part_slabs) {
  const int at_once = 256 * sh.per_unit, last = full % at_once;
  const auto pace = [&](int n) { return p.alone_us + (p.slab_us - p.alone_us) * std::min(1.0, (double)n / at_once); };
  double us = full / at_once * (slabs * p.slab_us + p.ends_us);
  if (last != 0) us += slabs * pace(last) + p.ends_us;
  return cut == 0 ? us : us + part_slabs * pace(cut * parts) + p.ends_us + p.join_us + p.join_all_us * cut * parts / at_once;
}

// depth: pieces of two bytes of (a segment of) the contraction; config, want_parts: the caller's choice, 0 for the library's.
static Plan plan_tiles(int kind, int rows, int cols, int depth, int config, int want_parts) {
  const int halves = halves_of(kind), segs = kind == DX_NK || kind == DX_KN ? 2 : 1, jobs = kind == DW ? 2 : 1;
  const int slabs = segs * ceil_div(depth, 64);
  Plan best;
  // Few rows: the kernel that reads weights once and cuts nothing (so "no cut" leaves it as it is), unless cut tiles are well ahead: few
  // columns over a long contraction give it few workgroups, and above 16 rows all of them read the rows.  The tiles' estimate knows nothing of
  // memory: it is no less than 3 us and the weights at 5.2 TB/s.  us, few / tiles (bf16, then 4 bits, gated): 1x256x12288 18.9 / 12.4, 7.5 / 9.3;
  // 64x256x12288 41.3 / 14.6, 13.7 / 10.0; 64x1024x8192 26.5 / 13.4, 10.0 / 11.5; 1x3584x8192 21.7 / 27.4, 8.1 / 12.1; 64x3584x8192 32.0 / 28.7,
  // 11.8 / 13.9; 64x8192x512 10.2 / 7.3, 7.8 / 5.0.  Over 597 products that the estimates were not fitted to the pick takes 1.7 % (bf16) and 0.8 %
  // (4 bits) longer in the mean than the faster one; always few would take 22 and 8 %, up to 4.7 times.  (1.3: with less, more products go to
  // tiles that take longer there.)
  double few = 0;
  best.few = config == FEW_CONFIG;
  if (config == 0 && want_parts <= 1 && few_fits(kind, rows, cols)) {
    few = few_us(kind, rows, cols, depth / 8);
    best.few = few <= 1.3 * (3.0 + 2.0 * halves * cols * depth / 5.2e6);
  }
  if (best.few) return best;
  double best_us = 0;
  for (int i = config ? config - 1 : 0; i < (config ? config : N_SHAPES); ++i) {
    const Shape& sh = SHAPES[i];
    const int sub = sh.bn / halves, tm = ceil_div(rows, sh.bm), tn = ceil_div(cols, sub);
    const int at_once = 256 * sh.per_unit, tiles = tm * tn * jobs;          // (results below 2^31 elements, no side over 2^28: below 2^25)
    // Whole rounds of tiles are a workgroup each; what is left over may be cut along the contraction, over no more workgroups than
    // run at once, since its parts wait for each other.
    const int rest = tiles % at_once;
    Plan pl;
    double pl_us = 0;
    for (int parts = 1; parts <= (want_parts ? want_parts : MAX_PARTS); ++parts) {
      int each = ceil_div(slabs, parts);
      if (kind >= MX_GEMM) each += each % 2;                    // (scales come for two slabs)
      if (parts > 1) {
        if (rest == 0 || parts > MAX_PARTS || (long long)rest * parts > at_once || each < (want_parts ? 1 : 4)) break;
        if ((long long)each * (parts - 1) >= slabs) continue;          // (a part would be left without slabs)
      }
      const int cut = parts > 1 ? rest : 0;
      const double us = tile_us(sh, sh.pace[kind >= MX_GEMM], tiles - cut, cut, parts, slabs, each);
      if (pl.slabs != 0 && !want_parts && us >= pl_us) continue;          // (asked for: the most that fit)
      pl_us = us;
      pl.shape = i;
      pl.full = tiles - cut;
      pl.cut = cut;
      pl.parts = parts;
      pl.part_slabs = each;
      pl.slabs = slabs;
      pl.tiles_m = tm;
      pl.tiles_n = tn;
      pl.edge = rows % sh.bm != 0 || cols % sub != 0 || depth % 64 != 0;
      pl.partial_bytes = (size_t)cut * parts * sh.bm * sh.bn * 4;
    }
    if (best.slabs != 0 && pl_us >= best_us) continue;
    best = pl;
    best_us = pl_us;
  }
  if (few > 0 && few <= 1.3 * best_us) {
    best = Plan();
    best.few = true;
  }
  return best;
}

static Plan plan_glu(const flux_glu_t* p) { return plan_tiles(p->w_is_nk ? GLU_NK : GLU_KN, p->M, p->N, p->K, p->tile_config, p->split_k); }
static Plan plan_dx(const flux_glu_t* p) { return plan_tiles(p->w_is_nk ? DX_KN : DX_NK, p->M, p->K, p->N, p->tile_config, p->split_k); }
static Plan plan_dw(const flux_glu_t* p) { return plan_tiles(DW, p->w_is_nk ? p->N : p->K, p->w_is_nk ? p->K : p->N, p->M, p->tile_config, p->split_k); }
static Plan plan_mx4(int op, const flux_mx4_t* p) {
  return plan_tiles(op == FLUX_MX4_GLU ? MX_GLU : MX_GEMM, p->M, p->N, (int)(row_bytes(p->K) / 2), p->tile_config, p->split_k);
}

// Rows of dG and of dU in the workspace are whole lines of 128 bytes: loads of a slab, 128 bytes a row, are one line each then.
static long long pitch_d(const flux_glu_t* p) {
  const long long whole = (p->N + 63ll) / 64 * 64;
  return p->M * whole < LIMIT ? whole : p->N;          // (offsets are 32 bits)
}
static size_t slope_bytes(const flux_glu_t* p) { return 4ull * p->M * pitch_d(p); }

// The workspace: a word a cut tile, zero between calls; then dG and dU (backward); then the cut tiles' sums.
constexpr size_t WS_HEADER = 512 * COUNTER_STRIDE * 4;
static size_t after_slopes(const flux_glu_t* p) { return WS_HEADER + (slope_bytes(p) + 255) / 256 * 256; }
static size_t need_of(const Plan& pl) { return pl.cut ? WS_HEADER + pl.partial_bytes : 0; }

static size_t need_of(const flux_glu_t* p, const Plan& dx, const Plan& dw) { return after_slopes(p) + std::max(dx.partial_bytes, dw.partial_bytes); }

static int workspace_ok(size_t need, const void* ws, size_t bytes) {
  if (need == 0) return FLUX_OK;
  return ws != nullptr && aligned(ws, 16) && bytes >= need ? FLUX_OK : FLUX_ERR_WORKSPACE;
}

// ---- dispatch ------------------------------------------------------------------------------------------------
static uint32_t extent(long long rows, long long pitch, long long row) { return (uint32_t)((rows - 1) * pitch + row); }

static int launch(int kind, const Plan& pl, TileArgs& t, void* ws, size_t partial_at, hipStream_t s) {
  typedef hipError_t (*Launcher)(int, const TileArgs&, bool, int, hipStream_t);
  static constexpr Launcher launchers[KINDS] = {launch_tile0, launch_tile1, launch_tile2, launch_tile3, launch_tile4, launch_tile5, launch_tile6};
  if (pl.few) {
    FewArgs f = {t.a[0], {t.b[0], t.b[1]}, t.sa, {t.sb[0], t.sb[1]}, t.pitch_a, t.pitch_b, t.bytes_a, t.bytes_b, t.pitch_s, t.rows, t.cols,
                 t.depth / 8, t.act, t.out_f32, t.ld, t.out[0], t.g, t.u};
    FFN_HIP(launch_few(kind, f, s));
    return FLUX_OK;
  }
  t.slabs = pl.slabs;
  t.seg_slabs = (t.depth + 63) / 64;
  t.full_tiles = pl.full;
  t.cut_tiles = pl.cut;
  t.parts = pl.parts;
  t.part_slabs = pl.part_slabs;
  t.tiles_m = pl.tiles_m;
  t.tiles_n = pl.tiles_n;
  t.band = pl.tiles_m < 8 ? pl.tiles_m : 8;
  // Results may go past the caches, which then keep the operands' panels.  Where the rows of H, C or the gradients are no whole lines they
  // may not, nor where the contraction of a plain product is short: it has more results than panels.  us, past the caches / kept there: 4-bit
  // 8192x12288x6144 281 / 303, 8192x8192x512 55 / 44, gated 8192x4096x1024 62 / 68; gradients of 8192x3584x8192 1318 / 1342, of
  // 1496x3400x5112 261 / 250.  G and U go the way of H, also where beside an fp32 H their own rows end in half a line (4096x3616x512 59 / 70,
  // 4096x3616x2048 127 / 145, 256x128 tiles), and so do the halves of lines that the waves of gated 128-column tiles store in bf16 (with G
  // and U 2048x8192x1024 77 / 85, 4096x3584x2048 120 / 134; H alone 73 / 75, 112 / 113).
  const int size = t.out_f32 ? 4 : 2;
  t.stream = t.ld * size % 128 == 0 && aligned(t.out[0], 128) && aligned(t.out[1], 128) && aligned(t.g, 128) && aligned(t.u, 128) &&
             (halves_of(kind) == 2 || t.slabs >= 20);
  t.counters = static_cast<uint32_t*>(ws);
  t.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + partial_at);
  FFN_HIP(launchers[kind](pl.shape, t, pl.edge, pl.full + pl.cut * pl.parts, s));
  return FLUX_OK;
}

static int mx4(int op, const flux_mx4_t* p, const void* Aq, const void* As, const void* B0, const void* S0, const void* B1, const void* S1,
               void* out, void* ws, size_t bytes, void* stream) {
  int st = validate(op, p);
  if (st != FLUX_OK) return st;
  for (const void* x : {Aq, As, B0, S0, B1, S1, static_cast<const void*>(out)})
    if (x == nullptr || !aligned(x, 16)) return FLUX_ERR_INVALID_ARG;
  const Plan pl = plan_mx4(op, p);
  st = workspace_ok(need_of(pl), ws, bytes);
  if (st != FLUX_OK) return st;
  TileArgs t = {};
  t.a[0] = Aq;
  t.b[0] = B0;
  t.b[1] = B1;
  t.sa = static_cast<const uint8_t*>(As);
  t.sb[0] = static_cast<const uint8_t*>(S0);
  t.sb[1] = static_cast<const uint8_t*>(S1);
  t.pitch_a = t.pitch_b = (uint32_t)row_bytes(p->K);
  t.pitch_s = (uint32_t)scale_row_bytes(p->K);
  t.bytes_a = (uint32_t)p->M * t.pitch_a;
  t.bytes_b = (uint32_t)p->N * t.pitch_b;
  t.rows = p->M;
  t.cols = p->N;
  t.depth = (int)(t.pitch_a / 2);
  t.act = p->act;
  t.out_f32 = p->out_dtype == FLUX_F32;
  t.ld = p->ldc ? p->ldc : p->N;
  t.out[0] = out;
  return launch(op == FLUX_MX4_GLU ? MX_GLU : MX_GEMM, pl, t, ws, WS_HEADER, static_cast<hipStream_t>(stream));
}

}  // namespace flux_ffn

using namespace flux_ffn;

extern "C" {

int flux_ffn_last_hip_error(void) { return g_last_hip_error; }

int flux_ffn_tile_config_count(void) { return FEW_CONFIG; }

int flux_ffn_tile_config_info(int32_t id, int32_t* tile_m, int32_t* tile_n) {
  if (id < 1 || id > FEW_CONFIG || tile_m == nullptr || tile_n == nullptr) return FLUX_ERR_INVALID_ARG;
  *tile_m = id == FEW_CONFIG ? 0 : SHAPES[id - 1].bm;
  *tile_n = id == FEW_CONFIG ? 0 : SHAPES[id - 1].bn;
  return FLUX_OK;
}

size_t flux_glu_workspace_bytes(int op, const flux_glu_t* p) {
  if (validate(op, p) != FLUX_OK) return 0;
  return op == FLUX_GLU_FORWARD ? need_of(plan_glu(p)) : need_of(p, plan_dx(p), plan_dw(p));
}

size_t flux_mx4_workspace_bytes(int op, const flux_mx4_t* p) { return validate(op, p) == FLUX_OK ? need_of(plan_mx4(op, p)) : 0; }

int flux_ffn_init(void* workspace, size_t workspace_bytes, void* stream) {
  if (workspace == nullptr && workspace_bytes != 0) return FLUX_ERR_INVALID_ARG;
  if (!aligned(workspace, 16)) return FLUX_ERR_WORKSPACE;
  const long long vecs = (long long)(std::min(workspace_bytes, WS_HEADER) / 16);           // (nothing else has to be zero)
  if (vecs == 0) return FLUX_OK;
  FFN_HIP(start(zero_kernel, dim3((unsigned)((vecs + 255) / 256)), static_cast<hipStream_t>(stream), static_cast<uint4*>(workspace), vecs));
  return FLUX_OK;
}

int flux_glu(const flux_glu_t* p, const void* X, const void* Wg, const void* Wu, void* H, void* G, void* U, void* workspace,
             size_t workspace_bytes, void* stream) {
  int st = validate(FLUX_GLU_FORWARD, p);
  if (st != FLUX_OK) return st;
  for (const void* x : {X, Wg, Wu, static_cast<const void*>(H)})
    if (x == nullptr || !aligned(x, 16)) return FLUX_ERR_INVALID_ARG;
  if ((G == nullptr) != (U == nullptr) || !aligned(G, 16) || !aligned(U, 16)) return FLUX_ERR_INVALID_ARG;
  const Plan pl = plan_glu(p);
  st = workspace_ok(need_of(pl), workspace, workspace_bytes);
  if (st != FLUX_OK) return st;
  TileArgs t = {};
  t.a[0] = X;
  t.b[0] = Wg;
  t.b[1] = Wu;
  const long long lx = pitch_x(p), lw = pitch_w(p);
  t.pitch_a = (uint32_t)(lx * 2);
  t.pitch_b = (uint32_t)(lw * 2);
  t.bytes_a = extent(p->M, lx * 2, p->K * 2ll);
  t.bytes_b = p->w_is_nk ? extent(p->N, lw * 2, p->K * 2ll) : extent(p->K, lw * 2, p->N * 2ll);
  t.rows = p->M;
  t.cols = p->N;
  t.depth = p->K;
  t.act = p->act;
  t.out_f32 = p->out_dtype == FLUX_F32;
  t.ld = pitch_h(p);
  t.out[0] = H;
  t.g = static_cast<__bf16*>(G);
  t.u = static_cast<__bf16*>(U);
  return launch(p->w_is_nk ? GLU_NK : GLU_KN, pl, t, workspace, WS_HEADER, static_cast<hipStream_t>(stream));
}

int flux_glu_backward(const flux_glu_t* p, const void* X, const void* Wg, const void* Wu, const void* G, const void* U,
                      const void* dH, void* dX, void* dWg, void* dWu, void* workspace, size_t workspace_bytes, void* stream) {
  int st = validate(FLUX_GLU_BACKWARD, p);
  if (st != FLUX_OK) return st;
  for (const void* x : {G, U, dH})
    if (x == nullptr) return FLUX_ERR_INVALID_ARG;
  if ((dX != nullptr && (Wg == nullptr || Wu == nullptr)) || (dWg != nullptr && X == nullptr)) return FLUX_ERR_INVALID_ARG;
  for (const void* x : {X, Wg, Wu, G, U, dH})
    if (!aligned(x, 16)) return FLUX_ERR_INVALID_ARG;
  if ((dWg == nullptr) != (dWu == nullptr) || !aligned(dX, 16) || !aligned(dWg, 16) || !aligned(dWu, 16)) return FLUX_ERR_INVALID_ARG;
  const Plan for_dx = plan_dx(p), for_dw = plan_dw(p);
  st = workspace_ok(need_of(p, for_dx, for_dw), workspace, workspace_bytes);
  if (st != FLUX_OK) return st;
  if (dX == nullptr && dWg == nullptr) return FLUX_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  SlopeArgs d = {};
  d.G = static_cast<const __bf16*>(G);
  d.U = static_cast<const __bf16*>(U);
  d.dH = static_cast<const __bf16*>(dH);
  d.dG = reinterpret_cast<__bf16*>(static_cast<char*>(workspace) + WS_HEADER);
  const long long ld = pitch_d(p);
  d.dU = d.dG + p->M * ld;
  d.ldh = pitch_h(p);
  d.ldd = ld;
  d.M = p->M;
  d.N = p->N;
  const dim3 grid((unsigned)(((long long)p->M * p->N / 8 + 255) / 256));
  FFN_HIP(start(p->act == FLUX_ACT_SILU ? slope_kernel<FLUX_ACT_SILU> : p->act == FLUX_ACT_GELU ? slope_kernel<FLUX_ACT_GELU> : slope_kernel<FLUX_ACT_GELU_TANH>, grid, s, d));
  const long long lw = pitch_w(p), lx = pitch_x(p);
  const uint32_t bytes_w = p->w_is_nk ? extent(p->N, lw * 2, p->K * 2ll) : extent(p->K, lw * 2, p->N * 2ll);
  const uint32_t bytes_d = extent(p->M, ld * 2, p->N * 2ll), bytes_x = extent(p->M, lx * 2, p->K * 2ll);
  if (dX != nullptr) {
    TileArgs t = {};
    t.a[0] = d.dG;
    t.a[1] = d.dU;
    t.b[0] = Wg;
    t.b[1] = Wu;
    t.pitch_a = (uint32_t)(ld * 2);
    t.pitch_b = (uint32_t)(lw * 2);
    t.bytes_a = bytes_d;
    t.bytes_b = bytes_w;
    t.rows = p->M;
    t.cols = p->K;
    t.depth = p->N;
    t.out_f32 = p->out_dtype == FLUX_F32;
    t.ld = lx;
    t.out[0] = dX;
    st = launch(p->w_is_nk ? DX_KN : DX_NK, for_dx, t, workspace, after_slopes(p), s);
    if (st != FLUX_OK) return st;
  }
  if (dWg != nullptr) {
    TileArgs t = {};
    const void* const dgu[2] = {d.dG, d.dU};
    for (int h = 0; h < 2; ++h) {
      t.a[h] = p->w_is_nk ? dgu[h] : X;
      t.b[h] = p->w_is_nk ? X : dgu[h];
    }
    const uint32_t pitch = (uint32_t)(ld * 2), pitch_of_x = (uint32_t)(lx * 2);
    t.pitch_a = p->w_is_nk ? pitch : pitch_of_x;
    t.pitch_b = p->w_is_nk ? pitch_of_x : pitch;
    t.bytes_a = p->w_is_nk ? bytes_d : bytes_x;
    t.bytes_b = p->w_is_nk ? bytes_x : bytes_d;
    t.rows = p->w_is_nk ? p->N : p->K;
    t.cols = p->w_is_nk ? p->K : p->N;
    t.depth = p->M;
    t.out_f32 = p->dw_dtype == FLUX_F32;
    t.accumulate = p->dw_accumulate;
    t.ld = lw;
    t.out[0] = dWg;
    t.out[1] = dWu;
    st = launch(DW, for_dw, t, workspace, after_slopes(p), s);
    if (st != FLUX_OK) return st;
  }
  return FLUX_OK;
}

int flux_mx4_gemm(const flux_mx4_t* p, const void* Aq, const void* As, const void* Bq, const void* Bs, void* C, void* workspace,
                  size_t workspace_bytes, void* stream) {
  return mx4(FLUX_MX4_GEMM, p, Aq, As, Bq, Bs, Bq, Bs, C, workspace, workspace_bytes, stream);
}

int flux_mx4_glu(const flux_mx4_t* p, const void* Xq, const void* Xs, const void* Wgq, const void* Wgs, const void* Wuq, const void* Wus,
                 void* H, void* workspace, size_t workspace_bytes, void* stream) {
  return mx4(FLUX_MX4_GLU, p, Xq, Xs, Wgq, Wgs, Wuq, Wus, H, workspace, workspace_bytes, stream);
}

}  // extern "C"
