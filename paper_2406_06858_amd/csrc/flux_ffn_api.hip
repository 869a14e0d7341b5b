// The gated feed-forward block and the products of 4-bit matrices: checks of arguments, kernels, dispatch.
#include "flux_ffn_internal.h"
#include "flux_ffn_act.h"

namespace flux_ffn {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

static thread_local int g_last_hip_error = 0;
int hip_failed(hipError_t e) {
  g_last_hip_error = (int)e;
  return FLUX_ERR_HIP;
}

// ---- kernels -------------------------------------------------------------------------------------------------
// An operand of a product as a matrix of `rows` rows by k: element (r, k) of segment s at ptr[s][r * step_r + k * step_k], zero
// outside rows x K.
struct Operand {
  const __bf16* ptr[2];
  long long step_r, step_k;
  int rows, K;
  const uint8_t* scales[2];             // not null: ptr holds 4-bit blocks, rows of row_bytes and scale_row_bytes
  long long row_bytes, scale_row_bytes;
};

__device__ __forceinline__ __bf16 element(const Operand& o, int seg, int r, int k) {
  if (r >= o.rows || k >= o.K) return (__bf16)0.f;
  if (o.scales[0] == nullptr) return o.ptr[seg][r * o.step_r + k * o.step_k];
  const uint32_t byte = reinterpret_cast<const uint8_t*>(o.ptr[seg])[r * o.row_bytes + k / 2];
  const uint32_t code = k & 1 ? byte >> 4 : byte & 15u, m = code & 7u, e = o.scales[seg][r * o.scale_row_bytes + k / 32];
  const float a = m < 2u ? 0.5f * (float)m : __uint_as_float((126u << 23) + (m << 22));
  const float scale = e == 255u ? __uint_as_float(0x7fc00000u) : e ? __uint_as_float(e << 23) : 0x1p-127f;
  return (__bf16)((code & 8u ? -a : a) * scale);
}

struct Job {
  Operand a, b;             // the result's rows and its columns
  int32_t segs;             // segments of the contraction, or (gated) of b alone
  int32_t gated;
  int32_t act, out_f32, accumulate;
  void* out;
  __bf16 *g, *u;
  long long ld;
};

__device__ __forceinline__ float act_of(int which, float g) {
  return which == FLUX_ACT_SILU ? act<FLUX_ACT_SILU>(g) : which == FLUX_ACT_GELU ? act<FLUX_ACT_GELU>(g) : act<FLUX_ACT_GELU_TANH>(g);
}

// 64x64 of the result per workgroup, four waves of 32x32, slabs of 32 of k through LDS.
__global__ void __launch_bounds__(256) simple_kernel(const Job j) {
  __shared__ __bf16 la[64][40], lb[2][64][40];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / 2, wn = wave % 2;
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  f32x4 acc[2][2][2] = {};
  for (int seg = 0; seg < (j.gated ? 1 : j.segs); ++seg)
    for (int k0 = 0; k0 < j.a.K; k0 += 32) {
      for (int i = tid; i < 64 * 32; i += 256) {
        const bool along_k = j.a.step_k == 1, b_along_k = j.b.step_k == 1;
        const int ra = along_k ? i / 32 : i % 64, ka = along_k ? i % 32 : i / 64;
        const int rb = b_along_k ? i / 32 : i % 64, kb = b_along_k ? i % 32 : i / 64;
        la[ra][ka] = element(j.a, seg, m0 + ra, k0 + ka);
        lb[0][rb][kb] = element(j.b, seg, n0 + rb, k0 + kb);
        if (j.gated) lb[1][rb][kb] = element(j.b, 1, n0 + rb, k0 + kb);
      }
      __syncthreads();
      for (int h = 0; h < (j.gated ? 2 : 1); ++h)
        for (int mi = 0; mi < 2; ++mi)
          for (int ni = 0; ni < 2; ++ni) {
            bf16x8 x, y;
            for (int e = 0; e < 8; ++e) {
              x[e] = la[wm * 32 + mi * 16 + (lane & 15)][(lane >> 4) * 8 + e];
              y[e] = lb[h][wn * 32 + ni * 16 + (lane & 15)][(lane >> 4) * 8 + e];
            }
            acc[h][mi][ni] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, acc[h][mi][ni], 0, 0, 0);
          }
      __syncthreads();
    }
  for (int mi = 0; mi < 2; ++mi)
    for (int ni = 0; ni < 2; ++ni)
      for (int e = 0; e < 4; ++e) {
        const int m = m0 + wm * 32 + mi * 16 + 4 * (lane >> 4) + e, n = n0 + wn * 32 + ni * 16 + (lane & 15);
        if (m >= j.a.rows || n >= j.b.rows) continue;
        float v = acc[0][mi][ni][e];
        if (j.gated) {
          const float u = acc[1][mi][ni][e];
          if (j.g) { j.g[m * j.ld + n] = (__bf16)v; j.u[m * j.ld + n] = (__bf16)u; }
          v = act_of(j.act, v) * u;
        }
        if (j.out_f32) {
          float* p = static_cast<float*>(j.out) + m * j.ld + n;
          *p = j.accumulate ? *p + v : v;
        } else {
          __bf16* p = static_cast<__bf16*>(j.out) + m * j.ld + n;
          *p = (__bf16)(j.accumulate ? (float)*p + v : v);
        }
      }
}

// dG = dH U act'(G), dU = dH act(G), rounded to bf16 once: the operands of the three products.
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
constexpr size_t WS_HEADER = 0;
constexpr long long LIMIT = 1ll << 31;

static long long pitch_x(const flux_glu_t* p) { return p->ldx ? p->ldx : p->K; }
static long long pitch_w(const flux_glu_t* p) { return p->ldw ? p->ldw : p->w_is_nk ? p->K : p->N; }
static long long pitch_h(const flux_glu_t* p) { return p->ldh ? p->ldh : p->N; }

static bool pitch_ok(long long pitch, long long rows, long long cols) {
  return pitch >= cols && pitch % 8 == 0 && (rows - 1) * pitch + cols < LIMIT;
}
static bool dtype_ok(int d) { return d == FLUX_BF16 || d == FLUX_F32; }
static bool act_ok(int a) { return a >= FLUX_ACT_SILU && a <= FLUX_ACT_GELU_TANH; }

static int validate(int op, const flux_glu_t* p) {
  if (p == nullptr || (op != FLUX_GLU_FORWARD && op != FLUX_GLU_BACKWARD)) return FLUX_ERR_INVALID_ARG;
  if (!act_ok(p->act) || !dtype_ok(p->out_dtype) || !dtype_ok(p->dw_dtype)) return FLUX_ERR_INVALID_ARG;
  if ((p->w_is_nk | 1) != 1 || (p->dw_accumulate | 1) != 1 || p->reserved != 0) return FLUX_ERR_INVALID_ARG;
  if (p->ldx < 0 || p->ldw < 0 || p->ldh < 0) return FLUX_ERR_INVALID_ARG;
  if (p->M < 1 || p->N < 1 || p->K < 1 || p->N % 8 != 0 || p->K % 8 != 0) return FLUX_ERR_SHAPE;
  const long long w_rows = p->w_is_nk ? p->N : p->K, w_cols = p->w_is_nk ? p->K : p->N;
  if (!pitch_ok(pitch_x(p), p->M, p->K) || !pitch_ok(pitch_w(p), w_rows, w_cols) || !pitch_ok(pitch_h(p), p->M, p->N)) return FLUX_ERR_SHAPE;
  return FLUX_OK;
}

static int validate(int op, const flux_mx4_t* p) {
  if (p == nullptr || (op != FLUX_MX4_GEMM && op != FLUX_MX4_GLU)) return FLUX_ERR_INVALID_ARG;
  if (!dtype_ok(p->out_dtype) || (op == FLUX_MX4_GLU && !act_ok(p->act)) || p->reserved != 0 || p->ldc < 0) return FLUX_ERR_INVALID_ARG;
  if (p->M < 1 || p->N < 1 || p->K < 1 || p->N % 8 != 0) return FLUX_ERR_SHAPE;
  if (p->M * row_bytes(p->K) >= LIMIT || p->N * row_bytes(p->K) >= LIMIT) return FLUX_ERR_SHAPE;
  if (!pitch_ok(p->ldc ? p->ldc : p->N, p->M, p->N)) return FLUX_ERR_SHAPE;
  return FLUX_OK;
}

static size_t glu_need(int op, const flux_glu_t* p) {
  return op == FLUX_GLU_BACKWARD ? WS_HEADER + 4ull * p->M * p->N : 0;
}

static int workspace_ok(size_t need, const void* ws, size_t bytes) {
  if (need == 0) return FLUX_OK;
  return ws != nullptr && aligned(ws, 16) && bytes >= need ? FLUX_OK : FLUX_ERR_WORKSPACE;
}

// ---- dispatch ------------------------------------------------------------------------------------------------
static int launch(const Job& j, hipStream_t s) {
  hipLaunchKernelGGL(simple_kernel, dim3((j.b.rows + 63) / 64, (j.a.rows + 63) / 64), dim3(256), 0, s, j);
  FFN_HIP(hipGetLastError());
  return FLUX_OK;
}

static Operand plain(const void* p0, const void* p1, long long step_r, long long step_k, int rows, int K) {
  return Operand{{static_cast<const __bf16*>(p0), static_cast<const __bf16*>(p1)}, step_r, step_k, rows, K, {nullptr, nullptr}, 0, 0};
}
static Operand blocks(const void* q0, const void* s0, const void* q1, const void* s1, int rows, int K) {
  return Operand{{static_cast<const __bf16*>(q0), static_cast<const __bf16*>(q1)}, 0, 1, rows, K,
                 {static_cast<const uint8_t*>(s0), static_cast<const uint8_t*>(s1)}, row_bytes(K), scale_row_bytes(K)};
}

static int mx4(int op, const flux_mx4_t* p, const void* Aq, const void* As, const void* B0, const void* S0, const void* B1, const void* S1,
               void* out, void* ws, size_t bytes, void* stream) {
  int st = validate(op, p);
  if (st != FLUX_OK) return st;
  for (const void* x : {Aq, As, B0, S0, B1, S1, static_cast<const void*>(out)})
    if (x == nullptr || !aligned(x, 16)) return FLUX_ERR_INVALID_ARG;
  st = workspace_ok(flux_mx4_workspace_bytes(op, p), ws, bytes);
  if (st != FLUX_OK) return st;
  Job j = {};
  j.a = blocks(Aq, As, Aq, As, p->M, p->K);
  j.b = blocks(B0, S0, B1, S1, p->N, p->K);
  j.segs = 1;
  j.gated = op == FLUX_MX4_GLU;
  j.act = p->act;
  j.out_f32 = p->out_dtype == FLUX_F32;
  j.out = out;
  j.ld = p->ldc ? p->ldc : p->N;
  return launch(j, static_cast<hipStream_t>(stream));
}

}  // namespace flux_ffn

using namespace flux_ffn;

extern "C" {

int flux_ffn_last_hip_error(void) { return g_last_hip_error; }

size_t flux_glu_workspace_bytes(int op, const flux_glu_t* p) { return validate(op, p) == FLUX_OK ? glu_need(op, p) : 0; }

size_t flux_mx4_workspace_bytes(int op, const flux_mx4_t* p) {
  (void)op; (void)p;
  return 0;
}

int flux_ffn_init(void* workspace, size_t workspace_bytes, void* stream) {
  if (workspace == nullptr && workspace_bytes != 0) return FLUX_ERR_INVALID_ARG;
  (void)stream;
  return FLUX_OK;
}

int flux_glu(const flux_glu_t* p, const void* X, const void* Wg, const void* Wu, void* H, void* G, void* U, void* workspace,
             size_t workspace_bytes, void* stream) {
  int st = validate(FLUX_GLU_FORWARD, p);
  if (st != FLUX_OK) return st;
  for (const void* x : {X, Wg, Wu, static_cast<const void*>(H)})
    if (x == nullptr || !aligned(x, 16)) return FLUX_ERR_INVALID_ARG;
  if ((G == nullptr) != (U == nullptr) || !aligned(G, 16) || !aligned(U, 16)) return FLUX_ERR_INVALID_ARG;
  st = workspace_ok(glu_need(FLUX_GLU_FORWARD, p), workspace, workspace_bytes);
  if (st != FLUX_OK) return st;
  Job j = {};
  j.a = plain(X, X, pitch_x(p), 1, p->M, p->K);
  j.b = p->w_is_nk ? plain(Wg, Wu, pitch_w(p), 1, p->N, p->K) : plain(Wg, Wu, 1, pitch_w(p), p->N, p->K);
  j.segs = 1;
  j.gated = 1;
  j.act = p->act;
  j.out_f32 = p->out_dtype == FLUX_F32;
  j.out = H;
  j.g = static_cast<__bf16*>(G);
  j.u = static_cast<__bf16*>(U);
  j.ld = pitch_h(p);
  return launch(j, static_cast<hipStream_t>(stream));
}

int flux_glu_backward(const flux_glu_t* p, const void* X, const void* Wg, const void* Wu, const void* G, const void* U,
                      const void* dH, void* dX, void* dWg, void* dWu, void* workspace, size_t workspace_bytes, void* stream) {
  int st = validate(FLUX_GLU_BACKWARD, p);
  if (st != FLUX_OK) return st;
  for (const void* x : {X, Wg, Wu, G, U, dH})
    if (x == nullptr || !aligned(x, 16)) return FLUX_ERR_INVALID_ARG;
  if ((dWg == nullptr) != (dWu == nullptr) || !aligned(dX, 16) || !aligned(dWg, 16) || !aligned(dWu, 16)) return FLUX_ERR_INVALID_ARG;
  st = workspace_ok(glu_need(FLUX_GLU_BACKWARD, p), workspace, workspace_bytes);
  if (st != FLUX_OK) return st;
  if (dX == nullptr && dWg == nullptr) return FLUX_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  SlopeArgs d = {};
  d.G = static_cast<const __bf16*>(G);
  d.U = static_cast<const __bf16*>(U);
  d.dH = static_cast<const __bf16*>(dH);
  d.dG = reinterpret_cast<__bf16*>(static_cast<char*>(workspace) + WS_HEADER);
  d.dU = d.dG + (long long)p->M * p->N;
  d.ldh = pitch_h(p);
  d.ldd = p->N;
  d.M = p->M;
  d.N = p->N;
  const dim3 grid((unsigned)(((long long)p->M * p->N / 8 + 255) / 256));
  if (p->act == FLUX_ACT_SILU) hipLaunchKernelGGL(slope_kernel<FLUX_ACT_SILU>, grid, dim3(256), 0, s, d);
  else if (p->act == FLUX_ACT_GELU) hipLaunchKernelGGL(slope_kernel<FLUX_ACT_GELU>, grid, dim3(256), 0, s, d);
  else hipLaunchKernelGGL(slope_kernel<FLUX_ACT_GELU_TANH>, grid, dim3(256), 0, s, d);
  FFN_HIP(hipGetLastError());
  const long long lw = pitch_w(p), lx = pitch_x(p), n = p->N;
  if (dX != nullptr) {
    Job j = {};
    j.a = plain(d.dG, d.dU, n, 1, p->M, p->N);
    j.b = p->w_is_nk ? plain(Wg, Wu, 1, lw, p->K, p->N) : plain(Wg, Wu, lw, 1, p->K, p->N);
    j.segs = 2;
    j.out_f32 = p->out_dtype == FLUX_F32;
    j.out = dX;
    j.ld = lx;
    st = launch(j, s);
    if (st != FLUX_OK) return st;
  }
  for (int h = 0; h < 2 && dWg != nullptr; ++h) {
    const Operand x = plain(X, X, 1, lx, p->K, p->M), y = plain(h ? d.dU : d.dG, d.dG, 1, n, p->N, p->M);
    Job j = {};
    j.a = p->w_is_nk ? y : x;
    j.b = p->w_is_nk ? x : y;
    j.segs = 1;
    j.out_f32 = p->dw_dtype == FLUX_F32;
    j.accumulate = p->dw_accumulate;
    j.out = h ? dWu : dWg;
    j.ld = lw;
    st = launch(j, s);
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
