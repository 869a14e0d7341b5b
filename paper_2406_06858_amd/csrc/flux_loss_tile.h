// What becomes of a tile of logits Z = X W^T, which nobody keeps (gfx950): out of the accumulators of the tile kernel's main loop either
//
//   statistics   of every row and each wave's run of columns the largest logit m and the sum of exp(Z - m), and the target's logit; or
//   dZ           dloss / D (exp(Z - lse) - [v = target]) in bf16, operand of the two products of the backward pass, whose results take the factor D.
#pragma once
#include "flux_ffn_tile.h"

namespace flux_ffn {

struct LossArgs {
  const void* target;            // [rows], 32 or 64 bits
  int32_t target_i64, dloss_one;
  long long v0, vocab;           // number of the product's first column; columns of the whole vocabulary
  // statistics
  float2* stats;                 // [runs of columns][rows]: m, sum
  float* logit;                  // written where the target is a column here
  // dZ
  const float *lse, *dloss;
  float* most;                   // D: the largest |dloss| (dloss_one: dloss itself)
  int32_t finds_most;            // every workgroup has all rows: it finds D itself, and the first leaves it there
  __bf16* dz;                    // pitch TileArgs::ld
};

// What a row's dZ is multiplied by: dloss / D.  Where every row that counts has the same dloss, as in a mean, that is 1, and the target's number, which
// outweighs the others, is p - 1: all but free of rounding to bf16 where p is small.  With dloss in dZ it is -dloss in every row, rounded the same way in
// every row: up to 2^-8 of the gradients.  Error of dX and dW in bf16 of a mean, 37x13183x6144 and the like against 64 bits, in parts of their norm: 1.7e-3, as the
// rounding of the results alone gives; with dloss in dZ up to 4e-3.  (In fp32 2e-4 to 8e-4; with a dloss of its own in every row 2.3e-3, in fp32 1.7e-3.)
__device__ __forceinline__ float row_dloss(const LossArgs& l, int row, bool counts) { return counts ? l.dloss[l.dloss_one ? 0 : row] : 0.f; }
__device__ __forceinline__ float row_factor(const LossArgs& l, float dloss, float most) {
  return l.dloss_one ? (dloss == 0.f ? 0.f : 1.f) : dloss / most;
}
__device__ __forceinline__ float sane_most(float m) { return m > 0.f && m < __builtin_inff() ? m : 1.f; }          // (0 and no number: no factor)
__device__ __forceinline__ float wave_max(float m) {
#pragma unroll
  for (int n = 1; n < 64; n *= 2) m = fmaxf(m, __shfl_xor(m, n));
  return m;
}

// exp(x), within |x| 2^-24 of itself: what that is off by matters for logits that count for nothing.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(LOG2E * x); }

// The row's target as a column of this product, -1 where it is none; counts: whether the row counts at all.
__device__ __forceinline__ int column_of(const LossArgs& l, long long target, int cols, bool& counts) {
  counts = target >= 0 && target < l.vocab;
  const long long c = target - l.v0;
  return counts && c >= 0 && c < cols ? (int)c : -1;
}
__device__ __forceinline__ int target_column(const LossArgs& l, int row, int cols, bool& counts) {
  return column_of(l, l.target_i64 ? static_cast<const long long*>(l.target)[row] : static_cast<const int32_t*>(l.target)[row], cols, counts);
}

// (m, s) and (m2, s2) of two sets of logits as of one.  An infinite m leaves exp its argument as it is: no infinity is taken from another.
__device__ __forceinline__ void join_stats(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2), at = __builtin_fabsf(top) == __builtin_inff() ? 0.f : top;
  s = s * exp_of(m - at) + s2 * exp_of(m2 - at);
  m = top;
}

// The largest of three.  (Of what the compiler does not know to be no signalling NaN it would make a quiet one first, an instruction a number.)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float m;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
  return m;
}

// 16 rows of a wave's part of the tile: a lane holds columns 16 n + 4 (lane / 16) .. + 3 of row lane % 16.
//
// A logit costs half a max, a difference, a product, an exp2 (four slots) and an addition; where the contraction is short these are what takes the time.
// (Not 2^(Z log2 e - m log2 e) with one rounding: of logits of 10^9 the product m log2 e alone is off by a factor e^50.)  Which lane has the target's
// logit is only asked where a row of the wave has its target among these columns.  Of 7490x44009x64 us, with a comparison a logit for
// the target and for the edge, and maxima made quiet / so: 235 / 198 (with the rows' targets asked for ahead, see Logits).
template <class C, bool ALL>
__device__ __forceinline__ void stats_of(const f32x4 (&acc)[C::NI], int left, int g, float& m, float& s) {
  const auto in = [&](int n, int e) { return ALL || n * 16 + 4 * g + e < left; };
  const float none = -__builtin_inff();
  m = none;
#pragma unroll
  for (int n = 0; n < C::NI; ++n)
#pragma unroll
    for (int e = 0; e < 4; e += 2) m = max3(m, in(n, e) ? acc[n][e] : none, in(n, e + 1) ? acc[n][e + 1] : none);
  m = fmaxf(m, __shfl_xor(m, 16));
  m = fmaxf(m, __shfl_xor(m, 32));
  const float at = __builtin_fabsf(m) == __builtin_inff() ? 0.f : m;
  s = 0.f;
#pragma unroll
  for (int n = 0; n < C::NI; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float v = exp_of(acc[n][e] - at);
      s += in(n, e) ? v : 0.f;
    }
  s += __shfl_xor(s, 16);
  s += __shfl_xor(s, 32);
}
template <class C>
__device__ __forceinline__ void finish_stats16(const TileArgs& t, const LossArgs& l, int target, const f32x4 (&acc)[C::NI], int row0, int col0, int lane) {
  const int g = lane >> 4, row = row0 + (lane & 15), off = target - col0;
  const bool in_row = !C::EDGE || row < t.rows;
  float m, s;
  if (!C::EDGE || col0 + C::WTN <= t.cols) stats_of<C, true>(acc, 0, g, m, s);
  else stats_of<C, false>(acc, t.cols - col0, g, m, s);
  if (in_row && g == 0) l.stats[(long long)(col0 / C::WTN) * t.rows + row] = make_float2(m, s);
  const bool here = in_row && off >= 0 && off < C::WTN && (off >> 2 & 3) == g;
  if (__ballot(here) == 0) return;
  float z = 0.f;
#pragma unroll
  for (int n = 0; n < C::NI; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n * 16 + 4 * g + e == off) z = acc[n][e];
  if (here) l.logit[row] = z;
}

// Columns past the last one are zeros as far as the 16 bytes that hold it reach: the products read them.  A row that does not count, or counts for 0, is zeros
// whatever its logits are.
template <class C>
__device__ __forceinline__ void finish_dz16(const TileArgs& t, const LossArgs& l, int target, float lse, float d, const f32x4 (&acc)[C::NI], int row0, int col0, int lane) {
  const int g = lane >> 4, in_bf16 = (g & 1) * 32 + (g >> 1) * 16, off = target - col0;      // (the target's place among the wave's columns)
  const bool target_here = __ballot(off >= 0 && off < C::WTN) != 0, all = !C::EDGE || col0 + C::WTN <= t.cols;
  const uint32_t keep = d == 0.f ? 0u : 0xffffffffu;
  u32x4 p[C::NI / 2];
#pragma unroll
  for (int n = 0; n < C::NI; n += 2) {
    float v[8];
    eight_columns(acc[n], acc[n + 1], v);
    const int col = n * 16 + 16 * (g & 1) + 8 * (g >> 1);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = exp_of(v[e] - lse);
    if (target_here) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] -= col + e == off ? 1.f : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= d;
    if (!all) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = col0 + col + e < t.cols ? v[e] : 0.f;
    }
    p[n / 2] = pack8(v);
#pragma unroll
    for (int e = 0; e < 4; ++e) p[n / 2][e] &= keep;
  }
  if constexpr (C::NI == 2) {
    store_piece<C::EDGE>(t, l.dz, 2, p[0], row0, col0, lane, in_bf16);
  } else {
#pragma unroll
    for (int n = 0; n < C::NI / 2; n += 2) store_pair<C::EDGE>(t, l.dz, 2, p[n], p[n + 1], row0, col0 + n * 32, lane, in_bf16);
  }
}

// What the rows of a tile need beside their sums: a lane asks for one row's ahead of the main loop, all lanes read them out of LDS behind it.  (Asked for 16 rows at a time where
// they are used, every 16 rows wait for memory: 7490x44009x64 214 us.)  As they come, and a target in two halves: anything that was done with them
// at once would wait for them before the first slab is asked for (2328x4096x1024 33.3 us, so 32.6).
template <class C, bool GRADIENT>
struct Logits {
  const TileArgs& t;
  const LossArgs& l;
  int m0;
  uint32_t low, high;
  float lse, d;
  struct Row { int target; float lse, d; };
  const Row* rows;
  __device__ __forceinline__ void ask(const TileArgs&, int m0_) {
    m0 = m0_;
    const int row = min(m0 + (int)threadIdx.x, t.rows - 1);
    const uint32_t* const from = static_cast<const uint32_t*>(l.target) + ((long long)row << l.target_i64);
    low = from[0];
    high = from[l.target_i64];
    if constexpr (GRADIENT) {
      lse = l.lse[row];
      d = l.dloss[l.dloss_one ? 0 : row];
    }
  }
  __device__ __forceinline__ void keep(unsigned char* pool) {
    static_assert(C::POOL_BYTES >= 1024 + C::BM * (int)sizeof(Row) && C::BM <= C::NT, "rows of a tile");
    Row* const to = reinterpret_cast<Row*>(pool + 1024);          // (the first word is finish_cut's)
    const long long is = l.target_i64 ? (long long)((uint64_t)high << 32 | low) : (int32_t)low;
    bool counts = false;
    int target = -1;
    if ((int)threadIdx.x < C::BM && m0 + (int)threadIdx.x < t.rows) target = column_of(l, is, t.cols, counts);
    if constexpr (GRADIENT) d = counts ? d : 0.f;
    __syncthreads();                                              // all waves are done with the ring
    if constexpr (GRADIENT) {
      float most = 1.f;
      if (l.finds_most) {
        float* const waves = reinterpret_cast<float*>(pool + 64);
        const float m = wave_max(__builtin_fabsf(d));
        if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = m;
        __syncthreads();
        most = waves[0];
#pragma unroll
        for (int w = 1; w < C::NT / 64; ++w) most = fmaxf(most, waves[w]);
        most = sane_most(most);
        if (blockIdx.x == 0 && threadIdx.x == 0) *l.most = most;
      } else if (!l.dloss_one) {
        most = *l.most;
      }
      d = row_factor(l, d, most);
    }
    if ((int)threadIdx.x < C::BM) to[threadIdx.x] = Row{target, lse, d};
    __syncthreads();
    rows = to;
  }
  __device__ __forceinline__ void operator()(int, const f32x4 (&x)[C::NI], int row0, int col0, int lane) const {
    const Row r = rows[row0 - m0 + (lane & 15)];
    if constexpr (GRADIENT) finish_dz16<C>(t, l, r.target, r.lse, r.d, x, row0, col0, lane);
    else finish_stats16<C>(t, l, r.target, x, row0, col0, lane);
  }
};

template <class C, bool GRADIENT>
__global__ void __launch_bounds__(C::NT, C::OCC) logits_kernel(const TileArgs t, const LossArgs l) {
  __shared__ __attribute__((aligned(1024))) unsigned char pool[C::POOL_BYTES];
  Logits<C, GRADIENT> logits{t, l};
  tile_body<C>(t, pool, logits);
}

}  // namespace flux_ffn
