// Matrices to 4-bit blocks of 32 with one power of two each, and back (flux_mx4_quantize, flux_mx4_dequantize); 8-bit blocks back
// (flux_mx8_dequantize: flux_norm writes them).
//
// For a block x with largest magnitude a:  e = max(floor(log2 a) - 2, -127),  code_i = E2M1(x_i / 2^e) rounded to nearest
// even and held at 6.  floor(log2 a) is a's exponent field, so the largest magnitude is taken over the bit patterns, where
// NaN and infinity come out on top and are told apart by being 0x7f800000 or more.
//
// What bounds both kernels is memory: 2 or 4 bytes read and 17/32 written a number, or the other way round.  Measured: to 4 bits
// 4096x8192 fp32 26 us (5.8 TB/s), 8192x3413 fp32 (rows at odd multiples of 4 bytes) 22.6 (5.6), 8192x8192 bf16 36 (4.7); back to bf16
// 8192x8192 27.5 (6.2), 8192x3413 15.6 (4.5).  Codes by comparisons with the midpoints instead of the conversion instruction took 29.5, 30.4
// and 54.8 us.
#include "flux_ffn_internal.h"
#include "flux_mx_blocks.h"
#include "flux_norm.h"

namespace flux_ffn {

constexpr int PER_WAVE = 64 * PER_LANE;          // 16 blocks: the 16 bytes of scales that a wave writes are the padding's unit

struct CastArgs {
  const void* src;
  void* dst;
  uint8_t* q;
  uint8_t* scales;
  long long ld;                                  // of src or dst, in elements
  int32_t rows, K, waves_per_row;
  uint32_t row_bytes, scale_row_bytes;
};

// Four waves a workgroup; a grid is at most 2^23 workgroups wide (2^32 threads are too many for the hardware's count).
constexpr long long GRID_X = 1ll << 23;
__device__ __forceinline__ long long wave_id() { return ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6); }

template <class T>
__global__ void __launch_bounds__(256) quantize_kernel(const CastArgs c) {
  const int lane = threadIdx.x & 63;
  const long long w = wave_id();
  if (w >= (long long)c.rows * c.waves_per_row) return;
  const int row = (int)(w / c.waves_per_row), seg = (int)(w % c.waves_per_row);
  const int k = seg * PER_WAVE + lane * PER_LANE;
  float x[PER_LANE];
  load8(static_cast<const T*>(c.src) + (long long)row * c.ld + k, c.K - k, x);
  uint32_t e;
  const uint32_t codes = encode4(x, e);
  const int block = k / 32;
  if (k < (c.K + 31) / 32 * 32) *reinterpret_cast<uint32_t*>(c.q + (long long)row * c.row_bytes + k / 2) = codes;
  if (lane % 4 == 0) c.scales[(long long)row * c.scale_row_bytes + block] = (uint8_t)e;
}

// What a lane's eight codes of BITS bits stand for.  4 bits: three significant bits at most, exact in bf16; 8 bits: four, of which the
// rounding to bf16 drops some where a result is below its normal numbers.
template <int BITS> struct Codes { typedef uint32_t type; };
template <> struct Codes<8> { typedef uint2 type; };
__device__ __forceinline__ void decode(uint32_t codes, float scale, float (&x)[PER_LANE]) {
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    // exponent and mantissa of E2M1 onto those of fp32: 0 and 0.5 by a product, the rest by place
    const uint32_t m = codes >> (4 * i) & 7u;
    const float a = (m < 2u ? 0.5f * (float)m : __uint_as_float((126u << 23) + (m << 22))) * scale;
    x[i] = __uint_as_float(__float_as_uint(a) | (codes >> (4 * i) & 8u) << 28);
  }
}
__device__ __forceinline__ void decode(const uint2& codes, float scale, float (&x)[PER_LANE]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int c = (int)(h ? codes.y : codes.x);
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
    x[4 * h] = lo[0] * scale;
    x[4 * h + 1] = lo[1] * scale;
    x[4 * h + 2] = hi[0] * scale;
    x[4 * h + 3] = hi[1] * scale;
  }
}

// A lane's eight numbers at k of a row.
template <class T, class V>
__device__ __forceinline__ void decode8(const CastArgs& c, int row, int k, const V& codes, uint32_t e) {
  const float scale = e == 255u ? __uint_as_float(0x7fc00000u) : e ? __uint_as_float(e << 23) : 0x1p-127f;
  float x[PER_LANE];
  decode(codes, scale, x);
  T v[PER_LANE];
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = x[i];
    else if constexpr (sizeof(V) == 4) v[i] = (uint16_t)(__float_as_uint(x[i]) >> 16);
    else v[i] = __builtin_bit_cast(uint16_t, (__bf16)x[i]);
  }
  T* const p = static_cast<T*>(c.dst) + (long long)row * c.ld + k;
  // (past the caches: us, kept there / past them, 8192x8192 40.6 / 27.7, 4096x8192 22.6 / 12.7)
  store8<true>(p, c.K - k, v);
}

// The byte that number k of a row is in.
template <int BITS>
constexpr __device__ int byte_of(int k) { return k / (8 / BITS); }
static_assert(byte_of<8>((1 << 30) - 8) == (1 << 30) - 8 && byte_of<4>((1 << 30) - 8) == (1 << 29) - 4, "rows of 2^30 numbers, in 32 bits");

// A wave takes SEGS neighbouring pieces of a row: their loads are out together.  us by SEGS, 1 / 2 / 4, to bf16: 64x8192 2.9 / 3.3 / 4.0,
// 1024x8192 6.1 / 5.7 / 5.9, 8192x8192 31.2 / 26.5 / 26.9, 8192x3413 16.3 / 14.7 / 16.1; to fp32: 64x8192 3.1 / 3.5 / 4.1, 8192x8192 105 / 102 / 115.
constexpr int SEGS = 4;
template <int BITS, class T>
__global__ void __launch_bounds__(256) dequantize_kernel(const CastArgs c) {
  const int lane = threadIdx.x & 63;
  const long long w = wave_id();
  if (w >= (long long)c.rows * c.waves_per_row) return;
  const int row = (int)(w / c.waves_per_row), seg = (int)(w % c.waves_per_row) * SEGS;
  typedef typename Codes<BITS>::type V;
  V codes[SEGS];
  uint32_t e[SEGS];
#pragma unroll
  for (int s = 0; s < SEGS; ++s) {
    const int k = min((seg + s) * PER_WAVE + lane * PER_LANE, (c.K - 1) / PER_LANE * PER_LANE);      // (past the end: the last again)
    codes[s] = *reinterpret_cast<const V*>(c.q + (long long)row * c.row_bytes + byte_of<BITS>(k));
    e[s] = c.scales[(long long)row * c.scale_row_bytes + k / 32];
  }
#pragma unroll
  for (int s = 0; s < SEGS; ++s) {
    const int k = (seg + s) * PER_WAVE + lane * PER_LANE;
    if (k < c.K) decode8<T>(c, row, k, codes[s], e[s]);
  }
}

static int cast_args(int32_t rows, int32_t K, int32_t dtype, const void* wide, int64_t ld, const void* q, const void* scales, int segs, int bits, CastArgs* c) {
  if (wide == nullptr || q == nullptr || scales == nullptr || (dtype != FLUX_BF16 && dtype != FLUX_F32)) return FLUX_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(scales, 16) || !aligned(wide, dtype == FLUX_BF16 ? 2 : 4)) return FLUX_ERR_INVALID_ARG;
  if (rows < 1 || K < 1 || K > (1 << 30)) return FLUX_ERR_SHAPE;          // (what a wave takes of a row may end past the row's end)
  const long long pitch = ld ? ld : K;
  if (pitch < K || !below_limit(rows, pitch, K)) return FLUX_ERR_SHAPE;
  c->q = static_cast<uint8_t*>(const_cast<void*>(q));
  c->scales = static_cast<uint8_t*>(const_cast<void*>(scales));
  c->ld = pitch;
  c->rows = rows;
  c->K = K;
  c->waves_per_row = (K + PER_WAVE * segs - 1) / (PER_WAVE * segs);
  c->row_bytes = (uint32_t)row_bytes(K) * (bits / 4);
  c->scale_row_bytes = (uint32_t)scale_row_bytes(K);
  return FLUX_OK;
}

static dim3 cast_grid(const CastArgs& c) {
  const long long n = ((long long)c.rows * c.waves_per_row + 3) / 4, x = n < GRID_X ? n : GRID_X;
  return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}

template <int BITS>
static int dequantize(int32_t rows, int32_t K, const void* q, const void* scales, int32_t dst_dtype, void* dst, int64_t ld, void* stream) {
  CastArgs c = {};
  const int st = cast_args(rows, K, dst_dtype, dst, ld, q, scales, SEGS, BITS, &c);
  if (st != FLUX_OK) return st;
  c.dst = dst;
  FFN_HIP(start(dst_dtype == FLUX_BF16 ? dequantize_kernel<BITS, uint16_t> : dequantize_kernel<BITS, float>, cast_grid(c), static_cast<hipStream_t>(stream), c));
  return FLUX_OK;
}

}  // namespace flux_ffn

using namespace flux_ffn;

extern "C" {

size_t flux_mx4_row_bytes(int32_t K) { return K < 1 ? 0 : (size_t)row_bytes(K); }
size_t flux_mx4_scale_row_bytes(int32_t K) { return K < 1 ? 0 : (size_t)scale_row_bytes(K); }

int flux_mx4_quantize(int32_t rows, int32_t K, int32_t src_dtype, const void* src, int64_t ld, void* q, void* scales, void* stream) {
  CastArgs c = {};
  const int st = cast_args(rows, K, src_dtype, src, ld, q, scales, 1, 4, &c);
  if (st != FLUX_OK) return st;
  c.src = src;
  FFN_HIP(start(src_dtype == FLUX_BF16 ? quantize_kernel<uint16_t> : quantize_kernel<float>, cast_grid(c), static_cast<hipStream_t>(stream), c));
  return FLUX_OK;
}

int flux_mx4_dequantize(int32_t rows, int32_t K, const void* q, const void* scales, int32_t dst_dtype, void* dst, int64_t ld, void* stream) {
  return dequantize<4>(rows, K, q, scales, dst_dtype, dst, ld, stream);
}

size_t flux_mx8_row_bytes(int32_t K) { return K < 1 ? 0 : 2 * (size_t)row_bytes(K); }

int flux_mx8_dequantize(int32_t rows, int32_t K, const void* q, const void* scales, int32_t dst_dtype, void* dst, int64_t ld, void* stream) {
  return dequantize<8>(rows, K, q, scales, dst_dtype, dst, ld, stream);
}

}  // extern "C"
