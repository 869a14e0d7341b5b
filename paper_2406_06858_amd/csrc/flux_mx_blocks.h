// Rows of numbers eight to a lane, and blocks of 32 numbers four lanes to a block, as the casts and the norm read and write them.
#pragma once
#include <hip/hip_runtime.h>

namespace flux_ffn {

constexpr int PER_LANE = 8;                      // numbers of a row that a lane takes: four lanes a block

__device__ __forceinline__ float from_bf16(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// The lane's numbers, zeros past the end of the row.  Rows need no alignment beyond their type's.  WHOLE: `left` is 8 and more, or 0 and less.
template <bool WHOLE = false, class T>
__device__ __forceinline__ void load8(const T* p, int left, float (&x)[PER_LANE]) {
  T v[PER_LANE];
  if (left >= PER_LANE) {
    __builtin_memcpy(v, p, sizeof(v));
  } else if (WHOLE) {
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) v[i] = T(0);
  } else {
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) v[i] = i < left ? p[i] : T(0);
  }
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) {
    if constexpr (sizeof(T) == 2) x[i] = from_bf16(v[i]);
    else x[i] = v[i];
  }
}

// The same, kept as they are in memory, in words, until they are used.  The lane at the end of a row that is no multiple of 8 asks for the row's last 8 numbers
// in one load as well, and they are put in their places when they are there: an answer for each number, waited for one after another, would keep the
// whole row's workgroup waiting.  (Rows of fewer than 8 numbers are read one by one.)
template <class T>
struct Raw8 {
  static constexpr int WORDS = PER_LANE * sizeof(T) / 4;
  uint32_t v[WORDS];
  // numbers k .. k + 7 of the row of K that `row` points to
  template <bool WHOLE>
  __device__ __forceinline__ void ask(const T* row, int k, int K) {
    if (k + PER_LANE <= K || (!WHOLE && K >= PER_LANE && k < K)) {
      __builtin_memcpy(v, row + (WHOLE ? k : min(k, K - PER_LANE)), sizeof(v));
      return;
    }
#pragma unroll
    for (int i = 0; i < WORDS; ++i) v[i] = 0u;
    if (WHOLE || k >= K) return;
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) {
      if (k + i >= K) continue;
      if constexpr (sizeof(T) == 2) v[i / 2] |= (uint32_t)row[k + i] << (i % 2 * 16);
      else v[i] = __float_as_uint(row[k + i]);
    }
  }
  // behind ask, ahead of the first use
  template <bool WHOLE>
  __device__ __forceinline__ void settle(int k, int K) {
    const int over = k + PER_LANE - K;                    // numbers at the front that are another lane's
    if (WHOLE || K < PER_LANE || over <= 0 || over >= PER_LANE) return;
    const int words = over * (int)sizeof(T) / 4;
#pragma unroll
    for (int step = 1; step < WORDS; step *= 2)
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        const uint32_t up = i + step < WORDS ? v[i + step] : 0u;
        v[i] = words & step ? up : v[i];
      }
    if (sizeof(T) == 2 && over % 2 != 0) {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) v[i] = v[i] >> 16 | (i + 1 < WORDS ? v[i + 1] << 16 : 0u);
    }
  }
  // What was made of the words so far is forgotten: they alone stay in registers.
  __device__ __forceinline__ void fold() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) asm volatile("" : "+v"(v[i]));
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 2) return __uint_as_float(i % 2 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
    else return __uint_as_float(v[i]);
  }
};

// 16 bytes at any address that the matrix's type allows
typedef uint32_t vec16 __attribute__((ext_vector_type(4), aligned(2)));

// The lane's numbers to a row that has `left` more; STREAM: past the caches.
template <bool STREAM, bool WHOLE = false, class T>
__device__ __forceinline__ void store8(T* p, int left, const T (&v)[PER_LANE]) {
  if (left >= PER_LANE) {
    vec16 w[sizeof(v) / 16];
    __builtin_memcpy(w, v, sizeof(v));
#pragma unroll
    for (unsigned i = 0; i < sizeof(v) / 16; ++i) {
      if (STREAM) __builtin_nontemporal_store(w[i], reinterpret_cast<vec16*>(p) + i);
      else reinterpret_cast<vec16*>(p)[i] = w[i];
    }
  } else if (!WHOLE) {
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i)
      if (i < left) p[i] = v[i];
  }
}

// The bits of the largest magnitude of a block (four neighbouring lanes): NaN and infinity come out on top, at 0x7f800000 or more.
__device__ __forceinline__ uint32_t block_top(const float (&x)[PER_LANE]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  return max(top, (uint32_t)__shfl_xor((int)top, 2));
}

// The lane's eight codes of 4 bits, and the block's byte.
// The hardware's conversion divides by 2^(exponent field - 127) of its scale (a field of 0 counts as one like any other), rounds to nearest
// even and saturates: what the format asks for, checked bit for bit over all bf16 numbers and at every tie.
__device__ __forceinline__ uint32_t encode4(const float (&x)[PER_LANE], uint32_t& byte) {
  const uint32_t top = block_top(x);
  const bool finite = top < 0x7f800000u;
  const int e = max((int)(top >> 23) - 2, 0);
  const float scale = __uint_as_float((uint32_t)e << 23);
  uint32_t codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
  byte = finite ? (uint32_t)e : 255u;
  return finite ? codes : 0u;
}

// The same of 8 bits (E4M3).  Numbers are held at 448 before the conversion, which makes NaN of what is beyond.
__device__ __forceinline__ uint2 encode8(const float (&x)[PER_LANE], uint32_t& byte) {
  typedef short short2_t __attribute__((ext_vector_type(2)));
  const uint32_t top = block_top(x);
  const bool finite = top < 0x7f800000u;
  const int e = max((int)(top >> 23) - 8, 0);
  const float scale = __uint_as_float((uint32_t)e << 23), most = 448.f * (e ? scale : 0x1p-127f);
  float v[PER_LANE];
#pragma unroll
  for (int i = 0; i < PER_LANE; ++i) v[i] = fminf(fmaxf(x[i], -most), most);
  short2_t lo = {0, 0}, hi = {0, 0};
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, v[0], v[1], scale, false);
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, v[2], v[3], scale, true);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, v[4], v[5], scale, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, v[6], v[7], scale, true);
  byte = finite ? (uint32_t)e : 255u;
  return finite ? make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)) : make_uint2(0u, 0u);
}

}  // namespace flux_ffn
