// Products of few rows (gfx950): the weights are read once, and nothing else counts.
//
// A workgroup takes 16 or 32 columns of products (gated: 16 of gate and the same 16 of up) and the whole contraction, which its
// four waves share out in turns of 128 or 256 bytes a row; the waves' sums meet in LDS, in ascending order.  Nobody joins
// anything across workgroups and no barrier stands in the main loop (4 bits: one in 8192 numbers, for the scales): a wave has LDS of its own
// and loads of its next turns on their way into it while it multiplies this one.  The rows are read by every workgroup, out of the L2.
//
// What bounds it is how a compute unit's loads are answered.  Of a load whose neighbouring lanes lie in different rows, as an
// MFMA's operand wants them, it answers 16 bytes a clock: 34 GB/s a unit from the L2, 27 from memory, wherever the bytes
// come from.  With eight or more lanes to a row it is 110 and 40 (one unit's loads in a loop of nothing else; what this kernel reaches in all is in
// few_us).  So rows go to LDS as runs of 128 bytes and the operands come out of LDS.
//
// bf16: MFMA 16x16x32, a lane of a fragment holds 8 numbers of one row.  4 bits: 16x16x128, a lane holds one block of 32.
//
// Measured: gated bf16 1x3584x8192 20 us (5.9 TB/s of weights); 4 bits 8x8192x3584 5.5 us (2.9 TB/s), gated 4 bits 64x3584x8192 10.5 us
// (2.9 TB/s; each of 224 workgroups reads the 64 rows, 64 MB out of the L2).  The tile kernel with cut tiles took 32, 13.8 and 17.8 us for
// them, launch included.
#pragma once
#include "flux_ffn_tile.h"

namespace flux_ffn {

struct FewArgs {
  const void* a;
  const void* b[2];
  const uint8_t* sa;
  const uint8_t* sb[2];
  uint32_t pitch_a, pitch_b, bytes_a, bytes_b, pitch_s;
  int32_t rows, cols;
  int32_t row_vecs;              // 16-byte pieces of a row of either operand
  int32_t act, out_f32;
  int64_t ld;
  void* out;
  __bf16 *g, *u;
};

// BLOCKS: 16-column blocks of products (gated: 2); MB: 16-row blocks; SLABS: 128-byte slabs of a turn; RING: turns in LDS, of which up to
// two hold all that a wave takes of a short row.
template <bool MX_, int HALVES_, int BLOCKS_, int MB_, int SLABS_, int RING_>
struct FewCfg {
  static constexpr bool MX = MX_;
  static constexpr int HALVES = HALVES_, BLOCKS = BLOCKS_, MB = MB_, SLABS = SLABS_, RING = RING_;
  static constexpr int WAVES = 4, NT = 256, COLS = 16 * BLOCKS / HALVES;
  static constexpr int ROWS = 16 * (BLOCKS + MB);                          // of both operands: the columns' first
  static constexpr int SLAB_BYTES = ROWS * 128;
  // 4 bits: scales of 8192 numbers (a chunk: 256 bytes) of every row at a time, for all waves, into the one of two places while the other
  // is in use; a load is four rows.
  static constexpr int CHUNK = 32 / SLABS, SC_BYTES = MX ? ROWS * 256 : 0, SC_LOADS = MX ? ROWS / 16 : 0;      // turns; bytes; loads of a wave
  static constexpr int TURN_BYTES = SLABS * SLAB_BYTES;
  static constexpr int LOADS = SLABS * ROWS / 8;                           // of a wave and turn
  static constexpr int PLACES = RING > 2 || MB == 4 ? 2 : 1;                // (a short row has one chunk)
  static constexpr int POOL_BYTES = WAVES * RING * TURN_BYTES + PLACES * SC_BYTES;
  static_assert((RING - 1) * LOADS < 64 && POOL_BYTES <= 160 * 1024, "loads in flight, LDS");
  static_assert(POOL_BYTES >= WAVES * MB * BLOCKS * 1024, "room for the waves' sums");
};

template <int OFF>
__device__ __forceinline__ void lds_read16(u32x4& v, uint32_t base) { asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(base), "n"(OFF)); }
template <int OFF>
__device__ __forceinline__ void lds_read2(uint32_t& v, uint32_t base) { asm volatile("ds_read_u16 %0, %1 offset:%2" : "=v"(v) : "v"(base), "n"(OFF)); }

// A workgroup's columns n0 .. n0 + COLS - 1 of the product: its waves' sums, in LDS for few_sum.
template <class C>
__device__ __forceinline__ const float* few_body(const FewArgs& t, unsigned char* pool, int n0) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = lane & 15, g = lane >> 4;
  constexpr uint32_t OUTSIDE = 0xfffffff0u;
  const auto rsrc = [](const void* p, uint32_t bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00027000); };
  const __amdgpu_buffer_rsrc_t ra = rsrc(t.a, t.bytes_a), rb[2] = {rsrc(t.b[0], t.bytes_b), rsrc(t.b[C::HALVES - 1], t.bytes_b)};
  const __amdgpu_buffer_rsrc_t rsa = rsrc(t.sa, C::MX ? (uint32_t)t.rows * t.pitch_s : 0u);
  const __amdgpu_buffer_rsrc_t rsb[2] = {rsrc(t.sb[0], C::MX ? (uint32_t)t.cols * t.pitch_s : 0u), rsrc(t.sb[C::HALVES - 1], C::MX ? (uint32_t)t.cols * t.pitch_s : 0u)};
  unsigned char* const mine = pool + wave * (C::RING * C::TURN_BYTES);

  // One load is eight rows by 128 bytes; the swizzle is in which 16 bytes a lane fetches.  A lane outside the matrices loads
  // zeros and touches no memory.
  const int r8 = lane >> 3, s8 = (lane & 7) ^ swizzle<C::MX>(r8);
  const auto ask = [&](int slot, int q) {
#pragma unroll
    for (int s = 0; s < C::SLABS; ++s) {
      const int vec = (q * C::SLABS + s) * 8 + s8;
      const bool in = vec < t.row_vecs;
#pragma unroll
      for (int d = 0; d < C::ROWS / 8; ++d) {
        unsigned char* const to = mine + slot * C::TURN_BYTES + s * C::SLAB_BYTES + d * 1024;
        if (d < 2 * C::BLOCKS) {
          const int half = C::HALVES == 2 ? d / 2 : 0, col = n0 + (C::HALVES == 2 ? d % 2 : d) * 8 + r8;
          const uint32_t off = in && col < t.cols ? (uint32_t)col * t.pitch_b + (uint32_t)vec * 16u : OUTSIDE;
          __builtin_amdgcn_raw_ptr_buffer_load_lds(rb[half], (flux::lds_void_t*)to, 16, (int)off, 0, 0, 2);      // (streamed: read once)
        } else {
          const int row = (d - 2 * C::BLOCKS) * 8 + r8;
          const uint32_t off = in && row < t.rows ? (uint32_t)row * t.pitch_a + (uint32_t)vec * 16u : OUTSIDE;
          __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (flux::lds_void_t*)to, 16, (int)off, 0, 0, 0);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  // 4 bits: this wave's share of the scales of chunk c.  Piece p (16 bytes, two slabs) of row r lies in place p ^ (r % 16).
  unsigned char* const scales = pool + C::WAVES * C::RING * C::TURN_BYTES;
  const auto ask_scales = [&](int c) {
    const int r = wave * 4 + (lane >> 4);               // in a block of 16, which the l-th load of the four waves is
    const uint32_t at = (uint32_t)c * 256u + (uint32_t)(((lane & 15) ^ r) * 16);
    const bool in = at < t.pitch_s;
#pragma unroll
    for (int l = 0; l < C::SC_LOADS; ++l) {
      unsigned char* const to = scales + c % C::PLACES * C::SC_BYTES + (l * C::WAVES + wave) * 1024;
      if (l < C::BLOCKS) {
        const int half = C::HALVES == 2 ? l : 0, col = n0 + (C::HALVES == 2 ? 0 : 16 * l) + r;
        const uint32_t off = in && col < t.cols ? (uint32_t)col * t.pitch_s + at : OUTSIDE;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsb[half], (flux::lds_void_t*)to, 16, (int)off, 0, 0, 0);
      } else {
        const int row = 16 * (l - C::BLOCKS) + r;
        const uint32_t off = in && row < t.rows ? (uint32_t)row * t.pitch_s + at : OUTSIDE;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsa, (flux::lds_void_t*)to, 16, (int)off, 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  f32x4 acc[C::MB][C::BLOCKS];
#pragma unroll
  for (int m = 0; m < C::MB; ++m)
#pragma unroll
    for (int h = 0; h < C::BLOCKS; ++h) acc[m][h] = f32x4{0.f, 0.f, 0.f, 0.f};
  uint32_t frag[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) frag[ks] = flux::lds_address(mine) + i * 128 + (((C::MX ? 2 * g + ks : ks * 4 + g) ^ swizzle<C::MX>(i)) << 4);
  const uint32_t scale = flux::lds_address(scales) + i * 256 + 2 * g;

  const auto multiply = [&](int slot, int q) {
    const uint32_t base = (uint32_t)(slot * C::TURN_BYTES);
    // (the chunk's place; in it the piece of this turn's slabs, and which half of it)
    const int in_chunk = q % C::CHUNK * C::SLABS;
    const uint32_t from = scale + (uint32_t)(q / C::CHUNK % C::PLACES * C::SC_BYTES) + (uint32_t)(((in_chunk >> 1) ^ i) << 4) + (uint32_t)((in_chunk & 1) * 8);
    flux::static_for<C::SLABS>([&](auto s_) {
      constexpr int s = decltype(s_)::value;
      u32x4 f[2][C::BLOCKS + C::MB];
      uint32_t sc[C::MX ? C::BLOCKS + C::MB : 1];
      const uint32_t f0 = frag[0] + base, f1 = frag[1] + base, fs = from + s * 8;
      flux::static_for<C::BLOCKS + C::MB>([&](auto b_) {
        constexpr int b = decltype(b_)::value, OFF = s * C::SLAB_BYTES + b * 2048;
        lds_read16<OFF>(f[0][b], f0);
        lds_read16<OFF>(f[1][b], f1);
        if constexpr (C::MX) lds_read2<b * 16 * 256>(sc[b], fs);
      });
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int b = 0; b < C::BLOCKS + C::MB; ++b) {
        asm volatile("" : "+v"(f[0][b]), "+v"(f[1][b]));
        if (C::MX) asm volatile("" : "+v"(sc[b]));
      }
      flux::static_for<2>([&](auto k_) {
        constexpr int ks = decltype(k_)::value;
#pragma unroll
        for (int m = 0; m < C::MB; ++m)
#pragma unroll
          for (int h = 0; h < C::BLOCKS; ++h) {
            const u32x4 x = f[ks][C::BLOCKS + m], y = f[ks][h];
            if constexpr (C::MX) {
              typedef __attribute__((ext_vector_type(8))) int i32x8;
              const i32x8 xw = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0}, yw = {(int)y[0], (int)y[1], (int)y[2], (int)y[3], 0, 0, 0, 0};
              acc[m][h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(xw, yw, acc[m][h], 4, 4, ks, (int)sc[C::BLOCKS + m], ks, (int)sc[h]);
            } else {
              acc[m][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc[m][h], 0, 0, 0);
            }
          }
      });
    });
  };

  const int turns = (t.row_vecs + 8 * C::SLABS - 1) / (8 * C::SLABS);
  if constexpr (C::MX) ask_scales(0);
#pragma unroll
  for (int j = 0; j < C::RING - 1; ++j) ask(j, wave + j * C::WAVES);
  int slot = 0, next = C::RING - 1;
  // (every wave goes through as many rounds as the first: a chunk begins with a barrier; a turn past the end is asked for as zeros)
  for (int q0 = 0; q0 < turns; q0 += C::WAVES) {
    ask(next, q0 + wave + (C::RING - 1) * C::WAVES);
    flux::wait_vm_at_most<(C::RING - 1) * C::LOADS>();
    asm volatile("" ::: "memory");
    if (C::MX && q0 % C::CHUNK == 0) {
      // this chunk's scales are there (older than this turn's loads), everybody's; the place of the chunk before is free
      flux::barrier_keeping_loads_in_flight();
      if (C::PLACES > 1 && q0 + C::CHUNK < turns) ask_scales(q0 / C::CHUNK + 1);
    }
    multiply(slot, q0 + wave);
    slot = slot + 1 == C::RING ? 0 : slot + 1;
    next = next + 1 == C::RING ? 0 : next + 1;
  }

  flux::wait_vm0_and_barrier();                         // the sums lie over the turns
  float* const red = reinterpret_cast<float*>(pool);
#pragma unroll
  for (int m = 0; m < C::MB; ++m)
#pragma unroll
    for (int h = 0; h < C::BLOCKS; ++h) *reinterpret_cast<f32x4*>(red + ((wave * C::MB + m) * C::BLOCKS + h) * 256 + lane * 4) = acc[m][h];
  __syncthreads();
  return red;
}

// The sum of row `row`, column c of the workgroup's, `half` of a gated product.  (A lane of a 16x16 block held rows 4g .. 4g+3 of column i.)
template <class C>
__device__ __forceinline__ float few_sum(const float* red, int row, int c, int half = 0) {
  const int at = ((row >> 4) * C::BLOCKS + c / 16 + half) * 256 + ((row >> 2 & 3) * 16 + c % 16) * 4 + (row & 3);
  float v = 0.f;
#pragma unroll
  for (int w = 0; w < C::WAVES; ++w) v += red[w * C::MB * C::BLOCKS * 256 + at];
  return v;
}

template <class C>
__global__ void __launch_bounds__(C::NT) few_kernel(const FewArgs t) {
  __shared__ __attribute__((aligned(1024))) unsigned char pool[C::POOL_BYTES];
  const int n0 = by_die((int)blockIdx.x, (int)gridDim.x) * C::COLS;
  const float* const red = few_body<C>(t, pool, n0);
  for (int e = threadIdx.x; e < C::MB * 16 * C::COLS; e += C::NT) {
    const int c = e % C::COLS, row = e / C::COLS, col = n0 + c;
    if (row >= t.rows || col >= t.cols) continue;
    float v = few_sum<C>(red, row, c);
    const float u = C::HALVES == 2 ? few_sum<C>(red, row, c, 1) : 0.f;
    const long long to = row * t.ld + col;
    if constexpr (C::HALVES == 2) {
      if (t.g != nullptr) {
        t.g[to] = (__bf16)v;
        t.u[to] = (__bf16)u;
      }
      const float a = t.act == FLUX_ACT_SILU ? act<FLUX_ACT_SILU, true>(v) : t.act == FLUX_ACT_GELU ? act<FLUX_ACT_GELU, true>(v) : act<FLUX_ACT_GELU_TANH, true>(v);
      v = a * u;
    }
    if (t.out_f32) static_cast<float*>(t.out)[to] = v;
    else static_cast<__bf16*>(t.out)[to] = (__bf16)v;
  }
}

}  // namespace flux_ffn
