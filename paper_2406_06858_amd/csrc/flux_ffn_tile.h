// The tile kernel of the gated block's products (gfx950): one main loop for bf16 operands in any order and for 4-bit
// blocks.
//
// A tile is BM rows by BN columns of products, four waves of BM/2 x BN/2, a slab of contraction 128 bytes a row.  The
// schedule is the one of the library's fused GEMMs (MmaPipe in flux_device.h): slabs go from memory into LDS directly,
// fragments of the next k-step are read and loads of the slab after next are issued between the MFMAs of this one, and a
// slab costs one barrier.  What differs by product:
//
//   gated    the columns of a wave are half gate, half up, of the SAME columns of the result: activation and product take
//            both from the wave's own accumulators, and A is read once for two weights.
//   dX       the contraction runs over dG Wg^T and then dU Wu^T: one accumulator, two segments of slabs.
//   dW       both operands hold the contraction (tokens) along their rows' index: both tiles lie in LDS as they do in memory
//            and both fragments are read transposing.  The gradients of both weights are one grid.
//   4 bits   a slab's 128 bytes are 256 numbers, a k-step's MFMA is 16x16x128 with one scale per lane and operand: a lane
//            holds one block of 32.  Same bytes, same fragment reads and same cycles per slab as bf16, four times the numbers.
//
// Measured with random operands (256x256 tiles), calls in turn: gated 4096x3584x8192 with G and U kept 345 us (1.39 PF), dX
// 8192x8192x2*3584 622 us (1.55 PF) and both weights' gradients 632 us (1.52 PF), 4 bits 8192x12288x6144 275 to 290 us (4.3 to 4.5 PF) and gated
// 4096x3584x8192 110 us (4.4 PF).  How busy the MFMA units were, at which clock, in one run of counters: gated 69 % at 1.87 GHz (357 us),
// gradients 78 % at 1.87 GHz, 4 bits 53 % at 1.94 GHz (287 us), gated 4 bits 47 % at 2.07 GHz (118 us).
// What bounds the bf16 ones is power: with operands of zeros the gated product takes 282 us, and 14 calls of it back to back take 339 to
// 446 us as the card's power control lowers the clock and raises it again.  4 bits: power takes 13 to 20 % (zeros: 241 and 96 us), the
// rest is that a ring of two slabs makes every barrier wait for all loads, those of the scales among them (zeros, us a slab: 1.54; 1.38 without the
// scales' loads, still waiting for every load; 1.11 without memory traffic).  Conflicts of the LDS: none in bf16, the 17 % of 4 bits are the scales'.
// Products that fill less than a round of the card wait for their loads: a slab of 256x128 in bf16, 48 KB, takes 0.55 us where few units
// are at work and 0.78 where all are (fitted, see SHAPES): 87 and 61 GB/s a unit, the latter 16 TB/s out of the L2s together.  Rows
// that are no whole lines of 128 bytes: gated backward 1496x3400x5112 229 us, 1496x3456x5120 214, most of it dX (115 / 103).
#pragma once
#include "flux_device.h"
#include "flux_ffn_act.h"

namespace flux_ffn {

using flux::bf16x8;
using flux::f32x4;
using flux::FragHalves;
using flux::u32x2;
using flux::u32x4;

// (LOGITS: the plan of a plain product along the contraction, whose tiles run the loop of DX_NK on one segment)
enum Kind : int { LOGITS = -1, GLU_NK = 0, GLU_KN = 1, DX_NK = 2, DX_KN = 3, DW = 4, MX_GEMM = 5, MX_GLU = 6, KINDS = 7 };

struct TileArgs {
  const void* a[2];              // dX: by segment; dW: by weight; else [0]
  const void* b[2];              // gated: gate, up; dX: by segment; dW: by weight; else [0]
  const uint8_t* sa;             // 4 bits: scales of A; of B
  const uint8_t* sb[2];
  uint32_t pitch_a, pitch_b;     // bytes
  uint32_t bytes_a, bytes_b;     // extents
  uint32_t pitch_s;              // of a row of scales
  int32_t rows, cols;            // of the result
  int32_t depth;                 // of the contraction (of a segment of it), in pieces of two bytes
  int32_t seg_slabs, slabs;      // slabs of a segment; of the whole contraction
  // The first full_tiles tiles are a workgroup each; of the cut_tiles after them the contraction is cut over `parts` workgroups, each
  // part_slabs slabs.
  int32_t full_tiles, cut_tiles, parts, part_slabs;
  int32_t tiles_m, tiles_n, band;
  int32_t act, out_f32, accumulate;
  int32_t stream;                // results go past the caches
  int64_t ld;                    // pitch of the results, elements
  void* out[2];                  // dW: by weight; else [0]
  __bf16 *g, *u;                 // gated: kept for the backward pass, or null
  // SCALED kernels of dX and dW
  const float* factor;           // the sums' factor
  const float* addend;           // dX: added to the product, pitch `ld`, in the place of `accumulate`; or null
  float* partial;                // [cut_tiles][parts][BM * BN]
  uint32_t* counters;            // a word a cut tile, COUNTER_STRIDE apart, 0 between calls
};

template <int KIND_, int BM_, int BN_, int NA_, int NB_, int OCC_, bool EDGE_, bool B_ONCE_ = false, bool PHASED_ = false>
struct Cfg {
  static constexpr int KIND = KIND_, BM = BM_, BN = BN_, NA = NA_, NB = NB_, OCC = OCC_;
  static constexpr bool EDGE = EDGE_;                                        // the tile does not divide the product
  static constexpr bool B_ONCE = B_ONCE_;                                    // one row of tiles: B's lines are read once, past the caches
  static constexpr bool PHASED = PHASED_;                                    // rows along the contraction may begin anywhere in a line (see Phase)
  static constexpr bool MX = KIND == MX_GEMM || KIND == MX_GLU, A_T = KIND == DW;
  static constexpr bool TIGHT = (KIND == DX_NK || KIND == DX_KN) && BM == 256 && BN == 256;
  static constexpr bool B_NK = MX || KIND == GLU_NK || KIND == DX_NK;
  static constexpr int HALVES = KIND == GLU_NK || KIND == GLU_KN || KIND == MX_GLU ? 2 : 1;
  static constexpr int NT = 256, BK = 64;
  static constexpr int WTM = BM / 2, WTN = BN / 2, MI = WTM / 16, NI = WTN / 16, NIH = NI / HALVES;
  static constexpr int SUBN = BN / HALVES;                                   // columns of the result
  static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, SUB_BYTES = B_BYTES / HALVES;
  static constexpr int RING_BYTES = NA * A_BYTES + NB * B_BYTES;
  // 4 bits: scales come for two slabs at a time, 16 bytes a row, into a ring of RS such pairs for either operand.  Those of A for a
  // pair are asked for beside the slab ahead of it, those of B beside its first slab; RS is what that takes (see Pipe::load).
  // The last KB takes what waves without a row write.
  static constexpr int RS = (NB + 3) / 2, SC_A = BM * 16, SC_B = BN * 16, SC_BYTES = MX ? RS * (SC_A + SC_B) + 1024 : 0;
  static constexpr int POOL_BYTES = RING_BYTES + SC_BYTES;
  static_assert(POOL_BYTES * OCC <= 160 * 1024, "LDS");
  static_assert(NB >= 2 && (NA == NB || NA == NB + 1) && (!MX || (NA == NB && NB % 2 == 0)), "rings (4 bits: scales come for two slabs)");
};

// Which 16-byte slot of a row holds slot s: s ^ swizzle(row).  A fragment's lanes are rows 0..15 of slot q, the next sixteen
// the same rows of the next slot that the k-step reads; an LDS read is answered in passes of sixteen lanes that hold every
// row once, half of them of the one slot and half of the next (see swz_a).  bf16: the next slot is q + 1, and bits 0..2 of the
// row serve.  4 bits: it is q + 2 (a lane reads blocks 2g and 2g + 1 of a slab, so that both their scales are two bytes side
// by side), so bits 0 and 1 change places.
template <bool MX>
__device__ __forceinline__ int swizzle(int row) {
  return MX ? (row & 4) | ((row & 1) << 1) | ((row >> 1) & 1) : row & 7;
}

// Rows that are no whole lines.  Row r begins 16 (at + r step) bytes into a line (mod 128).  An instruction's lanes are answered four at a time, 64 bytes of a line at
// once: a row's eight pieces of a slab take two such answers if it begins with a line, and mostly four if it does not.  So the pieces are dealt to
// the row's lanes by where they lie in their line: piece q goes to slot (q + at + r step) mod 8, and a row takes three answers at most.  With an odd step that alone
// spreads sixteen rows over the banks as the swizzle does; with an even one the swizzle comes on top (the lowest bit of the slot tells rows of different
// parity apart then, and each further bit what it leaves).  Whole lines lie as the swizzle alone puts them.  us of logits' statistics, pieces in their order /
// dealt so: 2328x4096x7640 175 / 157, 1496x4000x5112 82.6 / 77.6, 1496x50257x5112 729 / 711 (in whole lines 589: a line that two slabs share is fetched for
// either).
struct Phase {
  int at = 0, step = 0;
  __device__ __forceinline__ void of(const void* p, uint32_t pitch) {
    at = (int)(reinterpret_cast<uintptr_t>(p) >> 4) & 7;
    step = (int)(pitch >> 4) & 7;
  }
  __device__ __forceinline__ int mask(int row) const { return step & 1 ? 0 : row & 7; }
  __device__ __forceinline__ int slot(int piece, int row) const { return ((piece + at + row * step) & 7) ^ mask(row); }
  __device__ __forceinline__ int piece(int slot, int row) const { return ((slot ^ mask(row)) - at - row * step) & 7; }
};

// The scaled MFMA, accumulator in place; BYTE: which byte of the scale registers counts.
template <int BYTE>
__device__ __forceinline__ void mfma_scaled(f32x4& acc, const u32x4& a, const u32x4& b, uint32_t sa, uint32_t sb) {
  if constexpr (BYTE == 0)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4" : "+a"(acc) : "v"(a), "v"(b), "v"(sa), "v"(sb));
  else
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4" : "+a"(acc) : "v"(a), "v"(b), "v"(sa), "v"(sb));
}

// ---- operand loads ---------------------------------------------------------------------------------------------
// One operand tile of R rows (or columns) of the result by 128 bytes of contraction, in LDS in one of two ways:
//   along   rows of 128 bytes, one instruction 8 rows;
//   across  (T) one row per step of the contraction, R values each, one instruction 512 / R of those.
// (The same patterns as DmaLoader's.)  Where the contraction ends, and past the last column of a matrix that lies across, a lane loads from outside the buffer's records:
// zeros.  What it loads for a row of the result past the last one of a matrix that lies along is its finish's to leave alone (see load).
template <int R, bool T, bool EDGE, bool MX, bool ONCE, bool TIGHT>
struct OperandLoader {
  static constexpr int RPI = T ? 512 / R : 8;
  static constexpr int INSTR = (T ? 64 : R) / RPI / 4;         // per wave
  static constexpr int SLOTS = R / 8;
  static constexpr uint32_t OUTSIDE = 0xfffffff0u;
  static constexpr __device__ int wave_row(int wave) {
    return RPI == 8 ? 8 * wave : RPI == 4 ? 8 * (wave & 1) + 4 * (wave >> 1) : 2 * (wave & 1) + 8 * (wave >> 1);
  }
  static constexpr __device__ int instr_row(int p) { return RPI == 8 ? p * 32 : RPI == 4 ? 16 * p : 4 * (p & 1) + 16 * (p >> 1); }
  static_assert(RPI == 2 || RPI == 4 || RPI == 8, "the swizzle must not depend on the instruction");

  uint32_t voff, pitch;
  mutable uint32_t lds_wave;
  int k_vec;                       // along: the lane's place in the contraction
  __device__ __forceinline__ void init(uint32_t pitch_, int rows, int r0, int wave, int lane, const Phase* phase = nullptr) {
    pitch = pitch_;
    lds_wave = (uint32_t)(wave_row(wave) * (1024 / RPI));
    if constexpr (T) {
      const int k = wave_row(wave) + lane / SLOTS, s = lane % SLOTS ^ flux::swz_b<SLOTS>(wave_row(wave) + lane / SLOTS);
      // (of fewer rows than the tile takes, with gaps of 100 MB and more, a row past the last one may be past 32 bits too)
      const uint64_t at = (uint64_t)k * pitch + (uint32_t)(r0 + s * 8) * 2u;
      voff = EDGE && (r0 + s * 8 >= rows || at > OUTSIDE) ? OUTSIDE : (uint32_t)at;
    } else {
      const int row = 8 * wave + lane / 8, s = phase ? phase->piece(lane % 8, row) : lane % 8 ^ swizzle<MX>(row);
      voff = (uint32_t)(r0 + row) * pitch + (uint32_t)s * 16u;
      k_vec = s * 8;
    }
  }
  // The d-th of the wave's loads of the slab that starts at k (`depth` in all) into `tile`.  Rows of the contraction past the last one end up past the buffer's records by
  // themselves where the whole offset is the lane's (a sum that stays at the largest number instead of wrapping; a scalar offset takes no part in the range check): what is
  // left to ask is whether a slab's last pieces are in the row (once a slab), and whether rows of a contraction that lies across begin at all (uniform).  With a mask
  // for every load the 256x256 tile ran out of scalar registers: logits of 8192x4000x8192 409 us, 366 for 4096 columns without masks.
  // Along: a row of the result past the last one is mostly past the records too, but with 100 MB and more from row to row its offset may wrap to a place between the
  // caller's rows.  Whatever lies there, NaN too, comes into that row's (column's) sums and no others, and a finish neither stores these nor adds anything up over them.
  // TIGHT: the place in LDS is added up at each load.  Left to itself the compiler keeps all forty places of the large tile in scalar registers; beside the
  // segments of dX and logits there is no room for these, and they came back from vector lanes one by one.  us without / with: gradients of the loss
  // 8192x32000x8192 8518 / 8470, statistics of 8192x4000x8192 359 / 356, dX of 8192x8192 over two times 3584 633 / 625; dW, whose registers suffice, 617 / 624.
  __device__ __forceinline__ void load(int d, const __amdgpu_buffer_rsrc_t& rsrc, int k, int depth, unsigned char* tile) const {
    if constexpr (TIGHT) asm volatile("" : "+s"(lds_wave));
    uint32_t at = voff, from = T ? (uint32_t)(k + instr_row(d)) * pitch : (uint32_t)k * 2u + (uint32_t)instr_row(d) * pitch;
    if constexpr (EDGE) {
      if constexpr (T) from = k + instr_row(d) < depth ? from : OUTSIDE;
      else at = k_vec < depth - k ? voff : OUTSIDE;
      at = __builtin_elementwise_add_sat(at, from);
      from = 0u;
    }
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (flux::lds_void_t*)(tile + instr_row(d) * (1024 / RPI) + lds_wave), 16, (int)at, (int)from, 0, ONCE ? 2 : 0);
  }
};

// A slab to ask for: where it lies, or nothing in the place of one past the end (its loads touch no memory).
struct Slab {
  __amdgpu_buffer_rsrc_t r0, r1;
  int k;
};

template <class C>
struct Pipe {
  typedef OperandLoader<C::BM, C::A_T, C::EDGE, C::MX, false, C::TIGHT> LdA;
  typedef OperandLoader<C::SUBN, !C::B_NK, C::EDGE, C::MX, C::B_ONCE, C::TIGHT> LdB;
  static constexpr int NA = C::NA, NB = C::NB;
  static constexpr bool A_LEADS = NA > NB;                               // by one slab
  static constexpr int U = NA != NB ? NA * NB : NB;      // slabs after which the rings are where they were
  static constexpr int KS = 2;
  static constexpr int G = C::MI * C::NI;                                // MFMAs per k-step
  static constexpr int NF = C::MI + C::NI, NS = C::MX ? NF : 0;          // fragments of a k-step; scales of a slab
  static constexpr int LA = LdA::INSTR, LB = LdB::INSTR * C::HALVES, LS = C::MX ? 1 : 0, L = LA + LB + LS;
  static constexpr int LX = A_LEADS ? LA : 0;
  static constexpr int A_HI = (NA * C::A_BYTES + 65535) / 65536, B_HI = (NB * C::B_BYTES + 65535) / 65536;
  static constexpr int NAV = C::A_T ? C::MI : KS, NBV = C::B_NK ? KS : C::NIH;
  // Placement in MFMAs, as MmaPipe's: the barrier, the last fragment read of a k-step, the last load from the barrier on.
  static constexpr int BAR_AT = G / 8, SPREAD = (G * 15 + 15) / 16, SPAN = G * (NA != NB ? 13 : 11) / 8;
  static constexpr int load_slot(int d) { return BAR_AT + d * (SPAN - BAR_AT) / L; }
  static constexpr int loads_before(int slot) { int n = 0; while (n < L && load_slot(n) < slot) ++n; return n; }
  static constexpr int reads_before(int slot, int from, int all) { int n = 0; while (n < all && from + n * (SPREAD - from) / all < slot) ++n; return n; }
  static constexpr int L0 = loads_before(G);

  typedef std::conditional_t<C::MX, u32x4, bf16x8> Whole;
  typedef std::conditional_t<C::A_T, FragHalves, Whole> FragA;
  typedef std::conditional_t<C::B_NK, Whole, FragHalves> FragB;

  unsigned char* pool;
  LdA la;
  LdB lb;
  uint32_t voff_s[2];                // 4 bits: the lane's row of scales of A; of B
  int job, k0, KT, wave;             // first slab of this workgroup's, and how many
  uint32_t a[A_HI][NAV], b[B_HI][NBV], sc[2];
  FragA af[2][C::MI];
  FragB bf[2][C::NI];
  uint32_t fs[2][C::MX ? C::MI + C::NI : 1];

  __device__ __forceinline__ unsigned char* slab_a(int i) const { return pool + i * C::A_BYTES; }
  __device__ __forceinline__ unsigned char* slab_b(int i) const { return pool + NA * C::A_BYTES + i * C::B_BYTES; }
  // where the scales of a pair of slabs lie: place `at` of the ring
  __device__ __forceinline__ unsigned char* scales(int operand, int at) const {
    return pool + C::RING_BYTES + (operand ? C::RS * C::SC_A + at * C::SC_B : at * C::SC_A);
  }

  template <int R>
  static __device__ __forceinline__ uint32_t across(uint32_t base, int r, int i, int g) {      // transposing read of rows r.. of the result
    const int k = 8 * g + (i >> 2), n = r + 4 * (i & 3);
    return base + k * (R * 2) + (((n >> 3) ^ flux::swz_b<R / 8>(k)) << 4) + ((n >> 2) & 1) * 8;
  }
  static __device__ __forceinline__ uint32_t along(uint32_t base, int row, int ks, int g, const Phase& phase) {
    const int q = C::MX ? 2 * g + ks : ks * 4 + g;
    return base + row * 128 + ((C::PHASED ? phase.slot(q, row) : q ^ swizzle<C::MX>(row)) << 4);
  }

  __device__ __forceinline__ void init(const TileArgs& t, unsigned char* pool_, int m0, int n0, int wave_, int lane) {
    pool = pool_;
    wave = wave_;
    // (tiles begin at multiples of 8 rows, which leave a phase as it is, and so do the 16 and 32 rows from fragment to fragment and load to load)
    static_assert(!C::PHASED || (!C::A_T && C::B_NK && C::HALVES == 1 && !C::MX), "one matrix each, along the contraction");
    Phase pa, pb;
    if constexpr (C::PHASED) {
      pa.of(t.a[0], t.pitch_a);
      pb.of(t.b[0], t.pitch_b);
    }
    la.init(t.pitch_a, t.rows, m0, wave, lane, C::PHASED ? &pa : nullptr);
    lb.init(t.pitch_b, t.cols, n0, wave, lane, C::PHASED ? &pb : nullptr);
    const uint32_t base_a = flux::lds_address(pool), base_b = base_a + NA * C::A_BYTES;
    const int g = lane >> 4, i = lane & 15, wm = wave >> 1, wn = wave & 1, rb = wn * (C::SUBN / 2);
#pragma unroll
    for (int h = 0; h < A_HI; ++h)
#pragma unroll
      for (int v = 0; v < NAV; ++v) {
        if constexpr (C::A_T) a[h][v] = across<C::BM>(base_a + h * 65536u, wm * C::WTM + v * 16, i, g);
        else a[h][v] = along(base_a + h * 65536u, wm * C::WTM + i, v, g, pa);
      }
#pragma unroll
    for (int h = 0; h < B_HI; ++h)
#pragma unroll
      for (int v = 0; v < NBV; ++v) {
        if constexpr (C::B_NK) b[h][v] = along(base_b + h * 65536u, rb + i, v, g, pb);
        else b[h][v] = across<C::SUBN>(base_b + h * 65536u, rb + v * 16, i, g);
      }
    if constexpr (C::MX) {
      // wave w fetches 64 rows of each operand, 16 bytes (two slabs) a lane; of a gated B the lower half of the rows is gate's
      const int row = 64 * wave + lane, half = row / C::SUBN, col = row - half * C::SUBN;
      voff_s[0] = row < C::BM && m0 + row < t.rows ? (uint32_t)(m0 + row) * t.pitch_s : LdA::OUTSIDE;
      voff_s[1] = row < C::BN && n0 + col < t.cols ? (uint32_t)(n0 + col) * t.pitch_s : LdA::OUTSIDE;
      sc[0] = flux::lds_address(scales(0, 0)) + (wm * C::WTM + i) * 16 + 2 * g;
      sc[1] = flux::lds_address(scales(1, 0)) + (rb + i) * 16 + 2 * g;
    }
  }

  template <int OFF>
  static __device__ __forceinline__ void read(u32x4& f, uint32_t base) { asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f) : "v"(base), "n"(OFF)); }
  template <int OFF>
  static __device__ __forceinline__ void read(bf16x8& f, uint32_t base) {
    u32x4 v;
    read<OFF>(v, base);
    f = __builtin_bit_cast(bf16x8, v);
  }
  template <int OFF>
  static __device__ __forceinline__ u32x2 read_tr(uint32_t base) {
    u32x2 v;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(base), "n"(OFF));
    return v;
  }
  template <int OFF, int ROW_BYTES, int HI, int NV>
  static __device__ __forceinline__ void read_halves(FragHalves& f, const uint32_t (&base)[HI][NV], int v) {
    constexpr int UP = OFF + 4 * ROW_BYTES;
    f.lo = read_tr<OFF % 65536>(base[OFF / 65536][v]);
    f.hi = read_tr<UP % 65536>(base[UP / 65536][v]);
  }
  // fragment R, in the order the MFMAs want them, of k-step K out of A's slab SA / B's slab SB in LDS
  template <int SA, int SB, int K, int R>
  __device__ __forceinline__ void fetch() {
    constexpr bool IS_B = R == 0 || R > C::MI;
    constexpr int I = R == 0 ? 0 : (IS_B ? R - C::MI : R - 1);
    if constexpr (!IS_B) {
      if constexpr (C::A_T) {
        read_halves<SA * C::A_BYTES + K * 32 * C::BM * 2, C::BM * 2>(af[K][I], a, I);
      } else {
        constexpr int OFF = SA * C::A_BYTES + I * 16 * 128;
        read<OFF % 65536>(af[K][I], a[OFF / 65536][K]);
      }
    } else {
      constexpr int BASE = SB * C::B_BYTES + I / C::NIH * C::SUB_BYTES;
      if constexpr (C::B_NK) {
        constexpr int OFF = BASE + I % C::NIH * 16 * 128;
        read<OFF % 65536>(bf[K][I], b[OFF / 65536][K]);
      } else {
        read_halves<BASE + K * 32 * C::SUBN * 2, C::SUBN * 2>(bf[K][I], b, I % C::NIH);
      }
    }
  }
  // scales of fragment R (both k-steps) into set S % 2, S the slab's place in the unrolled loop; from_a, from_b: of its pair
  template <int S, int R>
  __device__ __forceinline__ void fetch_scale(uint32_t from_a, uint32_t from_b) {
    constexpr int OFF = R < C::MI ? R * 256 : ((R - C::MI) / C::NIH * C::SUBN + (R - C::MI) % C::NIH * 16) * 16;
    asm volatile("ds_read_u16 %0, %1 offset:%2" : "=v"(fs[S % 2][R]) : "v"(R < C::MI ? from_a : from_b), "n"(S % 2 * 8 + OFF));
  }

  __device__ __forceinline__ Slab slab(const TileArgs& t, bool is_b, int s) const {
    const bool there = s < KT;
    int k = k0 + s, seg = job;
    if constexpr (C::KIND == DX_NK || C::KIND == DX_KN) {
      seg = k >= t.seg_slabs ? 1 : 0;
      k -= seg * t.seg_slabs;
    }
    const uint32_t bytes = there ? (is_b ? t.bytes_b : t.bytes_a) : 0u;
    const auto rsrc = [&](const void* p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00027000); };
    if (!is_b) return Slab{rsrc(t.a[seg]), rsrc(t.a[seg]), k * C::BK};
    if constexpr (C::HALVES == 2) return Slab{rsrc(t.b[0]), rsrc(t.b[1]), k * C::BK};
    return Slab{rsrc(t.b[seg]), rsrc(t.b[seg]), k * C::BK};
  }
  __device__ __forceinline__ void load_b(const TileArgs& t, const Slab& w, int d, int place) const {
    const int half = d / LdB::INSTR;
    lb.load(d % LdB::INSTR, half ? w.r1 : w.r0, w.k, t.depth, slab_b(place) + half * C::SUB_BYTES);
  }
  // 4 bits: the scales of one operand, slabs 2 pair and 2 pair + 1
  __device__ __forceinline__ void load_scales(const TileArgs& t, int operand, int pair) const {
    const uint8_t* p = operand == 0 ? t.sa : t.sb[C::HALVES == 2 && 64 * wave >= C::SUBN ? 1 : 0];
    const int rows = operand == 0 ? t.rows : t.cols;
    const uint32_t at = (uint32_t)(k0 / 2 + pair) * 16u;
    const bool there = 2 * pair < KT && at < t.pitch_s;
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, there ? (int)((uint32_t)rows * t.pitch_s) : 0, 0x00027000);
    unsigned char* const to = 64 * wave < (operand ? C::BN : C::BM) ? scales(operand, pair % C::RS) + wave * 1024 : pool + C::POOL_BYTES - 1024;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (flux::lds_void_t*)to, 16, (int)voff_s[operand], (int)at, 0, 0);
  }

  // What step kt (place S of the unrolled loop; -1 ahead of the first) asks for from its barrier on: slab kt + NB, of A one
  // further where it leads, first the operand that the next barrier needs; and with it scales: of A, for the next two slabs,
  // beside an odd slab, of B beside an even one.
  struct Window { Slab a, b; int kt; };
  __device__ __forceinline__ Window window(const TileArgs& t, int kt) const { return Window{slab(t, false, kt + NA), slab(t, true, kt + NB), kt}; }
  __device__ __forceinline__ void load(const TileArgs& t, const Window& w, int d, int S) const {
    if (LS && d == L - 1) {
      if ((S + NB) % 2 == 1) load_scales(t, 0, (w.kt + NB + 1) / 2);
      else load_scales(t, 1, (w.kt + NB) / 2);
      return;
    }
    const bool is_a = A_LEADS ? d >= LB : d < LA;
    if (is_a) la.load(A_LEADS ? d - LB : d, w.a.r0, w.a.k, t.depth, slab_a((S + NA) % NA));
    else load_b(t, w.b, A_LEADS ? d : d - LA, (S + NB) % NB);
  }

  __device__ __forceinline__ void start(const TileArgs& t) {
    if (LS) load_scales(t, 0, 0);
#pragma unroll
    for (int j = 0; j < NB - 1; ++j) {
      const Slab sa = slab(t, false, j), sb = slab(t, true, j);
#pragma unroll
      for (int d = 0; d < LA; ++d) la.load(d, sa.r0, sa.k, t.depth, slab_a(j));
#pragma unroll
      for (int d = 0; d < LB; ++d) load_b(t, sb, d, j);
      if (LS) load_scales(t, (j + 1) % 2, (j + 1) / 2);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (A_LEADS) {
      const Slab sa = slab(t, false, NB - 1);
#pragma unroll
      for (int d = 0; d < LA; ++d) la.load(d, sa.r0, sa.k, t.depth, slab_a(NB - 1));
      __builtin_amdgcn_sched_barrier(0);
    }
    const Window w = window(t, -1);
#pragma unroll
    for (int d = 0; d < L0; ++d) load(t, w, d, U - 1);
    flux::wait_vm_at_most<(NB - 2) * L + LX + L0>();
    flux::barrier_keeping_loads_in_flight();
    flux::static_for<NF>([&](auto r) { fetch<0, 0, 0, decltype(r)::value>(); });
    flux::static_for<NS>([&](auto r) { fetch_scale<0, decltype(r)::value>(sc[0], sc[1]); });
    settle_reads(0, 0);
  }

  static __device__ __forceinline__ void settle(u32x4& f) { asm volatile("" : "+v"(f)); }
  static __device__ __forceinline__ void settle(bf16x8& f) { flux::frag_settle(f); }
  static __device__ __forceinline__ void settle(FragHalves& f) { flux::frag_settle(f); }
  __device__ __forceinline__ void settle_reads(int ks, int scale_set) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < C::MI; ++i) settle(af[ks][i]);
#pragma unroll
    for (int i = 0; i < C::NI; ++i) settle(bf[ks][i]);
#pragma unroll
    for (int i = 0; i < NS; ++i) asm volatile("" : "+v"(fs[scale_set][i]));
  }

  template <int S>
  __device__ __forceinline__ void step(const TileArgs& t, int kt, f32x4 (&acc)[C::MI][C::NI]) {
    kt = __builtin_amdgcn_readfirstlane(kt);
    const Window rest = window(t, kt - 1), first = window(t, kt);
    const uint32_t at = C::MX ? (uint32_t)((kt + 1) / 2 % C::RS) : 0u;                   // of the next slab's scales
    const uint32_t from_a = C::MX ? sc[0] + at * C::SC_A : 0u, from_b = C::MX ? sc[1] + at * C::SC_B : 0u;
    flux::static_for<KS>([&](auto ks_) {
      constexpr int ks = decltype(ks_)::value;
      constexpr bool LAST = ks == KS - 1;
      flux::static_for<G>([&](auto g_) {
        constexpr int g = decltype(g_)::value;
        // (the columns' fragment is held over a run of MFMAs; with the large tile every second run goes backwards: it begins with the
        // fragment that the run before ended with)
        constexpr int ni = g / C::MI, mi = G < 64 || ni % 2 == 0 ? g % C::MI : C::MI - 1 - g % C::MI;
        if constexpr (LAST && g == BAR_AT) {
          // slab kt + 1 is there (this wave's part, then everyone's); this slab has been read by all
          flux::wait_vm_at_most<(NB - 2) * L + LX>();
          flux::barrier_keeping_loads_in_flight();
        }
        if constexpr (C::MX) mfma_scaled<ks>(acc[mi][ni], bf[ks][ni], af[ks][mi], fs[S % 2][C::MI + ni], fs[S % 2][mi]);
        else flux::mfma_in_place(acc[mi][ni], flux::frag_value(bf[ks][ni]), flux::frag_value(af[ks][mi]));
        constexpr int d0 = loads_before(LAST ? g : G + g), d1 = loads_before((LAST ? g : G + g) + 1);
#pragma unroll
        for (int d = d0; d < d1; ++d) {
          if constexpr (LAST) load(t, first, d, S);
          else load(t, rest, d, S + U - 1);
        }
        constexpr int ALL = NF + (LAST ? NS : 0);
        constexpr int r0 = reads_before(g, LAST ? BAR_AT : 0, ALL), r1 = reads_before(g + 1, LAST ? BAR_AT : 0, ALL);
        flux::static_for<r1 - r0>([&](auto r_) {
          constexpr int r = r0 + decltype(r_)::value;
          if constexpr (r >= NF) fetch_scale<S + 1, r - NF>(from_a, from_b);
          else if constexpr (LAST) fetch<(S + 1) % NA, (S + 1) % NB, 0, r>();
          else fetch<S % NA, S % NB, ks + 1, r>();
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      settle_reads(1 - ks, (S + 1) % 2);
    });
  }

  __device__ __forceinline__ void run(const TileArgs& t, f32x4 (&acc)[C::MI][C::NI]) {
    int kt = 0;
    for (; kt + U <= KT; kt += U)
      flux::static_for<U>([&](auto s_) { step<decltype(s_)::value>(t, kt + decltype(s_)::value, acc); });
    flux::static_for<U - 1>([&](auto s_) {
      constexpr int S = decltype(s_)::value;
      if (kt + S < KT) step<S>(t, kt + S, acc);
    });
    flux::mfma_results_settle<C::MI, C::NI>(acc);
  }
};

// ---- results ---------------------------------------------------------------------------------------------------
// Nothing passes through LDS.  The columns' fragment goes first into the MFMAs, so a lane holds four consecutive columns of row
// lane % 16: 16 bytes of an fp32 result.  For bf16 one swap of neighbouring 16-lane rows between two blocks of columns makes that eight.
// Either way four lanes have 64 bytes of a row side by side, a piece.  Of two pieces that are neighbours, lanes 8..15 of every 16 of the one
// change places with lanes 0..7 of the other, and either store is eight rows by 128 bytes.
__device__ __forceinline__ void store16(void* p, bool stream, const u32x4& v) {
  // (written out: of two stores of the same value to the same place the compiler makes one, without the hint; and with the two wait states
  // that a write to the registers of a 16-byte store wants, which the compiler does not see here)
  if (stream) asm volatile("global_store_dwordx4 %0, %1, off nt\n\ts_nop 1" : : "v"(p), "v"(v) : "memory");
  else *(flux::global_u32x4*)p = v;
}
// The pieces x and y, which lie side by side from byte `at` of the wave's rows row0 .. row0 + 15 on; in_piece: where the lane's 16 bytes lie.
template <bool EDGE>
__device__ __forceinline__ void store_pair(const TileArgs& t, void* out, int size, const u32x4& x, const u32x4& y, int row0, int col0, int lane, int in_piece) {
  u32x4 a, b;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    constexpr int ROR8 = 0x128;
    a[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)x[e], (int)y[e], ROR8, 0xf, 0xc, false);
    b[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)y[e], (int)x[e], ROR8, 0xf, 0x3, false);
  }
  const int row = row0 + (lane & 7), off = col0 * size + (lane & 8) * 8 + in_piece;
  const long long pitch = t.ld * size;
  char* const to = static_cast<char*>(out) + row * pitch + off;
  const bool in = !EDGE || off < t.cols * size;
  if (in && (!EDGE || row < t.rows)) store16(to, t.stream, a);
  if (in && (!EDGE || row + 8 < t.rows)) store16(to + 8 * pitch, t.stream, b);
}
template <bool EDGE>
__device__ __forceinline__ void store_piece(const TileArgs& t, void* out, int size, const u32x4& x, int row0, int col0, int lane, int in_piece) {
  const int row = row0 + (lane & 15), off = col0 * size + in_piece;
  if (!EDGE || (row < t.rows && off < t.cols * size)) store16(static_cast<char*>(out) + row * (t.ld * size) + off, t.stream, x);
}
__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) {
  return u32x4{flux::pack_bf16x2(v[0], v[1]), flux::pack_bf16x2(v[2], v[3]), flux::pack_bf16x2(v[4], v[5]), flux::pack_bf16x2(v[6], v[7])};
}
// Columns 32 n' + 16 (g % 2) + 8 (g / 2) .. + 7 of two neighbouring blocks of columns, g = lane / 16.
__device__ __forceinline__ void eight_columns(const f32x4& x, const f32x4& y, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[e]), __float_as_uint(y[e]), false, false);
    v[e] = __uint_as_float(r[0]);
    v[4 + e] = __uint_as_float(r[1]);
  }
}

// v = act(v) * u
template <bool FINE, int N>
__device__ __forceinline__ void gate(int which, float (&v)[N], const float (&u)[N]) {
  if (which == FLUX_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = act<FLUX_ACT_SILU, FINE>(v[e]) * u[e];
  } else if (which == FLUX_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = act<FLUX_ACT_GELU, FINE>(v[e]) * u[e];
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = act<FLUX_ACT_GELU_TANH, FINE>(v[e]) * u[e];
  }
}

// 16 rows of the wave's part of the tile, out of its accumulators.  SCALED: the results are the sums times a factor, and dX may have an addend elsewhere than in its
// place.  (A kernel of its own: in the gated block's the branches alone cost dX of 8192x8192 over two times 3584 662 us to 673.)
template <class C, bool SCALED>
__device__ __forceinline__ void finish_rows16(const TileArgs& t, int job, f32x4 (&acc)[C::NI], int row0, int col0, int lane) {
  static_assert(!SCALED || C::KIND == DX_KN || C::KIND == DW, "");
  constexpr bool ADDEND = SCALED && C::KIND == DX_KN;
  if constexpr (SCALED) {
    const float by = *t.factor;
    // (no number, as the mean over no row has it: what no row added to stays 0)
    if (__builtin_fabsf(by) < __builtin_inff()) {
#pragma unroll
      for (int n = 0; n < C::NI; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][e] *= by;
    } else {
#pragma unroll
      for (int n = 0; n < C::NI; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][e] = acc[n][e] == 0.f ? 0.f : acc[n][e] * by;
    }
  }
  const int g = lane >> 4, row = row0 + (lane & 15), in_bf16 = (g & 1) * 32 + (g >> 1) * 16;
  const auto bf16 = [&](void* out, int col, const u32x4 (&p)[C::NIH / 2]) {
    if constexpr (C::NIH == 2) {
      store_piece<C::EDGE>(t, out, 2, p[0], row0, col, lane, in_bf16);
    } else {
#pragma unroll
      for (int n = 0; n < C::NIH / 2; n += 2) store_pair<C::EDGE>(t, out, 2, p[n], p[n + 1], row0, col + n * 32, lane, in_bf16);
    }
  };
  if constexpr (C::HALVES == 2) {
    if (t.g != nullptr) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 p[C::NIH / 2];
#pragma unroll
        for (int n = 0; n < C::NIH; n += 2) {
          float v[8];
          eight_columns(acc[h * C::NIH + n], acc[h * C::NIH + n + 1], v);
          p[n / 2] = pack8(v);
        }
        bf16(h ? t.u : t.g, col0, p);
      }
    }
  }
  // What is added to, asked for before the first of it is used (it may lie where the results go, so no load would pass a store).
  f32x4 old[C::HALVES == 2 ? 1 : C::NI];
  if constexpr (C::HALVES == 1) {
    const bool in_f32 = ADDEND ? t.addend != nullptr : t.accumulate && t.out_f32;
    if (in_f32) {
      // four columns a block
      const float* const from = (ADDEND ? t.addend : static_cast<const float*>(t.out[job])) + row * t.ld;
#pragma unroll
      for (int n = 0; n < C::NI; ++n) {
        const int col = col0 + n * 16 + 4 * g;
        if (!C::EDGE || (row < t.rows && col < t.cols)) old[n] = *reinterpret_cast<const f32x4*>(from + col);
      }
    } else if (!ADDEND && t.accumulate) {
      // eight columns of two blocks, in bf16
#pragma unroll
      for (int n = 0; n < C::NI; n += 2) {
        const int col = col0 + n * 16 + 16 * (g & 1) + 8 * (g >> 1);
        if (!C::EDGE || (row < t.rows && col < t.cols))
          old[n] = __builtin_bit_cast(f32x4, *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(t.out[job]) + row * t.ld + col));
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (in_f32) {
#pragma unroll
      for (int n = 0; n < C::NI; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) old[n][e] += acc[n][e];
    }
  }
  if (!t.out_f32) {
    u32x4 p[C::NIH / 2];
#pragma unroll
    for (int n = 0; n < C::NIH; n += 2) {
      float v[8];
      if constexpr (C::HALVES == 2) {
        float u[8];
        eight_columns(acc[n], acc[n + 1], v);
        eight_columns(acc[C::NIH + n], acc[C::NIH + n + 1], u);
        gate<false>(t.act, v, u);
      } else if (ADDEND && t.addend != nullptr) {
        eight_columns(old[n], old[n + 1], v);
      } else {
        eight_columns(acc[n], acc[n + 1], v);
        if (!ADDEND && t.accumulate) {
          const bf16x8 o = __builtin_bit_cast(bf16x8, old[n]);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += (float)o[e];
        }
      }
      p[n / 2] = pack8(v);
    }
    bf16(t.out[job], col0, p);
  } else {
#pragma unroll
    for (int n = 0; n < C::NIH; n += 2) {
      u32x4 p[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[4] = {acc[n + h][0], acc[n + h][1], acc[n + h][2], acc[n + h][3]};
        if constexpr (C::HALVES == 2) {
          const f32x4& y = acc[C::NIH + n + h];
          const float u[4] = {y[0], y[1], y[2], y[3]};
          gate<true>(t.act, v, u);
        } else if (ADDEND ? t.addend != nullptr : t.accumulate != 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = old[n + h][e];
        }
        p[h] = __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
      }
      store_pair<C::EDGE>(t, t.out[job], 4, p[0], p[1], row0, col0 + n * 16, lane, g * 16);
    }
  }
}

// ---- tiles whose contraction is cut ------------------------------------------------------------------------------
// Every part leaves its sums in memory and counts itself in; when all have, each part adds up a share of the tile, 16-row blocks in
// turn, in the parts' order whoever does it, and finishes those rows.  Nobody waits for long: a part that has waited 100 us for
// the others (they may not have been given a compute unit yet) leaves its share to whoever comes last.  The tile's word holds, in
// this order, how many have arrived, how many are done with the word, and a bit for every part that has left.  Arriving
// and leaving are one atomic addition each, so that the last to arrive either finds the bit, or the leaver finds that all have arrived.
//
// Sums are stored and read past this die's L2 (SC1): "my stores are acknowledged" before counting in is all that the others need.
//
// us, joined by a second kernel / here: gated 200x3584x8192 [N,K] 42.0 / 41.5, 8x3584x8192 [K,N] 29.1 / 26.7, 4 bits 512x6144x12288
// 172.6 / 165, both weights' gradients 1024x8192x2048 82.4 / 74.8.
constexpr int MAX_PARTS = 16, COUNTER_STRIDE = 16;             // (words: 64 bytes)
constexpr uint32_t ARRIVED = 1u, DONE = 1u << 8, LEFT = 1u << 16;
constexpr unsigned long long PATIENCE_TICKS = 10000;           // of 10 ns

// Which parts' shares this workgroup finishes, as bits.  One thread.
__device__ __forceinline__ uint32_t count_in(uint32_t* word, int part, int parts, bool has_share) {
  const auto add = [&](uint32_t v) { return __hip_atomic_fetch_add(word, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
  const uint32_t all = (uint32_t)parts;
  const auto done = [&](uint32_t before) {                     // the last one done puts the word back
    if ((before >> 8 & 255u) == all - 1u) __hip_atomic_store(word, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  uint32_t before = add(ARRIVED);
  const uint32_t mine = has_share ? 1u << part : 0u;
  if ((before & 255u) == all - 1u) {
    done(add(DONE));
    return mine | before >> 16;
  }
  if (has_share) {
    const unsigned long long until = wall_clock64() + PATIENCE_TICKS;
    while ((__hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & 255u) != all) {
      if (wall_clock64() >= until) {
        before = add(DONE + (LEFT << part));
        done(before);
        return (before & 255u) == all ? mine : 0u;
      }
      __builtin_amdgcn_s_sleep(4);
    }
  }
  done(add(DONE));
  return mine;
}

template <class C, class F>
__device__ __forceinline__ void finish_cut(const TileArgs& t, unsigned char* pool, f32x4 (&acc)[C::MI][C::NI], int cut, int part,
                                           int job, int m0, int n0, int lane, int wave, F& finish) {
  constexpr int SC1 = 16, BYTES = C::BM * C::BN * 4;
  const int tid = wave * 64 + lane, row0 = m0 + (wave >> 1) * C::WTM;
  float* const sums = t.partial + (size_t)cut * t.parts * (C::BM * C::BN);
  const auto rsrc = [&](int p) { return __builtin_amdgcn_make_buffer_rsrc(sums + (size_t)p * (C::BM * C::BN), 0, BYTES, 0x00027000); };
  // a vector is four columns of one row; one that lies past the last row is neither stored nor read (an offset past the records)
  const int below = C::EDGE ? t.rows - row0 - (lane & 15) : C::BM;
  const __amdgpu_buffer_rsrc_t own = rsrc(part);
#pragma unroll
  for (int mi = 0; mi < C::MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < C::NI; ++ni) {
      asm volatile("" : "+a"(acc[mi][ni]));            // (stored from where it is)
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[mi][ni]), own, mi * 16 < below ? ((mi * C::NI + ni) * 256 + tid) * 16 : BYTES, 0, SC1);
    }
  __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): acknowledged
  __syncthreads();
  uint32_t* const shared = reinterpret_cast<uint32_t*>(pool);
  if (tid == 0) *shared = count_in(t.counters + cut * COUNTER_STRIDE, part, t.parts, part < C::MI);
  __syncthreads();
  const uint32_t shares = (uint32_t)__builtin_amdgcn_readfirstlane((int)*shared);
#pragma unroll 1
  for (int mi = 0; mi < C::MI; ++mi) {
    if (!(shares >> mi % t.parts & 1u)) continue;      // (uniform)
    f32x4 sum[C::NI];
#pragma unroll
    for (int ni = 0; ni < C::NI; ++ni) sum[ni] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr int P = 16 / C::NI;                      // parts whose vectors are asked for before the first is used
#pragma unroll 1
    for (int p0 = 0; p0 < t.parts; p0 += P) {
      u32x4 v[P][C::NI];
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const bool there = p0 + p < t.parts;           // (one past the last: zeros)
        const __amdgpu_buffer_rsrc_t r = rsrc(there ? p0 + p : 0);
#pragma unroll
        for (int ni = 0; ni < C::NI; ++ni)
          v[p][ni] = __builtin_amdgcn_raw_buffer_load_b128(r, there && mi * 16 < below ? ((mi * C::NI + ni) * 256 + tid) * 16 : BYTES, 0, SC1);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int ni = 0; ni < C::NI; ++ni) sum[ni] += __builtin_bit_cast(f32x4, v[p][ni]);
    }
    finish(job, sum, row0 + mi * 16, n0 + (wave & 1) * (C::SUBN / 2), lane);
  }
}

// Workgroups are dealt round-robin to the eight dies: die d takes the d-th run of consecutive blocks, so that neighbouring tiles
// share panels in one L2.
__device__ __forceinline__ int by_die(int b, int n) {
  const int die = b % 8, each = n / 8, more = n % 8;
  return die * each + (die < more ? die : more) + b / 8;
}

// One workgroup's tile or part of one.  finish(job, sums, row, column, lane) takes 16 rows of a wave's part of the result (see finish_rows16);
// finish.ask(t, m0) asks for what it needs of the tile's rows ahead of the main loop, finish.keep(pool) leaves it in LDS behind it.
template <class C, class F>
__device__ __forceinline__ void tile_body(const TileArgs& t, unsigned char* pool, F& finish) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool is_cut = (int)blockIdx.x >= t.full_tiles;
  int b, cut = 0, part = 0, job = 0;
  if (is_cut) {
    const int r = by_die((int)blockIdx.x - t.full_tiles, t.cut_tiles * t.parts);
    part = r / t.cut_tiles;
    cut = r - part * t.cut_tiles;
    b = t.full_tiles + cut;
  } else {
    b = by_die((int)blockIdx.x, t.full_tiles);
  }
  if constexpr (C::KIND == DW) {
    job = b >= t.tiles_m * t.tiles_n ? 1 : 0;
    b -= job * (t.tiles_m * t.tiles_n);
  }
  const int band = b / (t.band * t.tiles_n), h = min(t.band, t.tiles_m - band * t.band);
  const int r = b - band * t.band * t.tiles_n;
  const int m0 = (band * t.band + r % h) * C::BM, n0 = r / h * C::SUBN;

  finish.ask(t, m0);
  Pipe<C> pipe;
  pipe.job = job;
  pipe.k0 = part * t.part_slabs;
  pipe.KT = is_cut ? min(t.part_slabs, t.slabs - pipe.k0) : t.slabs;
  pipe.init(t, pool, m0, n0, wave, lane);
  f32x4 acc[C::MI][C::NI];
#pragma unroll
  for (int mi = 0; mi < C::MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < C::NI; ++ni)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[mi][ni][e] = 0.f;
  pipe.start(t);
  pipe.run(t, acc);
  flux::wait_vm_at_most<0>();            // nothing of this wave is left in flight towards LDS that it gives up
  finish.keep(pool);
  if (is_cut) {
    __syncthreads();                     // (a word of LDS is used again)
    finish_cut<C>(t, pool, acc, cut, part, job, m0, n0, lane, wave, finish);
    return;
  }
  // (A loop in the code too, its block of accumulators picked by a branch: unrolled, the activations of a gated tile are over 100 KB of
  // instructions.)
#pragma unroll 1
  for (int mi = 0; mi < C::MI; ++mi) {
    f32x4 x[C::NI];
    flux::static_for<C::MI>([&](auto k_) {
      constexpr int k = decltype(k_)::value;
      if (mi == k) {
#pragma unroll
        for (int ni = 0; ni < C::NI; ++ni) {
          asm volatile("" : "+a"(acc[k][ni]));       // (it stays in its accumulation registers until here)
          x[ni] = acc[k][ni];
        }
      }
    });
    finish(job, x, m0 + (wave >> 1) * C::WTM + mi * 16, n0 + (wave & 1) * (C::SUBN / 2), lane);
  }
}

template <class C, bool SCALED>
struct Results {
  const TileArgs& t;
  __device__ __forceinline__ void ask(const TileArgs&, int) {}
  __device__ __forceinline__ void keep(unsigned char*) {}
  __device__ __forceinline__ void operator()(int job, f32x4 (&x)[C::NI], int row0, int col0, int lane) const { finish_rows16<C, SCALED>(t, job, x, row0, col0, lane); }
};

template <class C>
__global__ void __launch_bounds__(C::NT, C::OCC) tile_kernel(const TileArgs t) {
  __shared__ __attribute__((aligned(1024))) unsigned char pool[C::POOL_BYTES];
  Results<C, false> results{t};
  tile_body<C>(t, pool, results);
}

template <class C>
__global__ void __launch_bounds__(C::NT, C::OCC) scaled_kernel(const TileArgs t) {
  __shared__ __attribute__((aligned(1024))) unsigned char pool[C::POOL_BYTES];
  Results<C, true> results{t};
  tile_body<C>(t, pool, results);
}

}  // namespace flux_ffn
