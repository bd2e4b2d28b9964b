// Building blocks of the matrix-core kernels for gfx950: square tiles of one
// workgroup, the LDS ring that feeds them, direct global -> LDS loads, operand
// reads and the 16 x 16 x 32 matrix instruction.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tmk {
namespace tile {

// K elements per ring stage of the 8-wave (256) tile: rows of 128 bytes.
constexpr int kPingPongBK = 64;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

// Tile T x T computed by NW wave64s in a WGM x WGN grid (2 x 4, 2 x 2, or a
// single wave for the 32 tile); each wave owns TWM x TWN of the output as
// FM x FN blocks of 16 x 16, each accumulated by v_mfma_f32_16x16x32_bf16 (a
// 16 x 16 fp32 block, 4 registers per lane, 32 K values per instruction).
// The smaller tiles' Gram and polynomial add NP producer waves that only
// issue the ring's DMA (mainloop_pc); they leave after the main loop, so the
// epilogues run on the NT threads of the NW compute waves.  (The update's
// smaller tiles keep the DMA in their compute waves: producer waves made
// them slower.)
template <int T>
struct Tile {
  static constexpr int NW = T == 256 ? 8 : (T == 32 ? 1 : 4);   // 2 waves per SIMD for 256
  static constexpr int WGM = NW == 1 ? 1 : 2, WGN = NW / WGM;
  static constexpr int NT = 64 * NW;            // threads of the compute waves
  static constexpr int NP = T == 256 ? 0 : (T == 32 ? 1 : 2);   // producer waves
  static constexpr int NTT = 64 * (NW + NP);    // threads per workgroup
  static constexpr int TWM = T / WGM, TWN = T / WGN;
  static constexpr int FM = TWM / 16, FN = TWN / 16;
};

// The fp32 accumulators of one wave: block (fm, fn), lane L, element v holds
// output row 16 fm + 4 (L / 16) + v, column 16 fn + L % 16 of the wave's part
// (the operands fed the other way round, as the update does, give the
// transposed block: row 16 fm + L % 16, columns 16 fn + 4 (L / 16) + v).
template <int T>
using AccT = f32x4_t[Tile<T>::FM][Tile<T>::FN];

// LDS ring of one main loop: NSTAGE stages of BK K-elements of both operands
// (the 128 tile's 32-wide ring is 3 deep, 48 KB, so that three blocks share a
// compute unit in many-block launches).
// A K-contiguous operand row of a stage is RB = 2 BK bytes, stored as CPR
// 16-byte chunks; logical chunk c of row r lives at chunk c ^ ((r / RPB) %
// CPR), RPB being the rows that span the 64 banks once, so that the 16 lanes
// of a ds_read_b128 pass (16 rows, one chunk) hit every bank once.
template <int T, int BK>
struct Ring {
  static constexpr int NSTAGE = BK == 32 ? (T == 128 ? 3 : 4) : (T == 256 ? 2 : 3);
  static constexpr int RB = 2 * BK;
  static constexpr int CPR = RB / 16;
  static constexpr int RPB = 256 / RB;
  static constexpr int A_BYTES = T * RB;         // one operand stage
  static constexpr int STAGE = 2 * A_BYTES;
  // the 256 tile keeps five operand slots of A_BYTES (mainloop_pp_kc5)
  static constexpr int LDS = T == 256 ? 5 * A_BYTES : NSTAGE * STAGE;
  static constexpr int DMA_OP = T * BK / 512 / Tile<T>::NW;   // 1 KB DMAs per wave per operand
  static constexpr int PER_STAGE = 2 * DMA_OP;
  static_assert(T * BK % (512 * Tile<T>::NW) == 0, "whole DMA instructions per wave");
  static_assert(LDS <= 160 * 1024, "gfx950 LDS is 160 KB per workgroup");
};

__device__ inline float bf2f(uint16_t v) { return __uint_as_float(uint32_t(v) << 16); }
__device__ inline uint16_t f2bf(float f) {     // v_cvt_pk_bf16_f32: round to nearest even
  __bf16 h = static_cast<__bf16>(f);
  return __builtin_bit_cast(uint16_t, h);
}
__device__ inline float h2f(uint16_t v) { return float(__builtin_bit_cast(_Float16, v)); }
__device__ inline uint16_t f2h(float f) {      // v_cvt_f16_f32: round to nearest even
  return __builtin_bit_cast(uint16_t, static_cast<_Float16>(f));
}

__device__ inline uint32_t lds_addr(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p));
}

// One 16-byte-per-lane direct global -> LDS load: lane i writes LDS bytes
// [lds + 16 i, lds + 16 i + 16).  Issued through inline assembly so that the
// compiler does not serialise the LDS reads of other stages behind it; the
// ring's own s_waitcnt/s_barrier pairs order it.
__device__ inline void dma16(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, %1\n"
      :
      : "v"(voff), "s"(base), "s"(lds)
      : "memory", "m0");
}

// Wait until at most `pending` DMA instructions of this wave are in flight and
// all of its LDS reads are done, then join the workgroup barrier.  The LDS
// wait goes through the builtin so that the compiler knows the reads are
// complete; the DMA wait and the barrier are assembly, since the compiler does
// not see the DMA loads.
template <int PENDING>
__device__ inline void ring_sync_dma() {
  if constexpr (PENDING == 0) asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  else if constexpr (PENDING == 2) asm volatile("s_waitcnt vmcnt(2)\n\ts_barrier" ::: "memory");
  else if constexpr (PENDING == 4) asm volatile("s_waitcnt vmcnt(4)\n\ts_barrier" ::: "memory");
  else if constexpr (PENDING == 6) asm volatile("s_waitcnt vmcnt(6)\n\ts_barrier" ::: "memory");
  else if constexpr (PENDING == 8) asm volatile("s_waitcnt vmcnt(8)\n\ts_barrier" ::: "memory");
  else if constexpr (PENDING == 12) asm volatile("s_waitcnt vmcnt(12)\n\ts_barrier" ::: "memory");
  else if constexpr (PENDING == 16) asm volatile("s_waitcnt vmcnt(16)\n\ts_barrier" ::: "memory");
  else if constexpr (PENDING == 24) asm volatile("s_waitcnt vmcnt(24)\n\ts_barrier" ::: "memory");
  else if constexpr (PENDING == 32) asm volatile("s_waitcnt vmcnt(32)\n\ts_barrier" ::: "memory");
  else static_assert(PENDING == 0, "unsupported in-flight count");
}

template <int PENDING>
__device__ inline void ring_sync() {
  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0), vmcnt/expcnt untouched
  ring_sync_dma<PENDING>();
}

// Wait for all but `stages` of this wave's stages in flight, then barrier.
// (MAXS: the most stages a caller can leave in flight; larger counts are not
// instantiated, since vmcnt holds at most 63.)
template <int PS, int MAXS>
__device__ inline void ring_wait(int stages) {
  static_assert(MAXS * PS <= 63, "in-flight count beyond vmcnt");
  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0), vmcnt/expcnt untouched
  if constexpr (MAXS >= 3) {
    if (stages >= 3) { ring_sync_dma<3 * PS>(); return; }
  }
  if constexpr (MAXS >= 2) {
    if (stages == 2) { ring_sync_dma<2 * PS>(); return; }
  }
  if constexpr (MAXS >= 1) {
    if (stages == 1) { ring_sync_dma<PS>(); return; }
  }
  ring_sync_dma<0>();
}

// DMA-only wait (no barrier): at most PENDING DMA instructions of this wave
// still in flight.
template <int PENDING>
__device__ inline void dma_wait() {
  if constexpr (PENDING == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  else if constexpr (PENDING == 2) asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
  else if constexpr (PENDING == 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
  else if constexpr (PENDING == 6) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
  else if constexpr (PENDING == 8) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
  else if constexpr (PENDING == 12) asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
  else if constexpr (PENDING == 16) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
  else if constexpr (PENDING == 24) asm volatile("s_waitcnt vmcnt(24)" ::: "memory");
  else static_assert(PENDING == 0, "unsupported in-flight count");
}

// DMA-only wait for all but `stages` stages of PS instructions (stages <= MAXS).
template <int PS, int MAXS>
__device__ inline void dma_wait_upto(int stages) {
  static_assert(MAXS * PS <= 63, "in-flight count beyond vmcnt");
  if constexpr (MAXS >= 2) {
    if (stages >= 2) { dma_wait<2 * PS>(); return; }
  }
  if constexpr (MAXS >= 1) {
    if (stages == 1) { dma_wait<PS>(); return; }
  }
  dma_wait<0>();
}

__device__ inline void barrier_pinned() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// ---------------------------------------------------------------- DMA issue
// The per-lane offset of a DMA is 32 bits: the base address of every call
// starts at the instruction's first row, so an offset spans the rows of one
// wave's instructions (at most 256) of a row of at most 65536 + 7 elements.
//
// K-contiguous operand: T rows x BK bf16 in the swizzled row layout of Ring.
// One instruction fills 1 KB = 64 / CPR rows; lane i writes chunk i % CPR of
// its row, i.e. it loads logical chunk (i % CPR) ^ swizzle.  Split over NI
// issuing waves (w = 0 .. NI - 1): instruction q of wave w fills 1 KB block
// w + NI q of the operand stage.  The rows of that block's first row and the
// K offset go into the (uniform) base address, so the per-lane offset only
// holds the lane's row within the instructions of wave w and its swizzled
// chunk, which the compiler can keep in one or two registers.
template <int T, int BK, int NI>
__device__ inline void dma_kc_w(const uint16_t* src, int64_t ld, int k0, uint32_t lds, int q, int w) {
  using R = Ring<T, BK>;
  constexpr int RPI = 64 / R::CPR;
  const int lane = threadIdx.x & 63;
  const int j = w + NI * q;
  const int rq = NI * q * RPI;                  // uniform row offset of the instruction
  const int rl = w * RPI + lane / R::CPR;       // row within it
  const int r = rq + rl;
  const int c = (lane % R::CPR) ^ ((r / R::RPB) % R::CPR);
  const uint16_t* base = src + int64_t(rq) * ld + k0;
  const uint32_t voff = uint32_t((int64_t(rl) * ld + c * 8) * 2);
  dma16(base, voff, __builtin_amdgcn_readfirstlane(lds + uint32_t(j) * 1024u));
}

// All NW compute waves issuing: instruction q of wave w fills block w + NW q.
template <int T, int BK>
__device__ inline void dma_kc(const uint16_t* src, int64_t ld, int k0, uint32_t lds, int q) {
  dma_kc_w<T, BK, Tile<T>::NW>(src, ld, k0, lds, q, int(threadIdx.x >> 6));
}

template <int T, int BK>
__device__ inline void issue_kc(const uint16_t* src, int64_t ld, int k0, uint32_t lds) {
#pragma unroll
  for (int q = 0; q < Ring<T, BK>::DMA_OP; ++q) dma_kc<T, BK>(src, ld, k0, lds, q);
}

// The transposing reads of a 16 x 32 (K) operand block touch, per half wave,
// 8 rows (bits 0, 1 and 3 of the row vary) at one logical chunk: the swizzle
// sends them to 8 different 32-byte bank groups (with 4 chunks per row, the
// 64 tile, row parity supplies the third bit).
template <int T>
__device__ inline int swz_y(int r) {
  return T >= 128 ? ((r & 3) | (((r >> 3) & 1) << 2)) : (((r >> 1) & 1) | (((r >> 3) & 1) << 1));
}

// Row-major operand (the update's Y): BK rows (K) x T columns, row = 2T bytes,
// 32-byte chunks swizzled per row.  Split over NI issuing waves as dma_kc_w;
// the instruction's first row (K offset k0 + its rows) goes into the 64-bit
// base address, so the 32-bit per-lane offset spans a few rows only,
// whatever the matrix size.
template <int T, int BK, int NI>
__device__ inline void dma_rm_w(const uint16_t* src, int64_t ld, int k0, uint32_t lds, int q, int w) {
  constexpr int ROWB = 2 * T;
  constexpr int LPR = ROWB / 16;          // lanes per row
  constexpr int RPI = 1024 / ROWB;        // rows per instruction
  const int lane = threadIdx.x & 63;
  const int j = w + NI * q;
  const int rq = NI * q * RPI;
  const int rl = w * RPI + lane / LPR;
  const int p16 = lane % LPR;
  const int c = (p16 >> 1) ^ swz_y<T>(rq + rl);
  const uint16_t* base = src + int64_t(k0 + rq) * ld;
  const uint32_t voff = uint32_t((int64_t(rl) * ld + c * 16 + (p16 & 1) * 8) * 2);
  dma16(base, voff, __builtin_amdgcn_readfirstlane(lds + uint32_t(j) * 1024u));
}

template <int T, int BK>
__device__ inline void dma_rm(const uint16_t* src, int64_t ld, int k0, uint32_t lds, int q) {
  dma_rm_w<T, BK, Tile<T>::NW>(src, ld, k0, lds, q, int(threadIdx.x >> 6));
}

// ---------------------------------------------------------------- compute
template <int T>
struct Frags {
  uint4 a[Tile<T>::FM], b[Tile<T>::FN];
};

template <int T>
__device__ inline void zero_acc(AccT<T>& acc) {
#pragma unroll
  for (int fm = 0; fm < Tile<T>::FM; ++fm)
#pragma unroll
    for (int fn = 0; fn < Tile<T>::FN; ++fn) acc[fm][fn] = f32x4_t{0.f, 0.f, 0.f, 0.f};
}

// MFMA operands of the 32-wide K slice s of one stage.  K-contiguous operand,
// block of 16 rows: lane L loads the 16 bytes (8 K values) at K offset 32 s +
// 8 (L / 16) of row L % 16; the rows of a wave's blocks are 16 apart, which
// keeps the chunk swizzle, so one address serves all of them.  Row-major
// operand (the update's Y, RM): lane L needs the 8 K values 32 s + 8 (L / 16)
// .. + 7 of column L % 16 of the block, gathered by two transposing reads of
// four rows each: lane q of a 16-lane group addresses row kb + q / 4, columns
// 4 (q % 4) .. + 3 of the block, and receives rows kb .. kb + 3 of column q.
template <int T, int BK>
__device__ inline void load_frags_a(Frags<T>& fr, const char* sa, int s, int wm) {
  using R = Ring<T, BK>;
  const int lane = threadIdx.x & 63;
  const int lr = lane & 15, g = lane >> 4;
  const int c = 4 * s + g;
  const int r0 = wm * Tile<T>::TWM + lr;
  const char* p = sa + r0 * R::RB + 16 * (c ^ ((r0 / R::RPB) % R::CPR));
#pragma unroll
  for (int f = 0; f < Tile<T>::FM; ++f) fr.a[f] = *reinterpret_cast<const uint4*>(p + f * 16 * R::RB);
}

template <int T, bool RM, int BK>
__device__ inline void load_frags_b(Frags<T>& fr, const char* sb, int s, int wn) {
  constexpr int FN = Tile<T>::FN;
  using R = Ring<T, BK>;
  const int lane = threadIdx.x & 63;
  const int lr = lane & 15, g = lane >> 4;
  const int c = 4 * s + g;
  if constexpr (!RM) {
    const int r0 = wn * Tile<T>::TWN + lr;
    const char* p = sb + r0 * R::RB + 16 * (c ^ ((r0 / R::RPB) % R::CPR));
#pragma unroll
    for (int f = 0; f < FN; ++f) fr.b[f] = *reinterpret_cast<const uint4*>(p + f * 16 * R::RB);
  } else {
    // Column block f of wave wn is block f WGN + wn of the tile (the waves'
    // blocks interleave), i.e. 32-byte chunk f WGN + wn of a stage row.  Row of
    // the first read within the slice; the second read's row (+ 4) and every
    // slice share its swizzle (bits 0, 1 and 3 of the row).  chunk ^ sw =
    // (f ^ hi) WGN + (wn ^ lo) with hi = sw / WGN, lo = sw % WGN.
    constexpr int WGN = Tile<T>::WGN;
    const int rl = 8 * g + (lr >> 2);
    const int sw = swz_y<T>(rl);
    const int hi = sw / WGN;
    const char* base = sb + (32 * s + rl) * (2 * T) + 8 * (lr & 3) + 32 * (wn ^ (sw % WGN));
    // when hi is 0 or 1 (sw < 2 WGN), f ^ hi = f + hi for even f and f - hi for
    // odd f: two addresses and immediate offsets serve every block
    constexpr bool two = (T >= 128 ? 8 : 4) <= 2 * WGN;   // largest sw + 1 <= 2 WGN
    const char* pe = base + 32 * WGN * hi;
    const char* po = base - 32 * WGN * hi;
#pragma unroll
    for (int f = 0; f < FN; ++f) {
      const char* p = two ? ((f & 1) ? po : pe) + 32 * WGN * f : base + 32 * WGN * (f ^ hi);
      s16x4_t v[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4_t*)(lds_addr(p + h * 4 * (2 * T))));
      fr.b[f] = __builtin_bit_cast(uint4, v);
    }
  }
}

template <int T, bool RM, int BK>
__device__ inline void load_frags(Frags<T>& fr, const char* sa, const char* sb, int s, int wm,
                                  int wn) {
  load_frags_a<T, BK>(fr, sa, s, wm);
  load_frags_b<T, RM, BK>(fr, sb, s, wn);
}

// SWAP = false: acc[fm][fn] = a-rows x b-rows^T (the MFMA layout of AccT).
// SWAP = true feeds the operands the other way round, so acc[fm][fn] holds
// the transposed block: each lane then owns 4 consecutive columns of one row.
// H: the operands are fp16 (same rate and lane layout as bf16).
template <int T, bool SWAP, bool H>
__device__ inline void mma(AccT<T>& acc, const Frags<T>& fr) {
#pragma unroll
  for (int fm = 0; fm < Tile<T>::FM; ++fm)
#pragma unroll
    for (int fn = 0; fn < Tile<T>::FN; ++fn) {
      if constexpr (H)
        acc[fm][fn] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
            __builtin_bit_cast(f16x8_t, SWAP ? fr.b[fn] : fr.a[fm]),
            __builtin_bit_cast(f16x8_t, SWAP ? fr.a[fm] : fr.b[fn]), acc[fm][fn], 0, 0, 0);
      else if constexpr (SWAP)
        acc[fm][fn] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8_t, fr.b[fn]), __builtin_bit_cast(bf16x8_t, fr.a[fm]),
            acc[fm][fn], 0, 0, 0);
      else
        acc[fm][fn] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8_t, fr.a[fm]), __builtin_bit_cast(bf16x8_t, fr.b[fn]),
            acc[fm][fn], 0, 0, 0);
    }
}

// Runs slice(kt, s, cur, nxt) over every 32-wide slice s of every stage kt in
// increasing K order; cur holds the slice's operands, nxt receives the next
// one's.  With an even number of slices per stage the two operand buffers
// alternate within a stage; with one slice per stage, across stages.
template <int NS, class Fr, class Slice>
__device__ inline void for_each_slice(int nk, Fr& f0, Fr& f1, Slice slice) {
  if constexpr (NS % 2 == 0) {
    for (int kt = 0; kt < nk; ++kt)
#pragma unroll
      for (int s = 0; s < NS; s += 2) {
        slice(kt, s, f0, f1);
        slice(kt, s + 1, f1, f0);
      }
  } else {
    static_assert(NS == 1, "one or an even number of slices per stage");
    int kt = 0;
    for (; kt + 1 < nk; kt += 2) {
      slice(kt, 0, f0, f1);
      slice(kt + 1, 0, f1, f0);
    }
    if (kt < nk) slice(kt, 0, f0, f1);
  }
}

// The same address in every lane, in scalar registers (the DMA's base), said
// so that no register allocation moves it to vector ones.
__device__ inline const uint16_t* uniform(const uint16_t* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(v));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(uint32_t(v >> 32));
  return reinterpret_cast<const uint16_t*>((uint64_t(hi) << 32) | lo);
}


// ---------------------------------------------------------------- mapping
// Workgroup p runs on XCD p % 8 (round-robin dispatch).  Logical tiles are
// dealt to the XCDs in chunks of 32 consecutive tiles: XCD x's j-th group of
// 32 workgroups takes chunk 8 (j / 32) + x.  Neighbouring tiles (which share
// operand rows) then run together on one XCD and hit its L2, while the eight
// XCDs work on adjacent chunks of the same matrices, so operand panels that
// leave one L2 are still in the memory-side cache when the next XCD asks for
// them.  The workgroups past the last full round of 8 chunks (all of them in
// a launch of fewer than 256 tiles) split the remaining n tiles the same way:
// XCD x takes a contiguous run of n / 8 of them, one more for x < n % 8 (XCD
// x has exactly that many of those workgroups), so the tiles of one matrix
// still share an L2.
__device__ inline int xcd_remap(int p, int total) {
  constexpr int C = 32;
  const int full = total / (8 * C) * (8 * C);
  if (p < full) {
    const int x = p & 7, j = p >> 3;
    return ((j / C) * 8 + x) * C + (j % C);
  }
  const int n = total - full, q = p - full;
  const int x = q & 7, j = q >> 3;
  return full + x * (n >> 3) + min(x, n & 7) + j;
}

}  // namespace tile
}  // namespace tmk
