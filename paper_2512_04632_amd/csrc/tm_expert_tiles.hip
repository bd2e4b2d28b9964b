// Expert products of bf16 rows on the matrix cores: square tiles of 256, 128
// or 64 fed by direct global -> LDS loads, for operands whose rows are 16-byte
// aligned (the others: tm_expert_staged.hip).
//
//   rows    out tile = a rows (summed index contiguous) x W (k x n: row-major,
//           or n x k transposed: summed index contiguous)
//   wgrad   out tile = a^T b of one expert: both operands row-major, the
//           summed index is the expert's rows
//
// Tiles end where a group of rows, a matrix or the summed index does.  Loads
// past an end are clamped to the last row or 16-byte chunk before it, so that
// every address is inside its matrix; what they bring is dropped when the
// tile is stored (rows and columns), or masked to zero in the operand
// registers of the last stage (summed index), in both operands: a NaN that
// belongs to another expert never meets a product.
//
// Bound by the matrix cores and the operand stream that feeds them.  16384 rows over
// 8 experts of 4096 x 14336: forward 1.50-1.55 ms, 1.24-1.28 PFLOP/s; weight gradient with
// fp32 result 1.81-1.86 ms, 1.03-1.06 PFLOP/s (a large square product of one matrix: 1.34).
// Rows backwards of 8192 rows unevenly over 64 experts of 2048 x 1408, 126 us, 0.38 PFLOP/s:
// the tiles that a group's end cuts, and the last round of workgroups.
#include <algorithm>

#include "tm_elem.h"
#include "tm_expert.h"
#include "tm_tile.h"

namespace tmk {
namespace expert {

using namespace tile;

// The share of one of NI loading waves in an operand's stages: T x BK elements
// each, as Q instructions of 1 KB.  RM: the operand is row-major (BK rows of T
// columns, the summed index runs down); otherwise T rows of BK.
template <int T, int BK, int NI>
struct Feed {
  using R = Ring<T, BK>;
  static constexpr int Q = T * BK / 512 / NI;
  const uint16_t* base;   // stage 0 of the tile
  int64_t step;           // elements from a stage to the next
  uint32_t voff[Q];       // this lane's byte offset of each instruction

  // Offsets for a stage of `valid` values of the summed index; `limit` rows (RM: columns) are there.
  template <bool RM>
  __device__ void place(int64_t ld, int limit, int valid, int w) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if constexpr (RM) {
        constexpr int LPR = 2 * T / 16, RPI = 1024 / (2 * T);
        const int r = (NI * q + w) * RPI + lane / LPR, p16 = lane % LPR;
        const int c = ((p16 >> 1) ^ swz_y<T>(r)) * 16 + (p16 & 1) * 8;
        voff[q] = (uint32_t(min(r, valid - 1)) * uint32_t(ld) + uint32_t(min(c, limit - 8))) * 2u;
      } else {
        constexpr int RPI = 64 / R::CPR;
        const int r = (NI * q + w) * RPI + lane / R::CPR;
        const int c = ((lane % R::CPR) ^ ((r / R::RPB) % R::CPR)) * 8;
        voff[q] = (uint32_t(min(r, limit - 1)) * uint32_t(ld) + uint32_t(min(c, valid - 8))) * 2u;
      }
    }
  }
  template <bool RM>
  __device__ void start(const uint16_t* src, int64_t ld) {
    base = uniform(src);
    step = RM ? ld * BK : BK;
  }
  __device__ void issue(int kt, uint32_t lds, int q, int w) const {
    dma16(base + kt * step, voff[q], __builtin_amdgcn_readfirstlane(lds + uint32_t(w + NI * q) * 1024u));
  }
};

// One operand of a tile.
struct Operand {
  const uint16_t* p;
  int64_t ld;
  int limit;   // rows (row-major operand: columns) of the tile that are there
};

// Operands of slice s of a stage with `valid` values of the summed index: the
// others become zero.  A lane holds values 32 s + 8 (lane / 16) .. + 7.
template <int T>
__device__ inline void mask_frags(Frags<T>& fr, int s, int valid) {
  const int n = valid - (32 * s + 8 * int((threadIdx.x & 63) >> 4));
  uint32_t m[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) m[j] = n >= 2 * j + 2 ? 0xffffffffu : n == 2 * j + 1 ? 0xffffu : 0u;
  auto cut = [&](uint4& v) { v = make_uint4(v.x & m[0], v.y & m[1], v.z & m[2], v.w & m[3]); };
#pragma unroll
  for (int f = 0; f < Tile<T>::FM; ++f) cut(fr.a[f]);
#pragma unroll
  for (int f = 0; f < Tile<T>::FN; ++f) cut(fr.b[f]);
}

// The 8-wave tile: the ping-pong schedule described at mainloop_pp in
// tm_fast.hip (groups of four waves one phase apart, five operand slots).
template <int T, int BK, bool ARM, bool BRM>
__device__ inline void product_pp(AccT<T>& acc, char* smem, const Operand& a, const Operand& b, int K) {
  static_assert(Tile<T>::NW == 8 && BK == 64, "two waves per SIMD, two slices per stage");
  using R = Ring<T, BK>;
  using F = Feed<T, BK, 4>;
  constexpr int SLOTS = 5, QG = F::Q;
  const int wave = threadIdx.x >> 6;
  const int wm = wave / Tile<T>::WGN, wn = wave % Tile<T>::WGN;
  const int w4 = wave & 3;
  const bool g1 = __builtin_amdgcn_readfirstlane(wave) >= 4;
  zero_acc<T>(acc);

  const uint32_t lds0 = lds_addr(smem);
  const int nk = (K + BK - 1) / BK, last = K - (nk - 1) * BK;   // values in the last stage
  auto slot_lds = [&](int i) { return lds0 + uint32_t((i % SLOTS) * R::A_BYTES); };
  auto slot_ptr = [&](int i) { return smem + (i % SLOTS) * R::A_BYTES; };
  F feed;   // group 1 loads a, group 0 loads b
  auto place = [&](int valid) {
    if (g1) feed.template place<ARM>(a.ld, a.limit, valid, w4);
    else feed.template place<BRM>(b.ld, b.limit, valid, w4);
  };
  if (g1) feed.template start<ARM>(a.p, a.ld);
  else feed.template start<BRM>(b.p, b.ld);
  place(BK);
  auto issue = [&](int kt) {
    if (kt == nk - 1 && last < BK) place(last);   // no full stage follows
#pragma unroll
    for (int q = 0; q < QG; ++q) feed.issue(kt, slot_lds(2 * kt + (g1 ? 0 : 1)), q, w4);
  };
  issue(0);
  if (g1 && nk > 1) issue(1);
  __builtin_amdgcn_s_waitcnt(0xC07F);
  ring_sync_dma<0>();
  if (g1) barrier_pinned();

  Frags<T> f0, f1;
  for (int j = 0; j < nk; ++j) {
    const char* sa = slot_ptr(2 * j);
    const char* sb = slot_ptr(2 * j + 1);
    const int next = g1 ? j + 2 : j + 1;
    if (next < nk) issue(next);
    __builtin_amdgcn_sched_barrier(0);
    load_pair<T, BK, ARM, BRM>(f0, sa, sb, 0, wm, wn);
    load_pair<T, BK, ARM, BRM>(f1, sa, sb, 1, wm, wn);
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    if (g1) {
      if (j + 2 < nk) dma_wait<QG>();
      else dma_wait<0>();
    }
    barrier_pinned();
    if (j == nk - 1 && last < BK) {
      mask_frags<T>(f0, 0, last);
      mask_frags<T>(f1, 1, last);
    }
    mma<T, true, false>(acc, f0);
    mma<T, true, false>(acc, f1);
    if (!g1) dma_wait<0>();
    barrier_pinned();
  }
  if (!g1) barrier_pinned();
  __builtin_amdgcn_s_waitcnt(0xC07F);
  dma_wait<0>();
}

// The 4-wave tiles: every wave loads its share of stage kt + NSTAGE - 1, spread
// over the slices of stage kt, while it multiplies.
template <int T, int BK, bool ARM, bool BRM>
__device__ inline void product_ring(AccT<T>& acc, char* smem, const Operand& a, const Operand& b, int K) {
  using R = Ring<T, BK>;
  constexpr int PS = R::PER_STAGE, NS = BK / 32, NST = R::NSTAGE, DO = R::DMA_OP, PPS = PS / NS;
  static_assert(PPS * NS == PS && PPS >= 1, "whole DMA instructions per slice");
  using F = Feed<T, BK, Tile<T>::NW>;
  const int wave = threadIdx.x >> 6;
  const int wm = wave / Tile<T>::WGN, wn = wave % Tile<T>::WGN;
  zero_acc<T>(acc);

  const uint32_t lds0 = lds_addr(smem);
  const int nk = (K + BK - 1) / BK, last = K - (nk - 1) * BK;
  F fa, fb;
  fa.template start<ARM>(a.p, a.ld);
  fb.template start<BRM>(b.p, b.ld);
  auto place = [&](int valid) {
    fa.template place<ARM>(a.ld, a.limit, valid, wave);
    fb.template place<BRM>(b.ld, b.limit, valid, wave);
  };
  place(BK);
  auto stage_ptr = [&](int kt) { return smem + (kt % NST) * R::STAGE; };
  // instruction i (0 .. PS - 1) of stage kt: operand a first, then b
  auto dma_one = [&](int kt, int i) {
    if (i == 0 && kt == nk - 1 && last < BK) place(last);
    const uint32_t st = lds0 + uint32_t((kt % NST) * R::STAGE);
    if (i < DO) fa.issue(kt, st, i, wave);
    else fb.issue(kt, st + R::A_BYTES, i - DO, wave);
  };
#pragma unroll
  for (int s = 0; s + 1 < NST; ++s)
    if (s < nk)
#pragma unroll
      for (int i = 0; i < PS; ++i) dma_one(s, i);
  ring_wait<PS, NST - 2>(min(nk - 1, NST - 2));

  Frags<T> f0, f1;
  load_pair<T, BK, ARM, BRM>(f0, stage_ptr(0), stage_ptr(0) + R::A_BYTES, 0, wm, wn);
  for_each_slice<NS>(nk, f0, f1, [&](int kt, int s, Frags<T>& cur, Frags<T>& nxt) {
    const char* st = stage_ptr(kt);
    const int nx = kt + NST - 1;   // stage refilled during this one
    const bool fill = nx < nk;
    if (s + 1 < NS) {
      load_pair<T, BK, ARM, BRM>(nxt, st, st + R::A_BYTES, s + 1, wm, wn);
      if (fill)
#pragma unroll
        for (int i = 0; i < PPS; ++i) dma_one(nx, s * PPS + i);
    } else {
      if (fill)
#pragma unroll
        for (int i = 0; i < PPS; ++i) dma_one(nx, s * PPS + i);
      __builtin_amdgcn_sched_barrier(0);
      if (kt + 1 < nk) {
        ring_wait<PS, NST - 2>(min(nk - 1, kt + NST - 1) - (kt + 1));
        const char* nxp = stage_ptr(kt + 1);
        load_pair<T, BK, ARM, BRM>(nxt, nxp, nxp + R::A_BYTES, 0, wm, wn);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (kt == nk - 1 && last < BK) mask_frags<T>(cur, s, last);
    mma<T, true, false>(acc, cur);
  });
  ring_sync<0>();   // the ring is free for the epilogue
}

template <int T, int BK, bool ARM, bool BRM>
__device__ inline void product(AccT<T>& acc, char* smem, const Operand& a, const Operand& b, int K) {
  if (K <= 0) zero_acc<T>(acc);
  else if constexpr (Tile<T>::NW == 8) product_pp<T, BK, ARM, BRM>(acc, smem, a, b, K);
  else product_ring<T, BK, ARM, BRM>(acc, smem, a, b, K);
}

template <int T, int BK>
constexpr int lds_bytes() { return std::max(Ring<T, BK>::LDS, T * kStageRow<T>); }

// bf16 through LDS: whole rows of the tile, 16 bytes a lane.
template <int T, bool BRM>
__device__ inline void store_bf16(const AccT<T>& acc, char* smem, uint16_t* out, int64_t ld, int rows, int cols) {
  stage_bf16<T>(acc, smem, [](int fn) { return out_col<T, BRM>(fn); });
  constexpr int LPR = T / 8;   // lanes per row
  const int c = int(threadIdx.x % LPR) * 8;
  if (c >= cols) return;
  for (int r = threadIdx.x / LPR; r < rows; r += Tile<T>::NT / LPR)
    *reinterpret_cast<uint4*>(out + r * ld + c) = *reinterpret_cast<const uint4*>(smem + r * kStageRow<T> + c * 2);
}

// fp32 from the registers: 64-byte pieces of rows.
template <int T, bool BRM>
__device__ inline void store_f32(const AccT<T>& acc, float* out, int64_t ld, int rows, int cols) {
#pragma unroll
  for (int fm = 0; fm < Tile<T>::FM; ++fm) {
    const int r = out_row<T>(fm);
    if (r >= rows) continue;
#pragma unroll
    for (int fn = 0; fn < Tile<T>::FN; ++fn) {
      const int c = out_col<T, BRM>(fn);
      if (c < cols) *reinterpret_cast<f32x4_t*>(out + r * ld + c) = acc[fm][fn];
    }
  }
}

// The rows' product.  The 256 tile goes through LDS as the orthogonalizer's update
// does, eight waves and stages of 64 values; 128 and 64 (expert: choose_tile) as
// rings.  OUT32: fp32 results, the slices of a summed index that is split.
template <int T, int BK, bool TRANS, bool OUT32>
__global__ __launch_bounds__(Tile<T>::NT) void k_expert_rows(const ExpertArgs A, int row_tiles) {
  __shared__ __attribute__((aligned(1024))) char smem[lds_bytes<T, BK>()];
  const int nJ = (A.n + T - 1) / T;
  const Slice sl = slice_of(A, int(blockIdx.x), int(gridDim.x));
  const Place at = place_of(sl.id, row_tiles, nJ);
  Group g;
  if (!find_tile(A, T, at.I, g)) return;
  const int e = __builtin_amdgcn_readfirstlane(g.e), first = __builtin_amdgcn_readfirstlane(g.first);
  const int rows = __builtin_amdgcn_readfirstlane(g.last) - first;
  const int c0 = at.J * T, cols = min(T, A.n - c0);
  int k0 = 0, K = 0;
  if (e < A.experts) sl.range(A.k, 64, k0, K);
  const uint16_t* x = reinterpret_cast<const uint16_t*>(A.a) + first * A.lda + k0;
  const uint16_t* w = reinterpret_cast<const uint16_t*>(A.b);
  if (K > 0) w += e * A.stride_b + (TRANS ? c0 * A.ldb + k0 : k0 * A.ldb + c0);
  AccT<T> acc;
  product<T, BK, false, !TRANS>(acc, smem, Operand{x, A.lda, rows}, Operand{w, A.ldb, cols}, K);
  const int64_t out = sl.z * A.slice_out + first * A.ldo + c0;
  if constexpr (OUT32)
    store_f32<T, !TRANS>(acc, reinterpret_cast<float*>(A.out) + out, A.ldo, rows, cols);
  else
    store_bf16<T, !TRANS>(acc, smem, reinterpret_cast<uint16_t*>(A.out) + out, A.ldo, rows, cols);
}

// The weight gradient: rows run down both operands, so both are read with the
// transposing instruction; the 256 tile loses a fifth against the rows' product to
// the second one, and 1.9 GB of fp32 results to HBM (8 x 4096 x 14336).
template <int T, int BK, bool OUT32>
__global__ __launch_bounds__(Tile<T>::NT) void k_expert_wgrad(const ExpertArgs A) {
  __shared__ __attribute__((aligned(1024))) char smem[lds_bytes<T, BK>()];
  const int nI = (A.k + T - 1) / T, nJ = (A.n + T - 1) / T;
  GradTile t;
  if (!grad_tile(A, int(blockIdx.x), int(gridDim.x), nI * nJ, t)) return;
  const Place at = place_of(t.tile, nI, nJ);
  const int r0 = at.I * T, c0 = at.J * T, rows = min(T, A.k - r0), cols = min(T, A.n - c0);
  const uint16_t* x = reinterpret_cast<const uint16_t*>(A.a) + t.first * A.lda + r0;
  const uint16_t* dy = reinterpret_cast<const uint16_t*>(A.b) + t.first * A.ldb + c0;
  AccT<T> acc;
  product<T, BK, true, true>(acc, smem, Operand{x, A.lda, rows}, Operand{dy, A.ldb, cols}, t.K);
  const int64_t out = t.out * A.stride_b + r0 * A.ldo + c0;
  if constexpr (OUT32)
    store_f32<T, true>(acc, reinterpret_cast<float*>(A.out) + out, A.ldo, rows, cols);
  else
    store_bf16<T, true>(acc, smem, reinterpret_cast<uint16_t*>(A.out) + out, A.ldo, rows, cols);
}

template <int T, int BK, bool OUT32>
hipError_t rows_t(const ExpertArgs& A, bool transposed, hipStream_t st) {
  const uint64_t tiles = row_tiles(A, T);
  const uint64_t blocks = tiles * col_tiles(A, T) * uint64_t(A.slices);
  if (!launchable(blocks, Tile<T>::NT)) return hipErrorInvalidConfiguration;
  const dim3 grid{uint32_t(blocks)}, block(Tile<T>::NT);
  if (transposed) hipLaunchKernelGGL((k_expert_rows<T, BK, true, OUT32>), grid, block, 0, st, A, int(tiles));
  else hipLaunchKernelGGL((k_expert_rows<T, BK, false, OUT32>), grid, block, 0, st, A, int(tiles));
  return hipGetLastError();
}

template <int T, int BK, bool OUT32>
hipError_t wgrad_t(const ExpertArgs& A, hipStream_t st) {
  const uint64_t blocks = wgrad_blocks(A, T, T);
  if (!launchable(blocks, Tile<T>::NT)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((k_expert_wgrad<T, BK, OUT32>), dim3(uint32_t(blocks)), dim3(Tile<T>::NT), 0, st, A);
  return hipGetLastError();
}

}  // namespace expert

hipError_t launch_rows_tiles(const ExpertArgs& A, const ExpertPlan& P, bool transposed, hipStream_t st) {
  if (P.tile == 256) return expert::rows_t<256, 64, false>(A, transposed, st);
  if (P.tile == 128) return expert::rows_t<128, 32, false>(A, transposed, st);
  return P.slices > 1 ? expert::rows_t<64, 64, true>(A, transposed, st) : expert::rows_t<64, 64, false>(A, transposed, st);
}

hipError_t launch_wgrad_tiles(const ExpertArgs& A, const ExpertPlan& P, bool out_f32, hipStream_t st) {
  if (P.tile == 256) return out_f32 ? expert::wgrad_t<256, 64, true>(A, st) : expert::wgrad_t<256, 64, false>(A, st);
  if (P.tile == 128) return out_f32 ? expert::wgrad_t<128, 32, true>(A, st) : expert::wgrad_t<128, 32, false>(A, st);
  return out_f32 || P.chunk > 0 ? expert::wgrad_t<64, 64, true>(A, st) : expert::wgrad_t<64, 64, false>(A, st);
}

}  // namespace tmk
