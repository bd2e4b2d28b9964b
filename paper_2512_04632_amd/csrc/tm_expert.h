// What the expert products' kernels share: the rows of each expert, found on
// the device, the order of the tiles, operand reads and the output stage.
//
// The group sizes are only known on the device: a launch covers the most tiles
// that any sizes can need, and each workgroup finds its expert from `ends`; the
// ones left over end at once.
// Rows after the last expert's belong to a group of their own without a
// product and come out as zeros; so do the matrices of experts without rows.
#pragma once

#include <algorithm>

#include "tm_ops.h"
#include "tm_tile.h"

namespace tmk {
namespace expert {

using namespace tile;

// Longest run of a sum in fp32 instructions (tm_expert.hip: plan_expert_matmul).
constexpr uint64_t kLongest = 2816;

// A run of rows [first, last) of one expert (experts: the rows of none).
struct Group {
  int e, first, last;
};

// First and last row of group e.  Whatever `ends` holds, the rows stay within the matrix.
__device__ inline Group group_of(const ExpertArgs& A, int e) {
  Group g;
  g.e = e;
  g.first = e == 0 ? 0 : min(max(A.ends[e - 1], 0), A.rows);
  g.last = e == A.experts ? A.rows : min(max(A.ends[e], g.first), A.rows);
  return g;
}

// Row tile `tile` (of T rows, counted from group to group) of the launch: its
// group cut to the tile's rows.  Every lane of a wave calls it; the lanes look at
// 64 groups at a time.  False past the last tile.
__device__ inline bool find_tile(const ExpertArgs& A, int T, int tile, Group& out) {
  const int lane = threadIdx.x & 63;
  int before = 0;   // tiles of the groups looked at so far
  for (int base = 0; base <= A.experts; base += 64) {
    const int e = base + lane;
    Group g{e, 0, 0};
    if (e <= A.experts) g = group_of(A, e);
    const int tiles = (g.last - g.first + T - 1) / T;
    int sum = tiles;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(sum, o);
      if (lane >= o) sum += up;
    }
    const uint64_t past = __ballot(before + sum > tile);
    if (past != 0) {
      const int src = __ffsll((unsigned long long)past) - 1;
      const int first = __shfl(g.first, src) + (tile - before - __shfl(sum - tiles, src)) * T;
      out = Group{base + src, first, min(first + T, __shfl(g.last, src))};
      return true;
    }
    before += __shfl(sum, 63);
  }
  return false;
}

// Rows of T-row tiles that any group sizes can need: the whole tiles, one more for
// each group that has rows (the experts' and the one of no expert), and no more
// than there are rows.
inline uint64_t row_tiles(const ExpertArgs& A, int T) {
  const uint64_t rows = uint64_t(A.rows), groups = std::min(uint64_t(A.experts) + 1, rows);
  return std::min(rows / T + groups, rows);
}
inline uint64_t col_tiles(const ExpertArgs& A, int T) { return (uint64_t(A.n) + T - 1) / T; }
// Blocks of a weight gradient on TM x TN tiles: the experts' matrices, or those of
// the chunks of their rows.
inline uint64_t wgrad_blocks(const ExpertArgs& A, int TM, int TN) {
  return (A.chunk == 0 ? uint64_t(A.experts) : row_tiles(A, A.chunk)) * ((uint64_t(A.k) + TM - 1) / TM) * col_tiles(A, TN);
}

// Tiles (of T rows) of the groups before e; every lane of a wave calls it.
__device__ inline int64_t tiles_before(const ExpertArgs& A, int T, int e) {
  const int lane = threadIdx.x & 63;
  int64_t sum = 0;
  for (int base = 0; base < e; base += 64)
    if (base + lane < e) {
      const Group g = group_of(A, base + lane);
      sum += (g.last - g.first + T - 1) / T;
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor((long long)sum, o);
  return sum;
}

// A workgroup's tile and its slice z of the summed index.
struct Slice {
  int id, z, slices;
  // Slice of K values, in whole stages of `unit`: first value and number.
  __device__ void range(int K, int unit, int& k0, int& n) const {
    const int len = ((K + slices - 1) / slices + unit - 1) / unit * unit;
    k0 = min(z * len, K);
    n = min(len, K - k0);
  }
};
__device__ inline Slice slice_of(const ExpertArgs& A, int block, int blocks) {
  const int per = blocks / A.slices;
  const int z = A.slices > 1 ? block / per : 0;
  return Slice{xcd_remap(block - z * per, per), z, A.slices};
}

// Place of logical tile `id` in a grid of nI x nJ tiles, in groups of four rows
// of tiles: tiles that run together share operand panels.
struct Place {
  int I, J;
};
__device__ inline Place place_of(int id, int nI, int nJ) {
  constexpr int GM = 4;
  const int grp = id / (GM * nJ), first = grp * GM, size = min(nI - first, GM);
  const int rem = id - grp * GM * nJ;
  return Place{first + rem % size, rem / size};
}

// Row-major a operand: the wave's block f of 16 columns is chunk wm FM + f of
// the stage's rows; chunk ^ swizzle = ((wm FM) ^ swizzle) ^ f, since f < FM.
template <int T, int BK>
__device__ inline void load_frags_a_rm(Frags<T>& fr, const char* sa, int s, int wm) {
  constexpr int FM = Tile<T>::FM;
  const int lane = threadIdx.x & 63;
  const int lr = lane & 15, g = lane >> 4;
  const int rl = 8 * g + (lr >> 2);
  const char* base = sa + (32 * s + rl) * (2 * T) + 8 * (lr & 3);
  const int chunk = (wm * FM) ^ swz_y<T>(rl);
#pragma unroll
  for (int f = 0; f < FM; ++f) {
    const char* p = base + 32 * (chunk ^ f);
    s16x4_t v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4_t*)(lds_addr(p + h * 4 * (2 * T))));
    fr.a[f] = __builtin_bit_cast(uint4, v);
  }
}

template <int T, int BK, bool ARM, bool BRM>
__device__ inline void load_pair(Frags<T>& fr, const char* sa, const char* sb, int s, int wm, int wn) {
  if constexpr (ARM) load_frags_a_rm<T, BK>(fr, sa, s, wm);
  else load_frags_a<T, BK>(fr, sa, s, wm);
  load_frags_b<T, BRM, BK>(fr, sb, s, wn);
}

// Bytes of a row of the output stage: 16 more than a tile's row, so that the
// 16 rows that a wave writes at a time start in different banks.
template <int T>
constexpr int kStageRow = 2 * T + 16;

// Row and first of the four columns that a lane holds of block (fm, fn).
template <int T>
__device__ inline int out_row(int fm) {
  const int wave = threadIdx.x >> 6;
  return (wave / Tile<T>::WGN) * Tile<T>::TWM + 16 * fm + int(threadIdx.x & 15);
}
template <int T, bool BRM>
__device__ inline int out_col(int fn) {
  const int wn = int(threadIdx.x >> 6) % Tile<T>::WGN;
  return (BRM ? 16 * (fn * Tile<T>::WGN + wn) : wn * Tile<T>::TWN + 16 * fn) + 4 * (int(threadIdx.x & 63) >> 4);
}

// The tile's bf16 values in LDS, rows of kStageRow bytes; ends with a barrier.
template <int T, class FCol>
__device__ inline void stage_bf16(const AccT<T>& acc, char* smem, FCol col) {
#pragma unroll
  for (int fm = 0; fm < Tile<T>::FM; ++fm)
#pragma unroll
    for (int fn = 0; fn < Tile<T>::FN; ++fn) {
      uint32_t o[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) o[u] = f2bf(acc[fm][fn][u]);
      *reinterpret_cast<uint2*>(smem + out_row<T>(fm) * kStageRow<T> + col(fn) * 2) =
          make_uint2(o[0] | o[1] << 16, o[2] | o[3] << 16);
    }
  __syncthreads();
}

// A weight gradient's tile: rows [first, first + K) of expert e, summed into matrix
// `out` of the result (or, with chunks, of the workspace).
struct GradTile {
  int out, tile, first, K;
};
// Block `block` of a launch over `tiles` tiles a matrix; false for one that has nothing to do.
__device__ inline bool grad_tile(const ExpertArgs& A, int block, int blocks, int tiles, GradTile& t) {
  const int id = xcd_remap(block, blocks);
  t.out = id / tiles;
  t.tile = id - t.out * tiles;
  Group g;
  if (A.chunk == 0) {
    g = group_of(A, t.out);
  } else if (!find_tile(A, A.chunk, t.out, g) || g.e == A.experts) {
    return false;
  }
  t.first = __builtin_amdgcn_readfirstlane(g.first);
  t.K = __builtin_amdgcn_readfirstlane(g.last) - t.first;
  return true;
}

}  // namespace expert
}  // namespace tmk
