// Products of ragged groups of rows with one matrix per expert, for gfx950.
// Rows are sorted by expert; expert e owns rows ends[e - 1] .. ends[e] - 1.
//
//   matmul   out[i, :] = a[i, :] W[e(i)]        (W: k x n, or n x k transposed)
//   wgrad    out[e] = a_e^T b_e                 (k x n, the rows are summed over)
//
// The group sizes are only known on the device: a launch covers the most tiles
// that any sizes can need, ceil(rows / T) + experts + 1 row tiles, and each
// workgroup finds its expert from `ends`; the ones left over end at once.
// Rows after the last expert's belong to a group of their own without a
// product and come out as zeros; so do the matrices of experts without rows.
#include <algorithm>

#include "tm_elem.h"
#include "tm_expert.h"

namespace tmk {
namespace expert {

using elem::Bf16;
using elem::F32;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- any size and alignment
// 64 x 64 tiles by four waves in a 2 x 2 grid, both operands staged through
// registers into LDS as rows of BK values of the summed index, element by
// element with bounds checks.  fp32 multiplies with v_mfma_f32_16x16x4_f32,
// bf16 with v_mfma_f32_16x16x32_bf16.
template <class T>
struct Any;
template <>
struct Any<Bf16> {
  typedef uint16_t E;
  static constexpr int BK = 32, PAD = 8;
  __device__ static E raw(const char* p) { return *reinterpret_cast<const E*>(p); }
  __device__ static void step(f32x4_t (&acc)[2][2], const E* a, const E* b, int lr, int g) {
    bf16x8_t fa[2], fb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      fa[i] = *reinterpret_cast<const bf16x8_t*>(a + (16 * i + lr) * (BK + PAD) + 8 * g);
      fb[i] = *reinterpret_cast<const bf16x8_t*>(b + (16 * i + lr) * (BK + PAD) + 8 * g);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
  }
};
template <>
struct Any<F32> {
  typedef float E;
  static constexpr int BK = 16, PAD = 4;
  __device__ static E raw(const char* p) { return *reinterpret_cast<const E*>(p); }
  __device__ static void step(f32x4_t (&acc)[2][2], const E* a, const E* b, int lr, int g) {
#pragma unroll
    for (int s = 0; s < BK / 4; ++s) {
      float fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[i] = a[(16 * i + lr) * (BK + PAD) + 4 * s + g];
        fb[i] = b[(16 * i + lr) * (BK + PAD) + 4 * s + g];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[i], fb[j], acc[i][j], 0, 0, 0);
    }
  }
};

constexpr int kAnyTile = 64;

// One operand of the tile: R rows of the tile and K values of the summed
// index are there.  KC: the summed index runs along the stored row; otherwise
// the tile's rows do, and the stage is stored transposed.
template <class T, bool KC>
struct AnySide {
  typedef typename Any<T>::E E;
  static constexpr int BK = Any<T>::BK, LD = BK + Any<T>::PAD, N = kAnyTile * BK / 256;
  const char* base;
  int64_t ld;
  int R, K;
  E v[N];
  __device__ void place(int i, int& r, int& k) const {
    const int at = i * 256 + threadIdx.x;
    if constexpr (KC) {
      r = at / BK;
      k = at % BK;
    } else {
      r = at % kAnyTile;
      k = at / kAnyTile;
    }
  }
  __device__ void load(int k0) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int r, k;
      place(i, r, k);
      const bool in = r < R && k0 + k < K;
      const int64_t at = KC ? r * ld + k0 + k : (k0 + k) * ld + r;
      v[i] = in ? Any<T>::raw(base + at * int64_t(sizeof(E))) : E(0);
    }
  }
  __device__ void store(E* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int r, k;
      place(i, r, k);
      lds[r * LD + k] = v[i];
    }
  }
};

template <class T, bool AKC, bool BKC>
__device__ inline void any_product(f32x4_t (&acc)[2][2], AnySide<T, AKC>& sa, AnySide<T, BKC>& sb, int K) {
  typedef typename Any<T>::E E;
  constexpr int BK = Any<T>::BK, LD = BK + Any<T>::PAD;
  __shared__ __attribute__((aligned(16))) E la[kAnyTile * LD], lb[kAnyTile * LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const E* wa = la + (wave >> 1) * 32 * LD;
  const E* wb = lb + (wave & 1) * 32 * LD;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (K <= 0) return;
  sa.load(0);
  sb.load(0);
  for (int k0 = 0; k0 < K; k0 += BK) {
    __syncthreads();
    sa.store(la);
    sb.store(lb);
    __syncthreads();
    if (k0 + BK < K) {
      sa.load(k0 + BK);
      sb.load(k0 + BK);
    }
    Any<T>::step(acc, wa, wb, lane & 15, lane >> 4);
  }
}

template <class TO>
__device__ inline void any_store(const f32x4_t (&acc)[2][2], char* out, int64_t ld, int rows, int cols) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int r = (wave >> 1) * 32 + 16 * i + 4 * (lane >> 4) + u, c = (wave & 1) * 32 + 16 * j + (lane & 15);
        if (r < rows && c < cols) TO::store1(out + (r * ld + c) * TO::kBytes, acc[i][j][u]);
      }
}

template <class T, bool TRANS>
__global__ __launch_bounds__(256) void k_expert_any(const ExpertArgs A) {
  const int tiles_n = (A.n + kAnyTile - 1) / kAnyTile;
  Group g;
  if (!find_tile<kAnyTile>(A, int(blockIdx.x / uint32_t(tiles_n)), g)) return;
  const int c0 = int(blockIdx.x % uint32_t(tiles_n)) * kAnyTile;
  const int K = g.e < A.experts ? A.k : 0;
  const int cols = min(kAnyTile, A.n - c0), rows = g.last - g.first;
  AnySide<T, true> sa{A.a + g.first * A.lda * T::kBytes, A.lda, rows, K, {}};
  AnySide<T, TRANS> sb{A.b + (K > 0 ? g.e * A.stride_b + (TRANS ? c0 * A.ldb : int64_t(c0)) : 0) * T::kBytes,
                       A.ldb, cols, K, {}};
  f32x4_t acc[2][2];
  any_product<T, true, TRANS>(acc, sa, sb, K);
  any_store<T>(acc, A.out + (g.first * A.ldo + c0) * T::kBytes, A.ldo, rows, cols);
}

template <class T, class TO>
__global__ __launch_bounds__(256) void k_wgrad_any(const ExpertArgs A) {
  const uint32_t tiles_n = (A.n + kAnyTile - 1) / kAnyTile, tiles_k = (A.k + kAnyTile - 1) / kAnyTile;
  const uint32_t per = tiles_n * tiles_k;
  const int e = int(blockIdx.x / per), tile = int(blockIdx.x % per);
  const int r0 = tile / int(tiles_n) * kAnyTile, c0 = tile % int(tiles_n) * kAnyTile;
  const Group g = group_of(A, e);
  const int K = g.last - g.first, rows = min(kAnyTile, A.k - r0), cols = min(kAnyTile, A.n - c0);
  AnySide<T, false> sa{A.a + (g.first * A.lda + r0) * T::kBytes, A.lda, rows, K, {}};
  AnySide<T, false> sb{A.b + (g.first * A.ldb + c0) * T::kBytes, A.ldb, cols, K, {}};
  f32x4_t acc[2][2];
  any_product<T, false, false>(acc, sa, sb, K);
  any_store<TO>(acc, A.out + (e * A.stride_b + r0 * A.ldo + c0) * TO::kBytes, A.ldo, rows, cols);
}

inline bool too_many(uint64_t blocks) { return blocks >= (uint64_t(1) << 31); }

template <class T>
hipError_t matmul_any(const ExpertArgs& A, bool transposed, hipStream_t st) {
  const uint64_t blocks = (uint64_t(A.rows + kAnyTile - 1) / kAnyTile + uint64_t(A.experts) + 1) *
                          (uint64_t(A.n + kAnyTile - 1) / kAnyTile);
  if (too_many(blocks)) return hipErrorInvalidConfiguration;
  if (transposed) hipLaunchKernelGGL((k_expert_any<T, true>), dim3(uint32_t(blocks)), dim3(256), 0, st, A);
  else hipLaunchKernelGGL((k_expert_any<T, false>), dim3(uint32_t(blocks)), dim3(256), 0, st, A);
  return hipGetLastError();
}

template <class T, class TO>
hipError_t wgrad_any(const ExpertArgs& A, hipStream_t st) {
  const uint64_t blocks = uint64_t(A.experts) * (uint64_t(A.n + kAnyTile - 1) / kAnyTile) *
                          (uint64_t(A.k + kAnyTile - 1) / kAnyTile);
  if (too_many(blocks)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((k_wgrad_any<T, TO>), dim3(uint32_t(blocks)), dim3(256), 0, st, A);
  return hipGetLastError();
}

}  // namespace expert

// Whether the tiles of tm_expert_tiles.hip take an operand or result: rows of
// whole 16-byte pieces, and a stride that keeps a tile's byte offsets below 2^32.
static bool whole(const char* p, int64_t ld, int width) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && width % 8 == 0 && ld < (int64_t(1) << 22);
}

hipError_t launch_expert_matmul(const ExpertArgs& A, bool f32, bool transposed, hipStream_t st) {
  if (f32) return expert::matmul_any<elem::F32>(A, transposed, st);
  const bool fits = whole(A.a, A.lda, A.k) && whole(A.b, A.ldb, transposed ? A.k : A.n) && A.stride_b % 8 == 0 &&
                    whole(A.out, A.ldo, A.n);
  return fits ? launch_expert_matmul_tiles(A, transposed, st) : expert::matmul_any<elem::Bf16>(A, transposed, st);
}

hipError_t launch_expert_wgrad(const ExpertArgs& A, bool f32, bool out_f32, hipStream_t st) {
  if (f32) return expert::wgrad_any<elem::F32, elem::F32>(A, st);
  if (whole(A.a, A.lda, A.k) && whole(A.b, A.ldb, A.n) && A.stride_b % 8 == 0 && whole(A.out, A.ldo, A.n))
    return launch_expert_wgrad_tiles(A, out_f32, st);
  return out_f32 ? expert::wgrad_any<elem::Bf16, elem::F32>(A, st) : expert::wgrad_any<elem::Bf16, elem::Bf16>(A, st);
}

}  // namespace tmk
