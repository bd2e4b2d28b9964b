// Products of ragged groups of rows with one matrix per expert, for gfx950: how
// a call is run, and the sum of slices where the summed index is split.
//
//   matmul   out[i, :] = a[i, :] W[e(i)]        (W: k x n, or n x k transposed)
//   wgrad    out[e] = a_e^T b_e                 (k x n, the rows are summed over)
//
// bf16 operands with 16-byte rows: tm_expert_tiles.hip; the others and fp32:
// tm_expert_staged.hip.
#include <algorithm>

#include "tm_elem.h"
#include "tm_ops.h"

namespace tmk {
namespace expert {

// out = sum of the slices' results, in their order, each thread a vector: rows
// of n, `per` of them a matrix and the matrices `stride` elements apart.
template <class TO>
__global__ __launch_bounds__(256) void k_sum_slices(const float* part, int slices, char* out, int64_t ldo, int64_t per,
                                                    int64_t stride, int64_t rows, int n) {
  constexpr int W = elem::F32::W;
  const int vecs = (n + W - 1) / W;
  const int64_t slice = rows * n;
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const int64_t r = at / vecs;
  if (r >= rows) return;
  const int c = int(at - r * vecs) * W;
  float s[W] = {0.f, 0.f, 0.f, 0.f};
  for (int z = 0; z < slices; ++z) {
    float v[W];
    elem::load_vec<elem::F32>(reinterpret_cast<const char*>(part + z * slice + r * n), c, n, 0.f, v);
#pragma unroll
    for (int i = 0; i < W; ++i) s[i] += v[i];
  }
  char* to = out + (r / per * stride + r % per * ldo + c) * TO::kBytes;
#pragma unroll
  for (int i = 0; i < W; ++i)
    if (c + i < n) TO::store1(to + i * TO::kBytes, s[i]);
}

hipError_t sum_slices(const char* ws, int slices, bool out_f32, char* out, int64_t ldo, int64_t per, int64_t stride,
                      int64_t rows, int n, hipStream_t st) {
  const float* part = reinterpret_cast<const float*>(ws);
  const uint64_t blocks = (uint64_t(rows) * ((uint64_t(n) + 3) / 4) + 255) / 256;
  if (blocks >= (uint64_t(1) << 31)) return hipErrorInvalidConfiguration;
  const dim3 grid{uint32_t(blocks)};
  if (out_f32) hipLaunchKernelGGL((k_sum_slices<elem::F32>), grid, dim3(256), 0, st, part, slices, out, ldo, per, stride, rows, n);
  else hipLaunchKernelGGL((k_sum_slices<elem::Bf16>), grid, dim3(256), 0, st, part, slices, out, ldo, per, stride, rows, n);
  return hipGetLastError();
}

// Whether the tiles on direct loads take an operand or result: rows of whole
// 16-byte pieces, and a stride that keeps a tile's byte offsets below 2^32.
bool whole(const char* p, int64_t ld, int width) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && width % 8 == 0 && ld < (int64_t(1) << 22);
}

uint64_t up(uint64_t v, uint64_t d) { return (v + d - 1) / d; }

// Slices of a summed index of K values for a launch of `tiles` tiles: about
// `want` workgroups, none with fewer than `least` values.
int slices_for(uint64_t tiles, uint64_t K, uint64_t want, uint64_t least) {
  return int(std::max<uint64_t>(1, std::min<uint64_t>({want / std::max<uint64_t>(tiles, 1), K / least, 64})));
}

}  // namespace expert

using namespace expert;

// Tile and slices of a call by its number of tiles of each size and the length
// of its summed index (times in us, measured on both sides of each line).
//
// Direct loads: the 256 tile from 256 tiles on (16384 rows of 1024 x 1024, 260
// tiles: 35, 44 on 128, 58 on 64; 16384 rows over 16 experts of 512 x 512, 160: 21
// against 16); the 128 tile from 256 on (4096 rows over 8 of 1024 x 1024, 320: 18, 22
// on 64; 2048 over 4 of 2048 x 768, 120: 29 against 17), weight gradients from 384
// on (512 of them: 19, 22 on 64; 256: 24 against 20).
// Staged bf16: the 128 tile from 192 on (2048 rows of 2048 x 2048, 272: 35, 44 on 64;
// 2048 over 4 of 2048 x 768, 120: 34 against 25), a long summed index from 64 on, in
// slices (gradient of 1024 x 1024 over 16384 rows: 61 in eight, 88 on 64).
// Staged fp32: from 512 on (1043 rows over 10 of 1408 x 3520, 504: 133, 119 on 64; 8216 over
// 20 of 192 x 1088, 756: 42 against 50), a long summed index as bf16 (the same
// gradient: 213, 285 on 64).
// The 64 tile: slices up to about two workgroups per compute unit (1024 rows of
// 8192 x 1024, direct loads, 272 tiles: 44, 34 and 40 in 1, 2 and 4), fp32 three
// (24211 rows, gradient of 896 x 128: 64, 67 and 75 with 512, 768 and 1536; 17221
// rows over 19 of 1280 x 64: 51, 44 and 45), each of eight stages at least (7 rows over 2
// of 4608 x 64, fp32: 14.5, 17.5 from sixteen on, 16.6 from four on, 72 unsplit).
ExpertPlan plan_tiles(bool staged, bool f32, bool wgrad, const uint64_t (&tiles)[3], uint64_t K) {
  const uint64_t t64 = tiles[0], t128 = tiles[1], t256 = tiles[2];
  ExpertPlan P{};
  P.staged = staged;
  P.tile = 64;
  P.slices = 1;
  if (!staged) {
    if (t256 >= 256) P.tile = 256;
    else if (t128 >= (wgrad ? 384u : 256u)) P.tile = 128;
  } else if (t128 >= (f32 ? 512u : 192u) || (t128 >= 64 && K >= 8192)) {
    P.tile = 128;
    if (K >= 4096) P.slices = slices_for(t128, K, 544, 512);
  }
  if (P.tile == 64) P.slices = f32 ? slices_for(t64, K, 768, 256) : slices_for(t64, K, 544, 512);
  return P;
}

// Groups of up to 24 rows on average are bound by the reading of their matrices
// and take the staged tiles of 16 or 32 rows, whatever the type and alignment (63
// rows over 53 experts of 192 x 6976, bf16: 26 on 16 rows, 57 on the 64 tile of
// direct loads; 80 rows over 5 of 7960 x 1970, fp32: 95 on 32 rows, 184 on 64: the
// larger groups of an uneven call should not need two tiles).  fp32 and odd
// operands stay with 32 rows up to 64 (105 rows over 2 of 4869 x 5632, odd: 47, 51 on
// the 64 tile).
ExpertPlan plan_expert_matmul(const ExpertArgs& A, bool f32, bool transposed) {
  const bool staged = f32 || !(whole(A.a, A.lda, A.k) && whole(A.b, A.ldb, transposed ? A.k : A.n) &&
                               A.stride_b % 8 == 0 && whole(A.out, A.ldo, A.n));
  const uint64_t groups = uint64_t(std::min(A.experts, A.rows)), mean = uint64_t(A.rows) / groups;
  auto tiles = [&](uint64_t TM, uint64_t TN) { return (uint64_t(A.rows) / TM + groups) * up(A.n, TN); };
  ExpertPlan P;
  if (mean <= (staged ? 64u : 24u)) {
    P.staged = true;
    P.tile = mean <= 8 ? 16 : 32;
    P.slices = slices_for(tiles(P.tile, 64), A.k, 1024, f32 ? 256 : 512);
  } else {
    P = plan_tiles(staged, f32, false, {tiles(64, 64), tiles(128, 128), tiles(256, 256)}, A.k);
  }
  P.bytes = P.slices > 1 ? uint64_t(P.slices) * uint64_t(A.rows) * uint64_t(A.n) * 4u : 0u;
  return P;
}

ExpertPlan plan_expert_wgrad(const ExpertArgs& A, bool f32) {
  const bool staged = f32 || !(whole(A.a, A.lda, A.k) && whole(A.b, A.ldb, A.n) && A.stride_b % 8 == 0 &&
                               whole(A.out, A.ldo, A.n));
  auto tiles = [&](uint64_t T) { return uint64_t(A.experts) * up(A.k, T) * up(A.n, T); };
  ExpertPlan P = plan_tiles(staged, f32, true, {tiles(64), tiles(128), tiles(256)}, uint64_t(A.rows) / uint64_t(A.experts));
  P.bytes = P.slices > 1 ? uint64_t(P.slices) * uint64_t(A.experts) * uint64_t(A.k) * uint64_t(A.n) * 4u : 0u;
  return P;
}

hipError_t launch_expert_matmul(const ExpertArgs& call, const ExpertPlan& P, bool f32, bool transposed, char* ws,
                                hipStream_t st) {
  ExpertArgs A = call;
  A.slices = P.slices;
  if (P.slices > 1) {
    A.out = ws;
    A.ldo = A.n;
    A.slice_out = int64_t(A.rows) * A.n;
  }
  const hipError_t e = P.staged ? launch_rows_staged(A, P, f32, transposed, st) : launch_rows_tiles(A, P, transposed, st);
  if (e != hipSuccess || P.slices == 1) return e;
  return sum_slices(ws, P.slices, f32, call.out, call.ldo, A.rows, 0, A.rows, A.n, st);
}

hipError_t launch_expert_wgrad(const ExpertArgs& call, const ExpertPlan& P, bool f32, bool out_f32, char* ws,
                               hipStream_t st) {
  ExpertArgs A = call;
  A.slices = P.slices;
  if (P.slices > 1) {
    A.out = ws;
    A.ldo = A.n;
    A.stride_b = int64_t(A.k) * A.n;
    A.slice_out = A.experts * A.stride_b;
  }
  const hipError_t e = P.staged ? launch_wgrad_staged(A, P, f32, out_f32, st) : launch_wgrad_tiles(A, P, out_f32, st);
  if (e != hipSuccess || P.slices == 1) return e;
  return sum_slices(ws, P.slices, out_f32, call.out, call.ldo, A.k, call.stride_b, int64_t(A.experts) * A.k, A.n, st);
}

}  // namespace tmk
