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
#include "tm_expert.h"

namespace tmk {
namespace expert {

// Entries c .. c + 3 of a row of n: the sum of `count` results that lie `apart`
// elements from each other.
template <class TO>
__device__ inline void sum_vec(const float* part, int64_t apart, int count, char* out, int c, int n) {
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  for (int z = 0; z < count; ++z) {
    float v[4];
    elem::load_vec<elem::F32>(reinterpret_cast<const char*>(part + z * apart), c, n, 0.f, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += v[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (c + i < n) TO::store1(out + (c + i) * TO::kBytes, s[i]);
}

// out = sum of the slices' results, in their order, each thread a vector of the
// rows x n result.  Bound by the reading, from the caches that the slices were
// written to: 2 us and more.
template <class TO>
__global__ __launch_bounds__(256) void k_sum_slices(const float* part, int slices, char* out, int64_t ldo, int64_t rows, int n) {
  const int vecs = (n + 3) / 4;
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const int64_t r = at / vecs;
  if (r >= rows) return;
  sum_vec<TO>(part + r * n, rows * n, slices, out + r * ldo * TO::kBytes, int(at - r * vecs) * 4, n);
}

// out[e] = sum of the matrices of the chunks of e's rows, in their order; zeros for
// an expert without rows.  `per` blocks a matrix; `most` matrices are there, which
// only ends that decrease could pass.
template <class TO>
__global__ __launch_bounds__(256) void k_sum_chunks(const float* part, int64_t most, const ExpertArgs A, int per) {
  const int e = int(blockIdx.x / uint32_t(per)), vecs = (A.n + 3) / 4;
  const Group g = group_of(A, e);
  const int64_t before = min(tiles_before(A, A.chunk, e), most);
  const int chunks = int(min(int64_t((g.last - g.first + A.chunk - 1) / A.chunk), most - before));
  const int64_t at = int64_t(blockIdx.x % uint32_t(per)) * 256 + threadIdx.x, r = at / vecs;
  if (r >= A.k) return;
  const int64_t size = int64_t(A.k) * A.n;
  sum_vec<TO>(part + before * size + r * A.n, size, chunks, A.out + (e * A.stride_b + r * A.ldo) * TO::kBytes,
              int(at - r * vecs) * 4, A.n);
}

hipError_t sum_slices(const char* ws, int slices, bool out_f32, char* out, int64_t ldo, int64_t rows, int n, hipStream_t st) {
  const float* part = reinterpret_cast<const float*>(ws);
  const uint64_t blocks = (uint64_t(rows) * ((uint64_t(n) + 3) / 4) + 255) / 256;
  if (!launchable(blocks, 256)) return hipErrorInvalidConfiguration;
  const dim3 grid{uint32_t(blocks)};
  if (out_f32) hipLaunchKernelGGL((k_sum_slices<elem::F32>), grid, dim3(256), 0, st, part, slices, out, ldo, rows, n);
  else hipLaunchKernelGGL((k_sum_slices<elem::Bf16>), grid, dim3(256), 0, st, part, slices, out, ldo, rows, n);
  return hipGetLastError();
}

hipError_t sum_chunks(const char* ws, const ExpertArgs& A, bool out_f32, hipStream_t st) {
  const float* part = reinterpret_cast<const float*>(ws);
  const uint64_t per = (uint64_t(A.k) * ((uint64_t(A.n) + 3) / 4) + 255) / 256, blocks = per * uint64_t(A.experts);
  if (!launchable(blocks, 256)) return hipErrorInvalidConfiguration;
  const int64_t most = int64_t(row_tiles(A, A.chunk));
  const dim3 grid{uint32_t(blocks)};
  if (out_f32) hipLaunchKernelGGL((k_sum_chunks<elem::F32>), grid, dim3(256), 0, st, part, most, A, int(per));
  else hipLaunchKernelGGL((k_sum_chunks<elem::Bf16>), grid, dim3(256), 0, st, part, most, A, int(per));
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
//
// Groups of few rows on average leave most of a large tile empty, and a weight
// gradient's tile works as long as its group is: the 64 tile up to 64 rows (4096
// rows over 64 experts of 2048 x 1408, even and uneven groups: 86 and 97, 102 and 105 on 128,
// 120 and 122 on 256; 80 rows each: 111 and 110, 108 and 109 on 128), the 128 tile below
// 128 rows (the same experts with 120 rows each, 114 and 114, 120 and 116 on 256; 128: 112 and
// 141, 119 and 119; 144: 135 and 141, 121 and 119; transposed 120: 100 and 121, 98 and 127; 128: 102
// and 122, 99 and 128; 144: 136 and 138, 100 and 127; 40 of 2048 x 2048 are even to 5% from 136 on)
// and for weight gradients up to 256 (128 each: 154 and 164, 156 and 196 on 256; 512 each of
// 2048 x 2048: 116 and 125 against 94 and 146).
int choose_tile(bool staged, bool f32, bool wgrad, const uint64_t (&tiles)[3], uint64_t K, uint64_t mean) {
  const uint64_t t128 = tiles[1], t256 = tiles[2];
  if (!staged && !wgrad && mean <= 64) return 64;
  if (!staged) return t256 >= 256 && mean >= (wgrad ? 257u : 128u) ? 256 : t128 >= (wgrad ? 384u : 256u) ? 128 : 64;
  return t128 >= (f32 ? 512u : 192u) || (t128 >= 64 && K >= 8192) ? 128 : 64;
}

// Workgroups that a call with few tiles is split into, and the fewest values of
// the summed index of each.
uint64_t wanted(bool f32) { return f32 ? 768 : 544; }
uint64_t fewest(bool f32) { return f32 ? 256 : 512; }

// The staged 128 tile: slices from 8192 values on (2048 rows of 8201 x 2048, bf16: 104,
// 112 in one; fp32 450, 538; of 4098 x 2048, bf16, 60 against 54).
//
// An fp32 sum is no longer than kLongest values in one run of the fp32 instructions,
// whose error grows with the root of the number of roundings (464 rows over 55 experts of
// 7770 x 461: 1.1e-6 of the result and 170 us with runs of 5632, 9.1e-7 and 172 of 2816,
// 6.5e-7 and 177 of 1408; 400 over 10 of 5200 x 5000: 1.3e-6 and 363, 9.1e-7 and 367, 6.5e-7
// and 367; 2000 over 20 of 7770 x 461: 1.1e-6 and 256, 9.1e-7 and 221, 6.4e-7 and 224): the
// slices keep as much memory as that many results.  The 128 tile adds 32 products at a time, and its error is below that.
//
// Groups of up to 24 rows on average are bound by the reading of their matrices
// and take the staged tiles of 16 or 32 rows, whatever the type and alignment (63
// rows over 53 experts of 192 x 6976, bf16: 26 on 16 rows, 57 on the 64 tile of
// direct loads; 80 rows over 5 of 7960 x 1970, fp32: 95 on 32 rows, 184 on 64: the
// larger groups of an uneven call should not need two tiles); 16 rows up to 8 on average
// and for a call of no more than 16 (13 rows of 2356 x 6568, fp32: 23, 30 on 32 rows;
// 48 over 8 of 2048 x 4096: 35, 37; 192 over 16: 68 against 64), in slices
// of 512 values and more (24 rows over 8 of 768 x 2048, bf16 and fp32: 8.0 and 11.7, 10.7 and
// 16.1 from 256 on).  fp32 and odd operands stay with 32 rows up to 64 (105 rows over 2 of 4869 x 5632, odd: 47, 51 on
// the 64 tile).
ExpertPlan plan_expert_matmul(const ExpertArgs& A, bool f32, bool transposed) {
  const bool staged = f32 || !(whole(A.a, A.lda, A.k) && whole(A.b, A.ldb, transposed ? A.k : A.n) &&
                               A.stride_b % 8 == 0 && whole(A.out, A.ldo, A.n));
  const uint64_t groups = uint64_t(std::min(A.experts, A.rows)), mean = uint64_t(A.rows) / groups;
  auto tiles = [&](uint64_t TM, uint64_t TN) { return (uint64_t(A.rows) / TM + groups) * up(A.n, TN); };
  ExpertPlan P{};
  if (mean <= (staged ? 64u : 24u)) {
    P.staged = true;
    P.tile = mean <= 8 || A.rows <= 16 ? 16 : 32;
    P.slices = slices_for(tiles(P.tile, 64), A.k, 1024, 512);
  } else {
    const uint64_t t[3] = {tiles(64, 64), tiles(128, 128), tiles(256, 256)};
    P.staged = staged;
    P.tile = choose_tile(staged, f32, false, t, A.k, mean);
    P.slices = 1;
    if (P.tile == 64) P.slices = slices_for(t[0], A.k, wanted(f32), fewest(f32));
    else if (P.tile == 128 && staged && A.k >= 8192) P.slices = slices_for(t[1], A.k, 544, 512);
  }
  if (f32 && P.tile < 128) P.slices = std::max(P.slices, int(up(A.k, kLongest)));
  P.bytes = P.slices > 1 ? uint64_t(P.slices) * uint64_t(A.rows) * uint64_t(A.n) * 4u : 0u;
  return P;
}

// A weight gradient's summed index is a group's rows, and their number is not
// known here: where there are few tiles, groups are cut into chunks of so many
// rows that the call has about the wanted number of workgroups whoever owns the
// rows, and chunks are summed afterwards (24162 rows, unevenly over 11 experts of
// 73 x 2069, fp32: 128 us; 255 with every group cut into the same number of
// parts).  Short groups gain less than the sum costs: 10342 rows over 43 experts of
// 1133 x 103, bf16, are 19 us whole and 31 in chunks.  With fewer tiles than compute
// units the longest group alone may be the call's time, and groups of 256 rows on
// average are cut too (6000 rows unevenly over 20 of 128 x 128: fp32 41 and 15.5, bf16 14.3 and
// 11.5; evenly 9617 over 24 of 114 x 133: 15.2 and 17.8, 8.1 and 11.7); below 4096 rows the second
// launch costs more (1200 over 4 of 256 x 512, bf16: 7.8 and 10.6), and so it does on the 128
// tile (5000 over 12 of 768 x 300, bf16: 19 and 24).
ExpertPlan plan_expert_wgrad(const ExpertArgs& A, bool f32) {
  ExpertPlan P{};
  P.staged = f32 || !(whole(A.a, A.lda, A.k) && whole(A.b, A.ldb, A.n) && A.stride_b % 8 == 0 && whole(A.out, A.ldo, A.n));
  auto tiles = [&](uint64_t T) { return up(A.k, T) * up(A.n, T); };
  const uint64_t experts = uint64_t(A.experts), rows = uint64_t(A.rows);
  const uint64_t t[3] = {experts * tiles(64), experts * tiles(128), experts * tiles(256)};
  P.tile = choose_tile(P.staged, f32, true, t, rows / experts, rows / experts);
  const uint64_t want = P.tile == 64 ? wanted(f32) : 544;
  if ((P.tile == 64 || (P.tile == 128 && P.staged)) && experts * tiles(P.tile) <= want + want / 2) {
    const uint64_t chunk = std::max(fewest(f32), up(rows * tiles(P.tile), want * 64) * 64);
    const uint64_t mean = rows / experts;
    const bool uneven = P.tile == 64 && experts * tiles(64) <= 256 && mean >= 256 && rows >= 4096;
    if (rows >= 2 * chunk && (mean >= 2 * fewest(f32) || uneven)) P.chunk = int(chunk);
  }
  if (f32 && P.tile == 64 && rows / experts > kLongest)
    P.chunk = P.chunk > 0 ? std::min(P.chunk, int(kLongest)) : int(kLongest);
  if (P.chunk > 0)
    P.bytes = row_tiles(A, P.chunk) * uint64_t(A.k) * uint64_t(A.n) * 4u;
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
  return sum_slices(ws, P.slices, f32, call.out, call.ldo, A.rows, A.n, st);
}

hipError_t launch_expert_wgrad(const ExpertArgs& call, const ExpertPlan& P, bool f32, bool out_f32, char* ws,
                               hipStream_t st) {
  ExpertArgs A = call;
  A.chunk = P.chunk;
  if (P.chunk > 0) {
    A.out = ws;
    A.ldo = A.n;
    A.stride_b = int64_t(A.k) * A.n;
  }
  const hipError_t e = P.staged ? launch_wgrad_staged(A, P, f32, out_f32, st) : launch_wgrad_tiles(A, P, out_f32, st);
  if (e != hipSuccess || P.chunk == 0) return e;
  A.out = call.out;
  A.ldo = call.ldo;
  A.stride_b = call.stride_b;
  return sum_chunks(ws, A, out_f32, st);
}

}  // namespace tmk
