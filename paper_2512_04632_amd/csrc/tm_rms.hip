// Root-mean-square norm over the rows of a matrix, with the residual's addition,
// forward and backward, for gfx950.
//
//   forward   s = x + residual (rounded to the type; s = x without one),
//             rstd = 1 / sqrt(sum s^2 / d + eps),  y = s rstd weight
//   backward  h = s rstd,  g = dy weight,
//             ds = rstd (g - h sum(g h) / d) + dsum,
//             dweight = sum over rows of dy h
//
// As in layer norm a row stays in the registers of the threads that own it and is
// read once; there is one sum over it, of the rounded s, so that the backward pass,
// which reads s, sees the same values.  The backward pass keeps the columns' sums of
// dweight in registers over a workgroup's rows.  Statistics and sums are fp32; s, y and
// ds are rounded once.  Both passes are bound by HBM.
#include <algorithm>

#include "tm_norm.h"

namespace tmk {
namespace norm {

// A vector as stored, whole or up to the row's end.
template <class T>
__device__ inline void store_packed(char* row, int first, int n, u32x4_t q) {
  if (first + T::W <= n) {
    T::store(row + int64_t(first) * T::kBytes, q);
  } else {
    float v[T::W];
    T::unpack(q, v);
    store_vec<T>(row, first, n, v);
  }
}

// The rounded sum of two vectors.
template <class T>
__device__ inline u32x4_t add_rounded(u32x4_t a, u32x4_t b) {
  float x[T::W], y[T::W];
  T::unpack(a, x);
  T::unpack(b, y);
#pragma unroll
  for (int i = 0; i < T::W; ++i) x[i] += y[i];
  return T::pack(x);
}

// Forward.  s may take the place of x or of the residual: it is stored behind the
// row's sum, when every thread has what it loaded of the row.  16384 x 4096 bf16 with
// residual 92 us for 537 MB, 5.8 TB/s (107 at the rate of a large copy); 4 rows are the
// 9 us of a call on the host, 3 of them the kernel's.
template <class T, int NT, int E, bool TAIL, bool RES>
__global__ __launch_bounds__(block_threads<NT>()) void k_rms(const RmsArgs A) {
  constexpr int W = T::W, V = E / W, RB = block_threads<NT>() / NT, NW = NT > 64 ? NT / 64 : 1;
  __shared__ float slots[2][NW];
  const int t = threadIdx.x % NT, d = A.d;
  const float n = float(d);
  float w[E];
  load_cols<NT, E, T>(A.weight, 1.f, t, d, w);
  const int64_t step = int64_t(gridDim.x) * RB;
  int64_t r = int64_t(blockIdx.x) * RB + threadIdx.x / NT;
  u32x4_t q[V], p[RES ? V : 1];
  auto read = [&](int64_t at) __attribute__((always_inline)) {
    load_row<NT, V, T, TAIL>(A.x + at * A.ldx * T::kBytes, t, d, q);
    if constexpr (RES) load_row<NT, V, T, TAIL>(A.residual + at * A.ldr * T::kBytes, t, d, p);
  };
  if (r < A.rows) read(r);
  for (int turn = 0; r < A.rows; r += step, turn ^= 1) {
    u32x4_t s[V];
    float sum[1] = {0.f};
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * NT + t) * W;
      s[j] = settle<T, TAIL>(q[j], c, d);
      if constexpr (RES) s[j] = add_rounded<T>(s[j], settle<T, TAIL>(p[j], c, d));
      float v[W];
      T::unpack(s[j], v);
#pragma unroll
      for (int i = 0; i < W; ++i) sum[0] += v[i] * v[i];
    }
    // the next row is on its way while this one is summed
    if (r + step < A.rows) read(r + step);
    row_sum<NT>(sum, slots[turn]);
    const float rstd = 1.f / sqrtf(sum[0] / n + A.eps);
    if (t == 0) A.rstd[r] = rstd;
    char* y = A.out + r * A.ldo * T::kBytes;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * NT + t) * W;
      if (c >= d) continue;
      if constexpr (RES) store_packed<T>(A.sum + r * A.lds * T::kBytes, c, d, s[j]);
      float o[W];
      T::unpack(s[j], o);
#pragma unroll
      for (int i = 0; i < W; ++i) o[i] *= rstd * w[j * W + i];
      store_vec<T>(y, c, d, o);
    }
  }
}

// Backward: dy, s and dsum are read once, ds is written once.  16384 x 4096 bf16 with
// dsum 95 us for 537 MB, 5.7 TB/s, and 5 us to add up the 256 lines of partial sums;
// 2048 x 8190 fp32 70 us for 268 MB, 3.8 TB/s: a row whose width is no whole number of
// vectors needs registers of its own for its end.  fp32 rows of more than 8192 with dsum keep 8 to 10
// registers a lane in memory.
template <class T, int NT, int E, bool TAIL, bool ADD>
__global__ __launch_bounds__(block_threads<NT>()) void k_rms_backward(const RmsArgs A) {
  constexpr int W = T::W, V = E / W, RB = block_threads<NT>() / NT, NW = NT > 64 ? NT / 64 : 1;
  constexpr int AHEAD = NT < 1024 ? 1 : 0;
  __shared__ float slots[2][NW];
  const int t = threadIdx.x % NT, d = A.d;
  const float n = float(d);
  float w[E], aw[E];
  load_cols<NT, E, T>(A.weight, 1.f, t, d, w);
#pragma unroll
  for (int i = 0; i < E; ++i) aw[i] = 0.f;
  const int64_t step = int64_t(gridDim.x) * RB;
  int64_t r = int64_t(blockIdx.x) * RB + threadIdx.x / NT;
  u32x4_t qs[V], qy[V], qd[ADD ? V : 1];
  float scale = 0.f;
  auto read = [&](int64_t at) __attribute__((always_inline)) {
    load_row<NT, V, T, TAIL>(A.x + at * A.ldx * T::kBytes, t, d, qs);
    load_row<NT, V, T, TAIL>(A.dy + at * A.lddy * T::kBytes, t, d, qy);
    if constexpr (ADD) load_row<NT, V, T, TAIL>(A.residual + at * A.ldr * T::kBytes, t, d, qd);
    scale = A.rstd[at];
  };
  if (AHEAD > 0 && r < A.rows) read(r);
  for (int turn = 0; r < A.rows; r += step, turn ^= 1) {
    if constexpr (AHEAD == 0) read(r);
    float h[E], g[E], sum[1] = {0.f};
    u32x4_t add[ADD ? V : 1];
    const float rstd = scale;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (j * NT + t) * W;
      T::unpack(settle<T, TAIL>(qs[j], c, d), h + j * W);
      T::unpack(settle<T, TAIL>(qy[j], c, d), g + j * W);
      if constexpr (ADD) add[j] = settle<T, TAIL>(qd[j], c, d);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const int e = j * W + i;
        h[e] *= rstd;
        aw[e] += g[e] * h[e];
        g[e] *= w[e];
        sum[0] += g[e] * h[e];
      }
    }
    if (AHEAD > 0 && r + step < A.rows) read(r + step);
    row_sum<NT>(sum, slots[turn]);
    const float m = sum[0] / n;
    char* ds = A.out + r * A.ldo * T::kBytes;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float o[W], more[W];
      if constexpr (ADD) T::unpack(add[j], more);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const int e = j * W + i;
        o[i] = rstd * (g[e] - h[e] * m);
        if constexpr (ADD) o[i] += more[i];
      }
      store_vec<T>(ds, (j * NT + t) * W, d, o);
    }
  }
  // the sums of the block's rows: to its line of partial sums, or as the result
  float* to = A.part != nullptr ? A.part + int64_t(blockIdx.x) * d : A.dweight;
  if (to == nullptr) return;
  if constexpr (RB > 1) {   // the waves' rows first, one after the other
    __shared__ float sums[NT * E];
    for (int q = 0; q < RB; ++q) {
      if (int(threadIdx.x) / NT == q)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int at = (e / W * NT + t) * W + e % W;
          sums[at] = (q > 0 ? sums[at] : 0.f) + aw[e];
        }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < d; c += block_threads<NT>()) to[c] = sums[c];
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = (e / W * NT + t) * W + e % W;
      if (c < d) to[c] = aw[e];
    }
  }
}

// Rows wider than a workgroup's registers (kNormMaxFused): read once for the sum and once
// for the result, the second time from a cache.
template <class T, bool RES>
__global__ __launch_bounds__(kWide) void k_rms_wide(const RmsArgs A) {
  __shared__ float slots[2][kWide / 64];
  const int d = A.d;
  int turn = 0;
  for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x, turn ^= 1) {
    const char* x = A.x + r * A.ldx * T::kBytes;
    char* sum_row = RES ? A.sum + r * A.lds * T::kBytes : nullptr;
    const char* from = RES ? sum_row : x;   // each thread reads back what it wrote
    char* y = A.out + r * A.ldo * T::kBytes;
    float s[1] = {0.f}, v[T::W];
    each_vec<T>(d, [&](int c) {
      load_vec<T>(x, c, d, 0.f, v);
      if constexpr (RES) {
        float more[T::W];
        load_vec<T>(A.residual + r * A.ldr * T::kBytes, c, d, 0.f, more);
#pragma unroll
        for (int i = 0; i < T::W; ++i) v[i] += more[i];
        const u32x4_t q = T::pack(v);
        T::unpack(q, v);
        store_packed<T>(sum_row, c, d, q);
      }
#pragma unroll
      for (int i = 0; i < T::W; ++i) s[0] += v[i] * v[i];
    });
    row_sum<kWide>(s, slots[turn]);
    const float rstd = 1.f / sqrtf(s[0] / float(d) + A.eps);
    if (threadIdx.x == 0) A.rstd[r] = rstd;
    each_vec<T>(d, [&](int c) {
      load_vec<T>(from, c, d, 0.f, v);
#pragma unroll
      for (int i = 0; i < T::W; ++i) v[i] *= rstd * col(A.weight, 1.f, c + i, d);
      store_vec<T>(y, c, d, v);
    });
  }
}

template <class T>
__global__ __launch_bounds__(kWide) void k_rms_backward_wide(const RmsArgs A) {
  __shared__ float slots[2][kWide / 64];
  const int d = A.d;
  int turn = 0;
  for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x, turn ^= 1) {
    const char* x = A.x + r * A.ldx * T::kBytes;
    const char* dy = A.dy + r * A.lddy * T::kBytes;
    const char* more = A.residual != nullptr ? A.residual + r * A.ldr * T::kBytes : nullptr;
    char* ds = A.out + r * A.ldo * T::kBytes;
    const float rstd = A.rstd[r];
    float s[1] = {0.f}, h[T::W], g[T::W];
    auto read = [&](int c) {
      load_vec<T>(x, c, d, 0.f, h);
      load_vec<T>(dy, c, d, 0.f, g);
#pragma unroll
      for (int i = 0; i < T::W; ++i) {
        h[i] *= rstd;
        g[i] *= col(A.weight, 1.f, c + i, d);
      }
    };
    each_vec<T>(d, [&](int c) {
      read(c);
#pragma unroll
      for (int i = 0; i < T::W; ++i) s[0] += g[i] * h[i];
    });
    row_sum<kWide>(s, slots[turn]);
    const float m = s[0] / float(d);
    each_vec<T>(d, [&](int c) {
      read(c);
      float add[T::W];
#pragma unroll
      for (int i = 0; i < T::W; ++i) add[i] = 0.f;
      if (more != nullptr) load_vec<T>(more, c, d, 0.f, add);
#pragma unroll
      for (int i = 0; i < T::W; ++i) g[i] = rstd * (g[i] - h[i] * m) + add[i];
      store_vec<T>(ds, c, d, g);
    });
  }
}

// Column sums of such rows: one thread per column, each block a slice of the rows.
template <class T>
__global__ __launch_bounds__(256) void k_rms_columns(const RmsArgs A, int slices) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= A.d) return;
  float aw = 0.f;
  for (int64_t r = blockIdx.y; r < A.rows; r += slices)
    aw += T::load1(A.dy + (r * A.lddy + c) * T::kBytes) * (T::load1(A.x + (r * A.ldx + c) * T::kBytes) * A.rstd[r]);
  A.part[int64_t(blockIdx.y) * A.d + c] = aw;
}

// Most workgroups.  One a CU, where 16 KB or more are on the way to each while a row is worked on: that covers the
// latency, and fewer streams of reads and writes take turns at the memory (16384 rows with residual, us, 256 / 4096
// workgroups: 3504 bf16 87 / 91, 4096 91 / 99, 5120 118 / 123, 1752 fp32 85 / 91, 2048 91 / 99; backwards, 256 / 512:
// 85 / 89, 98 / 106, 125 / 137, 84 / 86, 96 / 102).  Where it is less, more (2560 bf16 77 / 63, backwards 72 / 66).  So do
// rows of a wave forwards, whose loads are not that long (16384 x 1024 bf16 24 / 21).  Backwards each workgroup
// has its line of partial sums, and the gradients' two streams, which are always there, are counted.
// An fp32 row that ends inside a vector has twice the vectors of a bf16 row to put right, which one workgroup a CU of up
// to 256 threads does not cover (16384 rows, 256 / 4096: 2049 269 / 113, 3001 332 / 159, 4095 391 / 208; 2048 x 8190
// 57 / 48; backwards, 256 / 512: 513 76 / 49, 1001 113 / 70, 2049 326 / 192, 4093 442 / 268; 8192 x 4097 184 / 187).
// Such a bf16 row is alike both ways (4097 129 / 121, 8191 without residual 122 / 119, 2048 x 4099 16 / 18; backwards
// 143 / 146, 188 / 198, 21 / 27).
template <class T>
int rms_blocks(const RmsArgs& A) {
  if (T::kBytes == 4 && A.d % T::W != 0) return 4096;
  return A.d > 1024 && A.d * T::kBytes * (A.residual != nullptr ? 2 : 1) >= 16384 ? 256 : 4096;
}
inline int most_lines(int64_t d, bool f32) {
  if (f32 && d % 4 != 0 && d <= 4096) return 512;
  return d * (f32 ? 4 : 2) * (d <= 1024 ? 4 : 1) >= 8192 ? 256 : 512;
}
constexpr int kRmsWideBlocks = 2048;

template <class T, int NT, int E>
hipError_t rms(const RmsArgs& A, hipStream_t st) {
  constexpr int RB = block_threads<NT>() / NT;
  const dim3 grid(uint32_t(std::min<int64_t>((int64_t(A.rows) + RB - 1) / RB, rms_blocks<T>(A)))), block(block_threads<NT>());
  const bool tail = A.d % T::W != 0, res = A.residual != nullptr;
  if (tail && res) hipLaunchKernelGGL((k_rms<T, NT, E, true, true>), grid, block, 0, st, A);
  else if (tail) hipLaunchKernelGGL((k_rms<T, NT, E, true, false>), grid, block, 0, st, A);
  else if (res) hipLaunchKernelGGL((k_rms<T, NT, E, false, true>), grid, block, 0, st, A);
  else hipLaunchKernelGGL((k_rms<T, NT, E, false, false>), grid, block, 0, st, A);
  return hipGetLastError();
}

template <class T, int NT, int E>
hipError_t rms_backward(const RmsArgs& A, int blocks, hipStream_t st) {
  const dim3 grid(blocks), block(block_threads<NT>());
  const bool tail = A.d % T::W != 0, add = A.residual != nullptr;
  if (tail && add) hipLaunchKernelGGL((k_rms_backward<T, NT, E, true, true>), grid, block, 0, st, A);
  else if (tail) hipLaunchKernelGGL((k_rms_backward<T, NT, E, true, false>), grid, block, 0, st, A);
  else if (add) hipLaunchKernelGGL((k_rms_backward<T, NT, E, false, true>), grid, block, 0, st, A);
  else hipLaunchKernelGGL((k_rms_backward<T, NT, E, false, false>), grid, block, 0, st, A);
  return hipGetLastError();
}

// Widest row of 16 threads: four of them a wave (30000 x 65 bf16 with residual, us forward and
// backward: 9.8 and 12.8, by a wave each 13.7 and 20.4).
constexpr int kNarrow = 128;

// Threads for a row and elements of each: as for layer norm, whose rows are held in the same way.
template <class T>
hipError_t rms_t(const RmsArgs& A, hipStream_t st) {
  const int d = A.d;
  if (d <= kNarrow) return rms<T, 16, 8>(A, st);
  if (d <= 512) return rms<T, 64, 8>(A, st);
  if (d <= 1024) return rms<T, 64, 16>(A, st);
  if (d <= 2048) return rms<T, 256, 8>(A, st);
  if (d <= 4096) return rms<T, 256, 16>(A, st);
  if (d <= 8192) return rms<T, 512, 16>(A, st);
  if (d <= kNormMaxFused) return rms<T, 1024, 16>(A, st);
  const dim3 grid(std::min(A.rows, kRmsWideBlocks)), block(kWide);
  if (A.residual != nullptr) hipLaunchKernelGGL((k_rms_wide<T, true>), grid, block, 0, st, A);
  else hipLaunchKernelGGL((k_rms_wide<T, false>), grid, block, 0, st, A);
  return hipGetLastError();
}

template <class T>
hipError_t rms_backward_t(const RmsArgs& A, int blocks, hipStream_t st) {
  const int d = A.d;
  if (d <= kNarrow) return rms_backward<T, 16, 8>(A, blocks, st);
  if (d <= 512) return rms_backward<T, 64, 8>(A, blocks, st);
  if (d <= 1024) return rms_backward<T, 64, 16>(A, blocks, st);
  if (d <= 2048) return rms_backward<T, 256, 8>(A, blocks, st);
  if (d <= 4096) return rms_backward<T, 256, 16>(A, blocks, st);
  if (d <= 8192) return rms_backward<T, 512, 16>(A, blocks, st);
  if (d <= kNormMaxFused) return rms_backward<T, 1024, 16>(A, blocks, st);
  // ds may take the place of dy or s, so the column sums come first
  if (A.part != nullptr) {
    hipLaunchKernelGGL((k_rms_columns<T>), dim3((d + 255) / 256, blocks), dim3(256), 0, st, A, blocks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_rms_backward_wide<T>), dim3(std::min(A.rows, kRmsWideBlocks)), dim3(kWide), 0, st, A);
  return hipGetLastError();
}

}  // namespace norm

// As norm_blocks (a few rows are summed by one workgroup, which saves a launch), with sixteen narrow rows a workgroup.
int rms_backward_blocks(int64_t rows, int64_t d, bool f32) {
  if (d > kNormMaxFused) return norm_blocks(rows, d, f32);
  const int64_t held = d <= norm::kNarrow ? 16 : d <= 1024 ? 4 : 1;
  if (rows <= 4 * held) return rows > 0;
  return int(std::min<int64_t>((rows + held - 1) / held, norm::most_lines(d, f32)));
}

hipError_t launch_rms(const RmsArgs& A, bool f32, hipStream_t st) {
  return f32 ? norm::rms_t<elem::F32>(A, st) : norm::rms_t<elem::Bf16>(A, st);
}

hipError_t launch_rms_backward(const RmsArgs& A, bool f32, int blocks, hipStream_t st) {
  return f32 ? norm::rms_backward_t<elem::F32>(A, blocks, st) : norm::rms_backward_t<elem::Bf16>(A, blocks, st);
}

}  // namespace tmk
