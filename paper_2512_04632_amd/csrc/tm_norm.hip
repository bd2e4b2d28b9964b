// Layer norm over the rows of a matrix, forward and backward, for gfx950.
//
//   forward   mean = sum x / d,  rstd = 1 / sqrt(sum (x - mean)^2 / d + eps),
//             y = (x - mean) rstd weight + bias
//   backward  h = (x - mean) rstd,  g = dy weight,
//             dx = rstd (g - sum g / d - h sum(g h) / d),
//             dweight = sum over rows of dy h,  dbias = sum over rows of dy
//
// A row stays in the registers of the NT threads that own it (E elements
// each), so it is read once: the variance is the mean of the squared
// distances from the finished mean, with none of the cancellation that sums
// of squares have.  Each thread owns the same columns of every row it sees,
// so the backward pass keeps its share of the weight's and the bias's
// gradients in registers too; blocks go through the rows with a stride of the
// grid and write one line of partial sums each, which k_norm_params adds up in
// a fixed order (no atomics: results are the same on every run).  Statistics
// and sums are fp32; y and dx are rounded once.
//
// Bound by HBM once there are rows enough (16384 x 4096 bf16: forward 53.7 us, 5.0
// TB/s, what a large copy reaches; backward 83.9 us, 4.8 TB/s) and by the host's
// 8 us a call below some hundred rows (64 x 768: 4.1 us of kernel).
#include <algorithm>

#include "tm_norm.h"

namespace tmk {
namespace norm {

// Forward.  NT threads a row, E elements each (forward_t); TAIL: rows that end
// inside a 16-byte vector.  Two sums
// over the row's threads and the load are a chain that one row leaves idle: the
// next row is loaded while this one is summed (16384 x 4096 bf16: 47 us of kernel).
template <class T, int NT, int E, bool TAIL>
__global__ __launch_bounds__(block_threads<NT>()) void k_norm(const NormArgs A) {
  constexpr int W = T::W, V = E / W, RB = block_threads<NT>() / NT, NW = NT / 64;
  __shared__ float slots[2][NW];
  const int t = threadIdx.x % NT, d = A.d;
  const float n = float(d);
  float w[E], b[E];
  load_cols<NT, E, T>(A.weight, 1.f, t, d, w);
  load_cols<NT, E, T>(A.bias, 0.f, t, d, b);
  const int64_t step = int64_t(gridDim.x) * RB;
  int64_t r = int64_t(blockIdx.x) * RB + threadIdx.x / NT;
  u32x4_t q[V];
  if (r < A.rows) load_row<NT, V, T, TAIL>(A.x + r * A.ldx * T::kBytes, t, d, q);
  for (; r < A.rows; r += step) {
    float v[E], s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < V; ++j) {
      T::unpack(settle<T, TAIL>(q[j], (j * NT + t) * W, d), v + j * W);
#pragma unroll
      for (int i = 0; i < W; ++i) s[0] += v[j * W + i];
    }
    // the next row is on its way while this one is summed
    if (r + step < A.rows) load_row<NT, V, T, TAIL>(A.x + (r + step) * A.ldx * T::kBytes, t, d, q);
    row_sum<NT>(s, slots[0]);
    const float mean = s[0] / n;
    s[0] = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float c = (j * NT + t) * W + i < d ? v[j * W + i] - mean : 0.f;
        v[j * W + i] = c;
        s[0] += c * c;
      }
    row_sum<NT>(s, slots[1]);
    const float rstd = 1.f / sqrtf(s[0] / n + A.eps);
    if (t == 0) {
      A.mean[r] = mean;
      A.rstd[r] = rstd;
    }
    char* y = A.out + r * A.ldo * T::kBytes;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float o[W];
#pragma unroll
      for (int i = 0; i < W; ++i) o[i] = v[j * W + i] * rstd * w[j * W + i] + b[j * W + i];
      store_vec<T>(y, (j * NT + t) * W, d, o);
    }
  }
}

// Rows that wait in registers: one, or three of 16 bytes a thread (5999 x 1998
// bf16: 29 us, 47 with one); two of 32 bytes cost more in occupancy than they bring
// (16384 x 4096 bf16: 88 us, 84 with one).  1024 threads have no registers for any.
template <class T, int NT, int E>
constexpr int rows_ahead() { return NT == 1024 ? 0 : NT <= 256 && E * T::kBytes <= 16 ? 3 : 1; }

// Backward: x and dy are read once, dx written once; the columns' sums stay in
// registers over a workgroup's rows, so few workgroups write few lines of partial
// sums (norm_blocks).  16384 x 4096 bf16: 80 us of kernel for 403 MB, 5.0 TB/s; 4001 x
// 1001 fp32 16.8 us, 2.9 TB/s: rows of odd length, four a workgroup, are bound by
// their chains of loads and sums.
template <class T, int NT, int E, bool TAIL>
__global__ __launch_bounds__(block_threads<NT>()) void k_norm_backward(const NormArgs A) {
  constexpr int W = T::W, V = E / W, RB = block_threads<NT>() / NT, NW = NT / 64;
  constexpr int AHEAD = rows_ahead<T, NT, E>(), D = AHEAD > 0 ? AHEAD : 1;
  __shared__ float slots[2][2 * NW];
  const int t = threadIdx.x % NT, d = A.d;
  const float n = float(d);
  float w[E], aw[E], ab[E];
  load_cols<NT, E, T>(A.weight, 1.f, t, d, w);
#pragma unroll
  for (int i = 0; i < E; ++i) aw[i] = ab[i] = 0.f;
  const int64_t step = int64_t(gridDim.x) * RB;
  int64_t r = int64_t(blockIdx.x) * RB + threadIdx.x / NT;
  u32x4_t qx[D][V], qy[D][V];
  float mean[D], rstd[D];
  auto read = [&](int u, int64_t at) __attribute__((always_inline)) {
    load_row<NT, V, T, TAIL>(A.x + at * A.ldx * T::kBytes, t, d, qx[u]);
    load_row<NT, V, T, TAIL>(A.dy + at * A.lddy * T::kBytes, t, d, qy[u]);
    mean[u] = A.mean[at];
    rstd[u] = A.rstd[at];
  };
  if constexpr (AHEAD > 0) {
#pragma unroll
    for (int u = 0; u < D; ++u)
      if (r + u * step < A.rows) read(u, r + u * step);
  }
  int turn = 0;
  while (r < A.rows) {
#pragma unroll
    for (int u = 0; u < D; ++u) {
      if (r >= A.rows) break;
      if constexpr (AHEAD == 0) read(u, r);
      float h[E], g[E], s[2] = {0.f, 0.f};
      const float m = mean[u], scale = rstd[u];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int c = (j * NT + t) * W;
        T::unpack(settle<T, TAIL>(qx[u][j], c, d), h + j * W);
        T::unpack(settle<T, TAIL>(qy[u][j], c, d), g + j * W);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const int e = j * W + i;
          h[e] = c + i < d ? (h[e] - m) * scale : 0.f;
          aw[e] += g[e] * h[e];
          ab[e] += g[e];
          g[e] *= w[e];
          s[0] += g[e];
          s[1] += g[e] * h[e];
        }
      }
      if (AHEAD > 0 && r + D * step < A.rows) read(u, r + D * step);
      row_sum<NT>(s, slots[turn]);
      turn ^= 1;
      const float m0 = s[0] / n, m1 = s[1] / n;
      char* dx = A.out + r * A.ldo * T::kBytes;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float o[W];
#pragma unroll
        for (int i = 0; i < W; ++i) o[i] = scale * (g[j * W + i] - m0 - h[j * W + i] * m1);
        store_vec<T>(dx, (j * NT + t) * W, d, o);
      }
      r += step;
    }
  }
  // the sums of the block's rows: to its line of partial sums, or as the result
  float *to_w = A.dweight, *to_b = A.dbias;
  if (A.part != nullptr) {
    to_w = A.part + int64_t(blockIdx.x) * 2 * d;
    to_b = to_w + d;
  }
  if (to_w == nullptr && to_b == nullptr) return;
  auto put = [&](int c, float sw, float sb) {
    if (c >= d) return;
    if (to_w != nullptr) to_w[c] = sw;
    if (to_b != nullptr) to_b[c] = sb;
  };
  if constexpr (RB > 1) {   // the waves' rows first, one after the other
    __shared__ float sums[2 * NT * E];
    for (int q = 0; q < RB; ++q) {
      if (int(threadIdx.x) / NT == q)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int at = (e / W * NT + t) * W + e % W;
          sums[at] = (q > 0 ? sums[at] : 0.f) + aw[e];
          sums[NT * E + at] = (q > 0 ? sums[NT * E + at] : 0.f) + ab[e];
        }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < d; c += block_threads<NT>()) put(c, sums[c], sums[NT * E + c]);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) put((e / W * NT + t) * W + e % W, aw[e], ab[e]);
  }
}

// Rows wider than a workgroup's registers (kNormMaxFused): one workgroup of
// 1024 threads per row, which reads the row once for each sum and once for the
// result (the later passes find it in a cache).  4096 x 20000 bf16 313 us, 1.05 TB/s of
// what has to move: three passes, and loops that fetch weight and bias an element at a time.
template <class T>
__global__ __launch_bounds__(kWide) void k_norm_wide(const NormArgs A) {
  __shared__ float slots[2][kWide / 64];
  const int d = A.d;
  const float n = float(d);
  for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x) {
    const char* x = A.x + r * A.ldx * T::kBytes;
    char* y = A.out + r * A.ldo * T::kBytes;
    float s[1] = {0.f}, v[T::W];
    each_vec<T>(d, [&](int c) {
      load_vec<T>(x, c, d, 0.f, v);
#pragma unroll
      for (int i = 0; i < T::W; ++i) s[0] += v[i];
    });
    row_sum<kWide>(s, slots[0]);
    const float mean = s[0] / n;
    s[0] = 0.f;
    each_vec<T>(d, [&](int c) {
      load_vec<T>(x, c, d, mean, v);
#pragma unroll
      for (int i = 0; i < T::W; ++i) s[0] += (v[i] - mean) * (v[i] - mean);
    });
    row_sum<kWide>(s, slots[1]);
    const float rstd = 1.f / sqrtf(s[0] / n + A.eps);
    if (threadIdx.x == 0) {
      A.mean[r] = mean;
      A.rstd[r] = rstd;
    }
    each_vec<T>(d, [&](int c) {
      load_vec<T>(x, c, d, mean, v);
#pragma unroll
      for (int i = 0; i < T::W; ++i)
        v[i] = (v[i] - mean) * rstd * col(A.weight, 1.f, c + i, d) + col(A.bias, 0.f, c + i, d);
      store_vec<T>(y, c, d, v);
    });
  }
}

// The same backwards: 4096 x 20000 bf16 410 us with the column sums.
template <class T>
__global__ __launch_bounds__(kWide) void k_norm_backward_wide(const NormArgs A) {
  __shared__ float slots[2][2 * kWide / 64];
  const int d = A.d;
  const float n = float(d);
  int turn = 0;
  for (int64_t r = blockIdx.x; r < A.rows; r += gridDim.x) {
    const char* x = A.x + r * A.ldx * T::kBytes;
    const char* dy = A.dy + r * A.lddy * T::kBytes;
    char* dx = A.out + r * A.ldo * T::kBytes;
    const float mean = A.mean[r], rstd = A.rstd[r];
    float s[2] = {0.f, 0.f}, h[T::W], g[T::W];
    auto read = [&](int c) {
      load_vec<T>(x, c, d, mean, h);
      load_vec<T>(dy, c, d, 0.f, g);
#pragma unroll
      for (int i = 0; i < T::W; ++i) {
        h[i] = (h[i] - mean) * rstd;
        g[i] *= col(A.weight, 1.f, c + i, d);
      }
    };
    each_vec<T>(d, [&](int c) {
      read(c);
#pragma unroll
      for (int i = 0; i < T::W; ++i) {
        s[0] += g[i];
        s[1] += g[i] * h[i];
      }
    });
    row_sum<kWide>(s, slots[turn]);
    turn ^= 1;
    const float m0 = s[0] / n, m1 = s[1] / n;
    each_vec<T>(d, [&](int c) {
      read(c);
#pragma unroll
      for (int i = 0; i < T::W; ++i) g[i] = rstd * (g[i] - m0 - h[i] * m1);
      store_vec<T>(dx, c, d, g);
    });
  }
}

// Column sums of such rows: one thread per column, each block a slice of the
// rows (x and dy are read once more).
template <class T>
__global__ __launch_bounds__(256) void k_norm_columns(const NormArgs A, int slices) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= A.d) return;
  float aw = 0.f, ab = 0.f;
  for (int64_t r = blockIdx.y; r < A.rows; r += slices) {
    const float g = T::load1(A.dy + (r * A.lddy + c) * T::kBytes);
    const float x = T::load1(A.x + (r * A.ldx + c) * T::kBytes);
    aw += g * ((x - A.mean[r]) * A.rstd[r]);
    ab += g;
  }
  float* part = A.part + int64_t(blockIdx.y) * 2 * A.d;
  part[c] = aw;
  part[A.d + c] = ab;
}

// out[c] = sum of the blocks' partial sums of column c (`lines` of them a block): 32 columns a block, 32
// threads each.  Bound by latency: 512 lines of 4096 columns, 16 MB, 4.5 us.
__global__ __launch_bounds__(1024) void k_norm_params(const float* part, int blocks, int lines, int d, float* dweight,
                                                      float* dbias) {
  float* out = blockIdx.y == 0 ? dweight : dbias;
  if (out == nullptr) return;
  constexpr int G = 32;
  __shared__ float sums[G][33];
  const int lc = threadIdx.x & 31, grp = threadIdx.x >> 5, c = blockIdx.x * 32 + lc;
  float s = 0.f;
  if (c < d) {
#pragma unroll 4
    for (int b = grp; b < blocks; b += G) s += part[(int64_t(b) * lines + blockIdx.y) * d + c];
  }
  sums[lc][grp] = s;
  __syncthreads();
  // a half wave per column
  s = sums[grp][lc];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor(s, o);
  const int col = blockIdx.x * 32 + grp;
  if (lc == 0 && col < d) out[col] = s;
}

// Workgroups of the forward pass (times of the whole call in us, bf16, inputs in
// turn): rows of 512 threads have two a compute unit (8192 x 8192: 46, 50 with
// 2048 workgroups), of 1024 one (4096 x 16384: 49, 69 with 2048), so that each goes
// through many rows, the next one on its way; narrower ones eight (16384 x 768: 12.5, 13.5
// with 512, 14.3 with a row each).
int forward_blocks(int d) { return d <= 4096 ? 2048 : d <= 8192 ? 512 : 256; }
constexpr int kWideBlocks = 2048;   // 4096 x 20000: 313, the same with 512 and 16384

template <class T, int NT, int E>
hipError_t forward(const NormArgs& A, hipStream_t st) {
  constexpr int RB = block_threads<NT>() / NT;
  const int blocks = int(std::min<int64_t>((int64_t(A.rows) + RB - 1) / RB, forward_blocks(A.d)));
  if (A.d % T::W == 0) hipLaunchKernelGGL((k_norm<T, NT, E, false>), dim3(blocks), dim3(block_threads<NT>()), 0, st, A);
  else hipLaunchKernelGGL((k_norm<T, NT, E, true>), dim3(blocks), dim3(block_threads<NT>()), 0, st, A);
  return hipGetLastError();
}

template <class T, int NT, int E>
hipError_t backward(const NormArgs& A, int blocks, hipStream_t st) {
  const dim3 grid(blocks), block(block_threads<NT>());
  if (A.d % T::W == 0) hipLaunchKernelGGL((k_norm_backward<T, NT, E, false>), grid, block, 0, st, A);
  else hipLaunchKernelGGL((k_norm_backward<T, NT, E, true>), grid, block, 0, st, A);
  return hipGetLastError();
}

// Threads for a row, and how many elements each holds: as few threads as hold it
// (us, bf16, forward and backward: 8192 x 512 on 64 threads of 8: 5.6 and 11.6, of 16:
// 7.9 and 13.6; 8192 x 1024 on 64: 8.3 and 16.1, on 256: 13.4 and 24.3; 8192 x 2048 on 256 of
// 8: 14.4 and 29.0, of 16: 19.2 and 33.6; 4096 x 4096 on 256: 13.4 and 31.5, on 512: 23.1
// and 39.0; 4096 x 8192 on 512: 25.6 and 46.8, on 1024: 46.5 and 62.1; 2048 x 16384 on
// 1024: 33 and 61, not held: 130 and 161).
template <class T>
hipError_t forward_t(const NormArgs& A, hipStream_t st) {
  const int d = A.d;
  if (d <= 512) return forward<T, 64, 8>(A, st);
  if (d <= 1024) return forward<T, 64, 16>(A, st);
  if (d <= 2048) return forward<T, 256, 8>(A, st);
  if (d <= 4096) return forward<T, 256, 16>(A, st);
  if (d <= 8192) return forward<T, 512, 16>(A, st);
  if (d <= kNormMaxFused) return forward<T, 1024, 16>(A, st);
  hipLaunchKernelGGL((k_norm_wide<T>), dim3(std::min(A.rows, kWideBlocks)), dim3(kWide), 0, st, A);
  return hipGetLastError();
}

template <class T>
hipError_t backward_t(const NormArgs& A, int blocks, hipStream_t st) {
  const int d = A.d;
  if (d <= 512) return backward<T, 64, 8>(A, blocks, st);
  if (d <= 1024) return backward<T, 64, 16>(A, blocks, st);
  if (d <= 2048) return backward<T, 256, 8>(A, blocks, st);
  if (d <= 4096) return backward<T, 256, 16>(A, blocks, st);
  if (d <= 8192) return backward<T, 512, 16>(A, blocks, st);
  if (d <= kNormMaxFused) return backward<T, 1024, 16>(A, blocks, st);
  // dx may take the place of x or dy, so the column sums come first
  if (A.part != nullptr) {
    hipLaunchKernelGGL((k_norm_columns<T>), dim3((d + 255) / 256, blocks), dim3(256), 0, st, A, blocks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_norm_backward_wide<T>), dim3(std::min(A.rows, kWideBlocks)), dim3(kWide), 0, st, A);
  return hipGetLastError();
}

}  // namespace norm

hipError_t launch_norm(const NormArgs& A, bool f32, hipStream_t st) {
  return f32 ? norm::forward_t<elem::F32>(A, st) : norm::forward_t<elem::Bf16>(A, st);
}

// Workgroups of the backward pass: each leaves a line of partial sums.  Two a
// compute unit, or one where the rows' registers leave room for no more (us, 512
// against 256 workgroups: 32768 x 2048 bf16 84 and 101; 16384 x 3000 fp32 120 and 109;
// 8192 x 8192 bf16 98 and 86; 1024 of them: 16384 x 768 bf16 24, 21 with 512); rows that
// are not held, with their column sums apart: 4096 x 20000 bf16 417, 409 with 128, 442 with 32.
int norm_blocks(int64_t rows, int64_t d, bool f32) {
  const int rb = d <= 1024 ? 4 : 1;
  // a few rows are summed by one workgroup: as fast (8 x 4096 bf16: 9.0 us both
  // ways, 13.4 and 9.1 from eight rows a wave on), and one launch less for the host
  if (d <= kNormMaxFused && rows > 0 && rows <= 4 * rb) return 1;
  const int most = d > kNormMaxFused ? 64 : d > (f32 ? 1024 : 4096) ? 256 : 512;
  return int(std::min<int64_t>((rows + rb - 1) / rb, most));
}

hipError_t launch_norm_backward(const NormArgs& A, bool f32, int blocks, hipStream_t st) {
  return f32 ? norm::backward_t<elem::F32>(A, blocks, st) : norm::backward_t<elem::Bf16>(A, blocks, st);
}

hipError_t launch_norm_params(const float* part, int blocks, int lines, int d, float* dweight, float* dbias,
                              hipStream_t st) {
  hipLaunchKernelGGL(norm::k_norm_params, dim3((d + 31) / 32, lines), dim3(1024), 0, st, part, blocks, lines, d, dweight, dbias);
  return hipGetLastError();
}

}  // namespace tmk
