// What the norms' kernels share: sums over a row's threads, a row's and its
// columns' elements in registers, rows that are not held.
#pragma once

#include "tm_elem.h"
#include "tm_ops.h"

namespace tmk {
namespace norm {

using namespace elem;

// Sum of v over the NT threads of a row, in every one of them.  `slot` holds
// NT / 64 floats and is not used again before another barrier.
template <int NT, int N>
__device__ inline void row_sum(float (&v)[N], float* slot) {
  if constexpr (NT < 64) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int o = NT / 2; o > 0; o >>= 1) v[i] += __shfl_xor(v[i], o);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
  if constexpr (NT > 64) {
    constexpr int NW = NT / 64;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) slot[i * NW + (threadIdx.x >> 6)] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) s += slot[i * NW + w];
      v[i] = s;
    }
  }
}

template <int NT>
constexpr int block_threads() { return NT < 256 ? 256 : NT; }

template <int NT, int E, class T>
__device__ inline void load_cols(const float* p, float fill, int t, int d, float* v) {
#pragma unroll
  for (int j = 0; j < E / T::W; ++j) {
    const int c = (j * NT + t) * T::W;
    if (p != nullptr && c + T::W <= d) {
#pragma unroll
      for (int i = 0; i < T::W; i += F32::W) load_vec<F32>(reinterpret_cast<const char*>(p), c + i, d, fill, v + j * T::W + i);
    } else {
#pragma unroll
      for (int i = 0; i < T::W; ++i) v[j * T::W + i] = p != nullptr && c + i < d ? p[c + i] : fill;
    }
  }
}

// This thread's vectors of a row, as stored.
template <int NT, int V, class T, bool TAIL>
__device__ inline void load_row(const char* row, int t, int d, u32x4_t (&q)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) q[j] = load_ahead<T, TAIL>(row, (j * NT + t) * T::W, d);
}

// Threads of a row that is not held in registers.
constexpr int kWide = 1024;

template <class T, class F>
__device__ inline void each_vec(int d, F f) {
  for (int c = threadIdx.x * T::W; c < d; c += kWide * T::W) f(c);
}

__device__ inline float col(const float* p, float fill, int c, int d) { return p != nullptr && c < d ? p[c] : fill; }

}  // namespace norm
}  // namespace tmk
