// Rows on their way to the experts' order and back, for gfx950.  Row i has `top` slots;
// a slot that is negative or past the filled rows is none.
//
//   gather    out[slot_ij] = x_i, zeros in the rows past the filled ones
//   combine   out_i = residual_i + sum_j w_ij y[slot_ij]
//   backward  dy[slot_ij] = w_ij dout_i (zeros past the filled rows),
//             dw_ij = sum over the columns of dout_i y[slot_ij]
//
// Each goes by the rows i: a row is read once and written to its slots, or its slots are
// read and summed in the order of j, in fp32, and rounded once.  L threads have a row;
// they go along it 16 bytes at a time.
#include <algorithm>

#include "tm_elem.h"
#include "tm_ops.h"

namespace tmk {
namespace rows {

using namespace elem;

constexpr int kThreads = 256;

// The place of choice i, -1 where it has none.  Whatever it holds, it lies within the filled rows.
__device__ inline int64_t slot_of(const RowsArgs& A, int64_t i, int64_t used) {
  const int s = A.slots[i];
  return s >= 0 && s < used ? s : -1;
}
__device__ inline int64_t used_of(const RowsArgs& A) {
  return A.used != nullptr ? min(max(int64_t(*A.used), int64_t(0)), A.count) : A.count;
}

// Elements first .. of a row as stored, whole vectors as they are.
template <class T>
__device__ inline void copy_vec(char* to, const char* from, int n, u32x4_t q, bool whole) {
  if (whole) {
    T::store(to, q);
  } else {
    for (int i = 0; i < n; ++i) T::store1(to + i * T::kBytes, T::load1(from + i * T::kBytes));
  }
}

// Zeros in the rows past the filled ones, dealt out among the groups of L threads.
template <class T, int L>
__device__ inline void zero_rest(const RowsArgs& A, int64_t used) {
  constexpr int G = kThreads / L;
  const int t = threadIdx.x % L;
  float z[T::W] = {};
  for (int64_t p = used + int64_t(blockIdx.x) * G + threadIdx.x / L; p < A.count; p += int64_t(gridDim.x) * G)
    for (int c = t * T::W; c < A.d; c += L * T::W) store_vec<T>(A.out + p * A.ldo * T::kBytes, c, A.d, z);
}

template <class T, int L>
__global__ __launch_bounds__(kThreads) void k_gather(const RowsArgs A) {
  constexpr int G = kThreads / L, W = T::W;
  const int t = threadIdx.x % L;
  const int64_t used = used_of(A);
  for (int64_t r = int64_t(blockIdx.x) * G + threadIdx.x / L; r < A.rows; r += int64_t(gridDim.x) * G) {
    const char* x = A.x + r * A.ldx * T::kBytes;
    for (int c = t * W; c < A.d; c += L * W) {
      const bool whole = c + W <= A.d;
      u32x4_t q = {0u, 0u, 0u, 0u};
      if (whole) q = T::load(x + int64_t(c) * T::kBytes);
      for (int j = 0; j < A.top; ++j) {
        const int64_t s = slot_of(A, r * A.top + j, used);
        if (s >= 0) copy_vec<T>(A.out + (s * A.ldo + c) * T::kBytes, x + int64_t(c) * T::kBytes, A.d - c, q, whole);
      }
    }
  }
  zero_rest<T, L>(A, used);
}

template <class T, int L>
__global__ __launch_bounds__(kThreads) void k_combine(const RowsArgs A) {
  constexpr int G = kThreads / L, W = T::W;
  const int t = threadIdx.x % L;
  for (int64_t r = int64_t(blockIdx.x) * G + threadIdx.x / L; r < A.rows; r += int64_t(gridDim.x) * G) {
    for (int c = t * W; c < A.d; c += L * W) {
      float acc[W] = {}, v[W];
      for (int j = 0; j < A.top; ++j) {
        const int64_t s = slot_of(A, r * A.top + j, A.count);
        if (s < 0) continue;
        const float w = A.weights != nullptr ? A.weights[r * A.top + j] : 1.f;
        load_vec<T>(A.y + s * A.ldy * T::kBytes, c, A.d, 0.f, v);
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] += w * v[i];
      }
      if (A.x != nullptr) {
        load_vec<T>(A.x + r * A.ldx * T::kBytes, c, A.d, 0.f, v);
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] += v[i];
      }
      store_vec<T>(A.out + r * A.ldo * T::kBytes, c, A.d, acc);
    }
  }
}

// Sum over the L threads of a row, in the first of them.
template <int L>
__device__ inline float row_total(float v, float* slots) {
#pragma unroll
  for (int o = (L < 64 ? L : 64) / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if constexpr (L > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slots[0];
#pragma unroll
    for (int w = 1; w < L / 64; ++w) v += slots[w];
  }
  return v;
}

template <class T, int L>
__global__ __launch_bounds__(kThreads) void k_combine_backward(const RowsArgs A) {
  constexpr int G = kThreads / L, W = T::W;
  __shared__ float slots[kThreads / 64];
  const int t = threadIdx.x % L;
  const int64_t used = used_of(A);
  for (int64_t r = int64_t(blockIdx.x) * G + threadIdx.x / L; r < A.rows; r += int64_t(gridDim.x) * G) {
    for (int j = 0; j < A.top; ++j) {
      const int64_t s = slot_of(A, r * A.top + j, used);
      float dot = 0.f;
      if (s >= 0) {
        const float w = A.weights != nullptr ? A.weights[r * A.top + j] : 1.f;
        for (int c = t * W; c < A.d; c += L * W) {
          float g[W], v[W];
          load_vec<T>(A.x + r * A.ldx * T::kBytes, c, A.d, 0.f, g);
          if (A.dweights != nullptr) {
            load_vec<T>(A.y + s * A.ldy * T::kBytes, c, A.d, 0.f, v);
#pragma unroll
            for (int i = 0; i < W; ++i) dot += g[i] * v[i];
          }
#pragma unroll
          for (int i = 0; i < W; ++i) g[i] *= w;
          store_vec<T>(A.out + s * A.ldo * T::kBytes, c, A.d, g);
        }
      }
      if (A.dweights != nullptr) {
        dot = row_total<L>(dot, slots);
        if (t == 0) A.dweights[r * A.top + j] = dot;
      }
    }
  }
  zero_rest<T, L>(A, used);
}

// f(L) with the threads of a row.
template <class T, class F>
void with_lanes(int d, F f) {
  const int vecs = (d + T::W - 1) / T::W;
  if (vecs <= 16) f(std::integral_constant<int, 16>{});
  else if (vecs <= 256) f(std::integral_constant<int, 64>{});
  else f(std::integral_constant<int, 256>{});
}

// Workgroups: a group of L threads for each row, or for each row past the filled ones.
template <int L>
dim3 grid_of(int64_t rows) {
  constexpr int G = kThreads / L;
  return dim3(uint32_t(std::clamp<int64_t>((rows + G - 1) / G, 1, 1 << 20)));
}

template <class T>
hipError_t gather(const RowsArgs& A, hipStream_t st) {
  with_lanes<T>(A.d, [&](auto l) {
    constexpr int L = decltype(l)::value;
    hipLaunchKernelGGL((k_gather<T, L>), grid_of<L>(A.rows), dim3(kThreads), 0, st, A);
  });
  return hipGetLastError();
}

template <class T>
hipError_t combine(const RowsArgs& A, hipStream_t st) {
  with_lanes<T>(A.d, [&](auto l) {
    constexpr int L = decltype(l)::value;
    hipLaunchKernelGGL((k_combine<T, L>), grid_of<L>(A.rows), dim3(kThreads), 0, st, A);
  });
  return hipGetLastError();
}

template <class T>
hipError_t combine_backward(const RowsArgs& A, hipStream_t st) {
  with_lanes<T>(A.d, [&](auto l) {
    constexpr int L = decltype(l)::value;
    hipLaunchKernelGGL((k_combine_backward<T, L>), grid_of<L>(A.rows), dim3(kThreads), 0, st, A);
  });
  return hipGetLastError();
}

}  // namespace rows

hipError_t launch_gather(const RowsArgs& A, bool f32, hipStream_t st) {
  return f32 ? rows::gather<elem::F32>(A, st) : rows::gather<elem::Bf16>(A, st);
}
hipError_t launch_combine(const RowsArgs& A, bool f32, hipStream_t st) {
  return f32 ? rows::combine<elem::F32>(A, st) : rows::combine<elem::Bf16>(A, st);
}
hipError_t launch_combine_backward(const RowsArgs& A, bool f32, hipStream_t st) {
  return f32 ? rows::combine_backward<elem::F32>(A, st) : rows::combine_backward<elem::Bf16>(A, st);
}

}  // namespace tmk
