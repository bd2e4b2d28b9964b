// Rows on their way to the experts' order and back, for gfx950.  Row i has `top` slots;
// a slot that is negative or past the filled rows is none.
//
//   gather    out[slot_ij] = x_i, zeros in the rows past the filled ones
//   combine   out_i = residual_i + sum_j w_ij y[slot_ij]
//   backward  dy[slot_ij] = w_ij dout_i (zeros past the filled rows),
//             dw_ij = sum over the columns of dout_i y[slot_ij]
//
// Each goes by the rows i: a row is read and written to its slots, or its slots are
// read and summed in the order of j, in fp32, and rounded once.  L threads have a row;
// they go along it 16 bytes at a time.  Up to eight slots (and weights) of a row are read once, by scalar loads
// where a wave or more has the row, and all of them are on the way together; what is read and
// written is what the definition asks for.  More go eight at a time: on the way out and backwards the row
// itself is read again for each eight, on the way back the slots are, for every 16 bytes.
//
// All three are bound by HBM (us; bytes at the 5.04 TB/s of a large copy in brackets): rows of 16384 x 4096 bf16 to two
// slots 68 to 76 (80, as the card writes faster than it copies), 8192 x 2048 bf16 joined from eight slots with residual 67
// (67), its backward 106 (113), backward of 3001 x 1023 fp32, three slots, 16.4 (16.1), of 32768 x 128 bf16, eight
// slots, 33 (29).  Few rows are the host's 7 to 10 us.
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

// Zeros in the rows past the filled ones, dealt out among the groups of L threads.
template <class T, int L>
__device__ inline void zero_rest(const RowsArgs& A, int64_t used) {
  constexpr int G = kThreads / L;
  const int t = threadIdx.x % L;
  float z[T::W] = {};
  for (int64_t p = used + int64_t(blockIdx.x) * G + threadIdx.x / L; p < A.count; p += int64_t(gridDim.x) * G)
    for (int c = t * T::W; c < A.d; c += L * T::W) store_vec<T>(A.out + p * A.ldo * T::kBytes, c, A.d, z);
}

// Row r, the same in every lane of a wave where L is a wave or more: what is read by it comes by scalar loads then.
template <int L>
__device__ inline int64_t row_of(int64_t r) {
  if constexpr (L < 64) return r;
  return int64_t(__builtin_amdgcn_readfirstlane(int(r >> 32))) << 32 | uint32_t(__builtin_amdgcn_readfirstlane(int(r)));
}

// K choices of a row, from `first` on: their places, or -1.
template <int K>
struct Choices {
  int64_t slot[K];
  float weight[K];
  __device__ void read(const RowsArgs& A, int64_t r, int first, int64_t used, bool weights) {
#pragma unroll
    for (int j = 0; j < K; ++j) {
      const int64_t i = r * A.top + first + j;
      slot[j] = first + j < A.top ? slot_of(A, i, used) : -1;
      weight[j] = 1.f;
      if (weights && slot[j] >= 0) weight[j] = A.weights[i];
    }
  }
};

// A row goes to its slots, K of them at a time: read once for all of them.  Bits are moved, not numbers.
template <class T, int L, int K>
__global__ __launch_bounds__(kThreads) void k_gather(const RowsArgs A) {
  constexpr int G = kThreads / L, W = T::W;
  const int t = threadIdx.x % L;
  const int64_t used = used_of(A);
  for (int64_t at = int64_t(blockIdx.x) * G + threadIdx.x / L; at < A.rows; at += int64_t(gridDim.x) * G) {
    const int64_t r = row_of<L>(at);
    const char* x = A.x + r * A.ldx * T::kBytes;
    for (int first = 0; first < A.top; first += K) {
      Choices<K> to;
      to.read(A, r, first, used, false);
      for (int c = t * W; c < A.d; c += L * W) {
        const uint32_t by = uint32_t(c) * T::kBytes;
        if (c + W <= A.d) {
          const u32x4_t q = T::load(x + by);
#pragma unroll
          for (int j = 0; j < K; ++j)
            if (to.slot[j] >= 0) T::store(A.out + to.slot[j] * A.ldo * T::kBytes + by, q);
        } else if (A.d >= W) {   // the row's last W elements: some are written a second time, as they are
          const uint32_t end = uint32_t(A.d - W) * T::kBytes;
          const u32x4_t q = T::load(x + end);
#pragma unroll
          for (int j = 0; j < K; ++j)
            if (to.slot[j] >= 0) T::store(A.out + to.slot[j] * A.ldo * T::kBytes + end, q);
        } else {
          typedef std::conditional_t<T::kBytes == 2, uint16_t, uint32_t> Bits;
          for (int i = 0; i < A.d - c; ++i) {
            const Bits v = reinterpret_cast<const Bits*>(x + by)[i];
#pragma unroll
            for (int j = 0; j < K; ++j)
              if (to.slot[j] >= 0) reinterpret_cast<Bits*>(A.out + to.slot[j] * A.ldo * T::kBytes + by)[i] = v;
          }
        }
      }
    }
  }
  zero_rest<T, L>(A, used);
}

// Elements c .. of a row, zeros past its end, from what load_ahead read.
template <class T>
__device__ inline void part(u32x4_t q, int c, int d, float* v) {
  if (d % T::W == 0) T::unpack(q, v);
  else T::unpack(settle<T, true>(q, c, d), v);
}

// K slots are read at a time; ONE: a row has no more, and its slots stay in registers.
template <class T, int L, int K, bool ONE>
__global__ __launch_bounds__(kThreads) void k_combine(const RowsArgs A) {
  constexpr int G = kThreads / L, W = T::W;
  const int t = threadIdx.x % L;
  const int64_t used = used_of(A);
  for (int64_t at = int64_t(blockIdx.x) * G + threadIdx.x / L; at < A.rows; at += int64_t(gridDim.x) * G) {
    const int64_t r = row_of<L>(at);
    Choices<K> from;
    if constexpr (ONE) from.read(A, r, 0, used, A.weights != nullptr);
    for (int c = t * W; c < A.d; c += L * W) {
      float acc[W] = {}, v[W];
      u32x4_t res = {0u, 0u, 0u, 0u};
      if (A.x != nullptr) res = load_ahead<T, true>(A.x + r * A.ldx * T::kBytes, c, A.d);
      for (int first = 0; first < (ONE ? 1 : A.top); first += K) {
        if constexpr (!ONE) from.read(A, r, first, used, A.weights != nullptr);
        u32x4_t q[K];
#pragma unroll
        for (int j = 0; j < K; ++j) {
          q[j] = u32x4_t{0u, 0u, 0u, 0u};
          if (from.slot[j] >= 0) q[j] = load_ahead<T, true>(A.y + from.slot[j] * A.ldy * T::kBytes, c, A.d);
        }
#pragma unroll
        for (int j = 0; j < K; ++j) {
          if (from.slot[j] < 0) continue;   // a weight that is not a number would show
          part<T>(q[j], c, A.d, v);
#pragma unroll
          for (int i = 0; i < W; ++i) acc[i] += from.weight[j] * v[i];
        }
      }
      if (A.x != nullptr) {
        part<T>(res, c, A.d, v);
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] += v[i];
      }
      store_vec<T>(A.out + r * A.ldo * T::kBytes, c, A.d, acc);
    }
  }
}

// Sums over the L threads of a row, in the first of them.  `slots`: LDS of K floats a wave, for rows of 256.
template <int L, int K>
__device__ inline void row_totals(float (&v)[K], float* slots) {
#pragma unroll
  for (int j = 0; j < K; ++j) {
    if constexpr (L >= 64) {
      v[j] = wave_sum(v[j]);
    } else {
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) v[j] += __shfl_xor(v[j], o);
    }
  }
  if constexpr (L > 64) {
    __syncthreads();   // the last row's are read
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int j = 0; j < K; ++j) slots[(threadIdx.x >> 6) * K + j] = v[j];
    __syncthreads();
    if (threadIdx.x == 0)
#pragma unroll
      for (int w = 1; w < L / 64; ++w)
#pragma unroll
        for (int j = 0; j < K; ++j) v[j] += slots[w * K + j];
  }
}

// The gradient's row is read once for K slots.  DOTS: with the weights' gradient.
template <class T, int L, int K, bool DOTS>
__global__ __launch_bounds__(kThreads) void k_combine_backward(const RowsArgs A) {
  constexpr int G = kThreads / L, W = T::W;
  __shared__ float slots[L > 64 ? L / 64 * K : 1];
  const int t = threadIdx.x % L;
  const int64_t used = used_of(A);
  for (int64_t at = int64_t(blockIdx.x) * G + threadIdx.x / L; at < A.rows; at += int64_t(gridDim.x) * G) {
    const int64_t r = row_of<L>(at);
    for (int first = 0; first < A.top; first += K) {
      Choices<K> to;
      to.read(A, r, first, used, A.weights != nullptr);
      float dot[K] = {};
      for (int c = t * W; c < A.d; c += L * W) {
        float g[W], v[W];
        u32x4_t q[K];
        const u32x4_t own = load_ahead<T, true>(A.x + r * A.ldx * T::kBytes, c, A.d);
        if constexpr (DOTS) {
#pragma unroll
          for (int j = 0; j < K; ++j) {
            q[j] = u32x4_t{0u, 0u, 0u, 0u};
            if (to.slot[j] >= 0) q[j] = load_ahead<T, true>(A.y + to.slot[j] * A.ldy * T::kBytes, c, A.d);
          }
        }
        part<T>(own, c, A.d, g);
#pragma unroll
        for (int j = 0; j < K; ++j) {
          if (to.slot[j] < 0) continue;
          if constexpr (DOTS) {
            part<T>(q[j], c, A.d, v);
#pragma unroll
            for (int i = 0; i < W; ++i) dot[j] += g[i] * v[i];
          }
#pragma unroll
          for (int i = 0; i < W; ++i) v[i] = g[i] * to.weight[j];
          store_vec<T>(A.out + to.slot[j] * A.ldo * T::kBytes, c, A.d, v);
        }
      }
      if constexpr (DOTS) {
        row_totals<L, K>(dot, slots);
#pragma unroll
        for (int j = 0; j < K; ++j)
          if (t == 0 && first + j < A.top) A.dweights[r * A.top + first + j] = to.slot[j] >= 0 ? dot[j] : 0.f;
      }
    }
  }
  zero_rest<T, L>(A, used);
}

// f(L) with the threads of a row: what wastes least of them, vecs being a row's 16-byte parts.  A wave of 64 up to 192
// (20000 rows of 125 parts to 4 slots: 41 us gathered and 45 joined, 51 and 59 with 256 threads a row; 129 parts: 30 and
// 40 against 31 and 52), 256 beyond (8192 rows of 256 parts, 8 slots: 53 and 66 us, a wave 74 and 72; 4096 columns to 2
// slots: 68, a wave 73; 16 such rows: 7 against 12); at 192 itself they are alike.  16 threads for the narrowest.
template <class T, class F>
void with_lanes(int d, F f) {
  const int vecs = (d + T::W - 1) / T::W;
  if (vecs <= 16) f(std::integral_constant<int, 16>{});
  else if (vecs <= 192) f(std::integral_constant<int, 64>{});
  else f(std::integral_constant<int, 256>{});
}

// f(K, whether a row has no more) with the slots that are gone through at a time: as many as there are, up to the eight
// whose vectors the registers hold (8192 x 2048 bf16 from eight slots: 67 us; one slot after the other 82).
template <class F>
void with_slots(int top, F f) {
  using std::integral_constant;
  if (top <= 2) f(integral_constant<int, 2>{}, std::true_type{});
  else if (top <= 4) f(integral_constant<int, 4>{}, std::true_type{});
  else if (top <= 8) f(integral_constant<int, 8>{}, std::true_type{});
  else f(integral_constant<int, 8>{}, std::false_type{});
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
    with_slots(A.top, [&](auto k, auto) {
      hipLaunchKernelGGL((k_gather<T, L, decltype(k)::value>), grid_of<L>(A.rows), dim3(kThreads), 0, st, A);
    });
  });
  return hipGetLastError();
}

template <class T>
hipError_t combine(const RowsArgs& A, hipStream_t st) {
  with_lanes<T>(A.d, [&](auto l) {
    constexpr int L = decltype(l)::value;
    with_slots(A.top, [&](auto k, auto one) {
      hipLaunchKernelGGL((k_combine<T, L, decltype(k)::value, decltype(one)::value>), grid_of<L>(A.rows), dim3(kThreads), 0, st, A);
    });
  });
  return hipGetLastError();
}

template <class T>
hipError_t combine_backward(const RowsArgs& A, hipStream_t st) {
  with_lanes<T>(A.d, [&](auto l) {
    constexpr int L = decltype(l)::value;
    with_slots(A.top, [&](auto k, auto) {
      constexpr int K = decltype(k)::value;
      if (A.dweights != nullptr) hipLaunchKernelGGL((k_combine_backward<T, L, K, true>), grid_of<L>(A.rows), dim3(kThreads), 0, st, A);
      else hipLaunchKernelGGL((k_combine_backward<T, L, K, false>), grid_of<L>(A.rows), dim3(kThreads), 0, st, A);
    });
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
