// Routing of rows to experts, with the balance loss, forward and backward, for gfx950.
//
// Row i of N that take part has scores l over E experts; p = softmax(l).
//
//   chosen    the `top` largest l, of equal ones the lowest index (NaN counts as -inf)
//   weights   w_j = scale p_j, over the sum of the chosen p where renormalised
//   slots     the choices' places in the experts' order: by expert, then by row
//   ends      c_0 + .. + c_e, with c_e the choices of expert e
//   balance   E sum_e f_e P_e,  f_e = c_e / (top N),  P_e = sum of p_e over the rows / N
//   gradient  u_e = dbalance E f_e / N, and scale dw_j added at the chosen where they are not
//             renormalised: dl = p (u - sum p u); renormalised, the chosen share a softmax of
//             their own, q = w / scale: q_j (scale dw_j - sum q scale dw) is added at them
//
// Forward in two launches.  The first holds each row in the registers of L lanes, which
// take the maximum `top` times; a block marks a choice with the row's bit in a word of 64 per
// expert, so that a choice's place among the block's is a count of the bits below it, and
// no order of atomics shows.  The second adds up the blocks' counts (16 bits each) and moves every
// choice by what lies before its block.  Sums of probabilities are fp32 over a block's rows,
// 64-bit over the blocks, in a fixed order.
#include <algorithm>

#include "tm_elem.h"
#include "tm_ops.h"

namespace tmk {
namespace route {

using namespace elem;

constexpr int kThreads = 256, kRows = kRouteRows;

// A reduction over the L lanes of a row, in each of them.  `slot`: LDS of a row of 256.
template <int L, class V, class F>
__device__ inline V over_row(V v, V* slot, F f) {
#pragma unroll
  for (int o = (L < 64 ? L : 64) / 2; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o));
  if constexpr (L > 64) {
    __syncthreads();   // the last use of the slot is over
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slot[0];
#pragma unroll
    for (int w = 1; w < L / 64; ++w) v = f(v, slot[w]);
  }
  return v;
}

template <int L>
struct Slots {
  float f[L > 64 ? L / 64 : 1];
  int i[L > 64 ? L / 64 : 1];
};
template <int L>
__device__ inline float row_max(float v, Slots<L>& s) { return over_row<L>(v, s.f, [](float a, float b) { return fmaxf(a, b); }); }
template <int L>
__device__ inline float row_sum(float v, Slots<L>& s) { return over_row<L>(v, s.f, [](float a, float b) { return a + b; }); }
template <int L>
__device__ inline int row_max(int v, Slots<L>& s) { return over_row<L>(v, s.i, [](int a, int b) { return max(a, b); }); }
template <int L>
__device__ inline int row_min(int v, Slots<L>& s) { return over_row<L>(v, s.i, [](int a, int b) { return min(a, b); }); }

// Whole numbers in the order of the floats; -0 is 0, NaN is -inf.
__device__ inline int ordered(float v) {
  const int b = __float_as_int(v > -INFINITY ? v + 0.f : -INFINITY);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ inline float value_of(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7fffffff)); }

// L lanes a row, J vectors each: element (j L + t) W + i of the row is number j W + i of lane t.
template <class T, int L, int J>
struct Held {
  static constexpr int W = T::W, N = J * W, MOST = L * N;
  __device__ static int place(int t, int n) { return ((n / W) * L + t) * W + n % W; }
  __device__ static void load(const char* row, int t, int experts, float* v) {
#pragma unroll
    for (int j = 0; j < J; ++j) load_vec<T>(row, (j * L + t) * W, experts, -INFINITY, v + j * W);
  }
};

template <class T, int L, int J>
__global__ __launch_bounds__(kThreads) void k_route(const RouteArgs A) {
  using H = Held<T, L, J>;
  constexpr int N = H::N, G = kThreads / L;
  __shared__ uint64_t mask[H::MOST];
  __shared__ int before[H::MOST];
  __shared__ float share[kRows * TM_MAX_TOP], whole[kRows];
  __shared__ uint16_t sel[kRows * TM_MAX_TOP];
  __shared__ Slots<L> slots;
  const int t = threadIdx.x % L, grp = threadIdx.x / L, experts = A.experts, top = A.top;
  float acc[N];
#pragma unroll
  for (int n = 0; n < N; ++n) acc[n] = 0.f;
  for (int e = threadIdx.x; e < experts; e += kThreads) before[e] = 0;
  for (int turn = 0; turn < A.turns; ++turn) {
    const int64_t first = (int64_t(blockIdx.x) * A.turns + turn) * kRows;
    const int rows = int(min(int64_t(kRows), A.rows - first));
    if (rows <= 0) break;
    for (int e = threadIdx.x; e < experts; e += kThreads) mask[e] = 0;
    __syncthreads();
    for (int at = grp; at < rows; at += G) {
      const int64_t r = first + at;
      if (A.active != nullptr && A.active[r] == 0) {
        if (t == 0) whole[at] = -1.f;
        continue;
      }
      float v[N];
      H::load(A.logits + r * A.ld * T::kBytes, t, experts, v);
      float m = v[0];
#pragma unroll
      for (int n = 1; n < N; ++n) m = fmaxf(m, v[n]);
      m = row_max<L>(m, slots);
      int key[N];
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const bool there = H::place(t, n) < experts;
        key[n] = there ? ordered(v[n]) : INT32_MIN;
        v[n] = there ? expf(v[n] - m) : 0.f;
        sum += v[n];
      }
      sum = row_sum<L>(sum, slots);
      const float inv = 1.f / sum;
#pragma unroll
      for (int n = 0; n < N; ++n) acc[n] += v[n] * inv;
      float chosen = 0.f;
      for (int j = 0; j < top; ++j) {
        int best = key[0], place = 0;
#pragma unroll
        for (int n = 1; n < N; ++n)
          if (key[n] > best) {
            best = key[n];
            place = n;
          }
        const int most = row_max<L>(best, slots);
        const int mine = best == most ? H::place(t, place) : INT32_MAX;
        const int e = row_min<L>(mine, slots);
#pragma unroll
        for (int n = 0; n < N; ++n)
          if (e == mine && n == place) key[n] = INT32_MIN;
        const float p = expf(value_of(most) - m);
        chosen += p;
        if (t == 0) {
          sel[at * top + j] = uint16_t(e);
          share[at * top + j] = p;
          atomicOr((unsigned long long*)&mask[e], 1ull << at);
        }
      }
      // a sum that is not a number shows in the weights either way
      if (t == 0) whole[at] = A.renormalize ? chosen + 0.f * sum : sum;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * top; i += kThreads) {
      const int at = i / top;
      const int64_t out = first * top + i;
      if (whole[at] == -1.f) {
        A.chosen[out] = A.slots[out] = -1;
        A.weights[out] = 0.f;
        continue;
      }
      const int e = sel[i];
      A.chosen[out] = e;
      A.weights[out] = A.scale * (share[i] / whole[at]);
      A.slots[out] = before[e] + __popcll(mask[e] & ((1ull << at) - 1));
    }
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += kThreads) before[e] += __popcll(mask[e]);
  }
  // the groups' sums, one after the other, in the words that the last turn leaves free
  float* sums = reinterpret_cast<float*>(mask);
  for (int q = 0; q < G; ++q) {
    __syncthreads();
    if (grp == q)
#pragma unroll
      for (int n = 0; n < N; ++n) sums[H::place(t, n)] = (q > 0 ? sums[H::place(t, n)] : 0.f) + acc[n];
  }
  __syncthreads();
  const int width = (experts + 7) / 8 * 8;
  for (int e = threadIdx.x; e < width; e += kThreads) {
    A.counts[int64_t(blockIdx.x) * width + e] = uint16_t(e < experts ? before[e] : 0);
    A.shares[int64_t(blockIdx.x) * width + e] = e < experts ? sums[e] : 0.f;
  }
}

constexpr int kPlace = 1024;

// `span` blocks of k_route a workgroup; the first writes ends, the last the balance loss.
template <int MOST>
__global__ __launch_bounds__(kPlace) void k_route_place(const RouteArgs A, int span) {
  __shared__ int total[MOST], base[MOST], waves[kPlace / 64];
  __shared__ double parts[kPlace / 64];
  const int experts = A.experts, width = (experts + 7) / 8 * 8, tid = threadIdx.x, lane = tid & 63;
  const int own = int(blockIdx.x) * span;
  for (int e = tid; e < width; e += kPlace) total[e] = base[e] = 0;
  __syncthreads();
  // the blocks' counts: vectors of eight experts, the blocks dealt out among the threads
  const int vecs = width / 8, segments = max(kPlace / vecs, 1);
  for (int at = tid; at < vecs * segments; at += kPlace) {
    const int v = at % vecs;
    int all[8] = {}, low[8] = {};
    for (int b = at / vecs; b < A.blocks; b += segments) {
      const u32x4_t q = *reinterpret_cast<const u32x4_t*>(A.counts + int64_t(b) * width + v * 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int n = int(i % 2 ? q[i / 2] >> 16 : q[i / 2] & 0xffffu);
        all[i] += n;
        if (b < own) low[i] += n;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (all[i] != 0) atomicAdd(&total[v * 8 + i], all[i]);
      if (low[i] != 0) atomicAdd(&base[v * 8 + i], low[i]);
    }
  }
  __syncthreads();
  // exclusive sums of the totals: PER neighbouring experts a thread
  constexpr int PER = (MOST + kPlace - 1) / kPlace;
  int mine[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    mine[i] = tid * PER + i < experts ? total[tid * PER + i] : 0;
    sum += mine[i];
  }
  int scan = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(scan, o);
    if (lane >= o) scan += up;
  }
  if (lane == 63) waves[tid >> 6] = scan;
  __syncthreads();
  int start = scan - sum, used = 0;
#pragma unroll
  for (int w = 0; w < kPlace / 64; ++w) {
    if (w < tid >> 6) start += waves[w];
    used += waves[w];
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = tid * PER + i;
    if (e >= experts) continue;
    base[e] += start;
    start += mine[i];
    if (blockIdx.x == 0) A.ends[e] = start;
  }
  for (int b = own; b < min(own + span, A.blocks); ++b) {
    __syncthreads();
    const int64_t first = int64_t(b) * A.turns * kRows * A.top;
    const int64_t last = min(first + int64_t(A.turns) * kRows * A.top, int64_t(A.rows) * A.top);
    for (int64_t i = first + tid; i < last; i += kPlace) {
      const int e = A.chosen[i];
      if (e >= 0) A.slots[i] += base[e];
    }
    __syncthreads();
    for (int e = tid; e < experts; e += kPlace) base[e] += A.counts[int64_t(b) * width + e];
  }
  if (blockIdx.x + 1 != gridDim.x) return;
  double dot = 0.0;
  for (int at = tid; at < vecs * segments; at += kPlace) {
    const int v = at % vecs;
    double s[8] = {};
    for (int b = at / vecs; b < A.blocks; b += segments) {
      const float* from = A.shares + int64_t(b) * width + v * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += double(from[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) dot += s[i] * double(total[v * 8 + i]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
  if (lane == 0) parts[tid >> 6] = dot;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kPlace / 64; ++w) dot += parts[w];
    const double rows = double(used) / double(A.top);
    *A.balance = used > 0 ? float(double(experts) * dot / (double(used) * rows)) : 0.f;
  }
}

template <class T, int L, int J>
__global__ __launch_bounds__(kThreads) void k_route_backward(const RouteGradArgs A) {
  using H = Held<T, L, J>;
  constexpr int N = H::N, G = kThreads / L;
  __shared__ Slots<L> slots;
  const int t = threadIdx.x % L, experts = A.experts, top = A.top;
  const float used = float(A.ends[experts - 1]), taking = used / float(top);
  const float per = A.dbalance != nullptr && used > 0.f ? *A.dbalance * float(experts) / (used * taking) : 0.f;
  float u[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int e = H::place(t, n);
    u[n] = e < experts ? per * float(A.ends[e] - (e > 0 ? A.ends[e - 1] : 0)) : 0.f;
  }
  for (int64_t r = int64_t(blockIdx.x) * G + threadIdx.x / L; r < A.rows; r += int64_t(gridDim.x) * G) {
    const char* row = A.logits + r * A.ld * T::kBytes;
    char* out = A.dlogits + r * A.ldd * T::kBytes;
    const int32_t* chosen = A.chosen + r * top;
    const float* dw = A.dweights != nullptr ? A.dweights + r * top : nullptr;
    float v[N], g[N], add[N];
    const bool on = chosen[0] >= 0;
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = add[n] = 0.f;
    if (on) {
      H::load(row, t, experts, v);
      float m = v[0];
#pragma unroll
      for (int n = 1; n < N; ++n) m = fmaxf(m, v[n]);
      m = row_max<L>(m, slots);
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        v[n] = H::place(t, n) < experts ? expf(v[n] - m) : 0.f;
        sum += v[n];
        g[n] = u[n];
      }
      sum = row_sum<L>(sum, slots);
      const float inv = 1.f / sum;
      if (dw != nullptr) {
        float most = -INFINITY, whole = 0.f, mean = 0.f;
        if (A.renormalize) {   // about the chosen's own maximum
          for (int j = 0; j < top; ++j) {
            const int e = chosen[j];
            if (e < 0 || e >= experts) continue;
            const float l = T::load1(row + int64_t(e) * T::kBytes);
            if (l > most) most = l;
          }
          for (int j = 0; j < top; ++j) {
            const int e = chosen[j];
            if (e < 0 || e >= experts) continue;
            const float q = expf(T::load1(row + int64_t(e) * T::kBytes) - most);
            whole += q;
            mean += q * (A.scale * dw[j]);
          }
          mean /= whole;
        }
        for (int j = 0; j < top; ++j) {
          const int e = chosen[j];
          if (e < 0 || e >= experts) continue;
          float at = A.scale * dw[j];
          if (A.renormalize) at = expf(T::load1(row + int64_t(e) * T::kBytes) - most) / whole * (at - mean);
#pragma unroll
          for (int n = 0; n < N; ++n)
            if (H::place(t, n) == e) (A.renormalize ? add[n] : g[n]) += at;
        }
      }
      float dot = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        v[n] *= inv;
        dot += v[n] * g[n];
      }
      dot = row_sum<L>(dot, slots);
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] = v[n] * (g[n] - dot) + add[n];
    }
#pragma unroll
    for (int j = 0; j < J; ++j) store_vec<T>(out, (j * L + t) * T::W, experts, v + j * T::W);
  }
}

// f(L, J) with the lanes of a row and vectors of each that hold `experts`.
template <class T, class F>
void with_shape(int experts, F f) {
  using std::integral_constant;
  constexpr int W = T::W;
  if (experts <= 16 * W) f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  else if (experts <= 128) f(integral_constant<int, 16>{}, integral_constant<int, 8 / W>{});
  else if (experts <= 256) f(integral_constant<int, 16>{}, integral_constant<int, 16 / W>{});
  else if (experts <= 1024) f(integral_constant<int, 64>{}, integral_constant<int, 16 / W>{});
  else f(integral_constant<int, 256>{}, integral_constant<int, 32 / W>{});
}

template <class T>
hipError_t forward(const RouteArgs& A, hipStream_t st) {
  with_shape<T>(A.experts, [&](auto l, auto j) {
    hipLaunchKernelGGL((k_route<T, decltype(l)::value, decltype(j)::value>), dim3(A.blocks), dim3(kThreads), 0, st, A);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int span = (A.blocks + 127) / 128;
  const dim3 grid((A.blocks + span - 1) / span);
  if (A.experts <= 1024) hipLaunchKernelGGL((k_route_place<1024>), grid, dim3(kPlace), 0, st, A, span);
  else hipLaunchKernelGGL((k_route_place<TM_MAX_EXPERTS>), grid, dim3(kPlace), 0, st, A, span);
  return hipGetLastError();
}

template <class T>
hipError_t backward(const RouteGradArgs& A, hipStream_t st) {
  with_shape<T>(A.experts, [&](auto l, auto j) {
    constexpr int G = kThreads / decltype(l)::value;
    const dim3 grid(uint32_t(std::min<int64_t>((int64_t(A.rows) + G - 1) / G, 2048)));
    hipLaunchKernelGGL((k_route_backward<T, decltype(l)::value, decltype(j)::value>), grid, dim3(kThreads), 0, st, A);
  });
  return hipGetLastError();
}

}  // namespace route

void plan_route(RouteArgs& A) {
  // every workgroup of the second launch reads all counts: fewer blocks where there are many experts
  const int64_t runs = std::max<int64_t>((int64_t(A.rows) + kRouteRows - 1) / kRouteRows, 1);
  const int64_t most = std::clamp<int64_t>((1 << 18) / A.experts, 64, 1024);
  const int64_t turns = std::min<int64_t>((runs + most - 1) / most, 65535 / kRouteRows);
  A.turns = int32_t(turns);
  A.blocks = int32_t((runs + turns - 1) / turns);
}

hipError_t launch_route(const RouteArgs& A, bool f32, hipStream_t st) {
  return f32 ? route::forward<elem::F32>(A, st) : route::forward<elem::Bf16>(A, st);
}

hipError_t launch_route_backward(const RouteGradArgs& A, bool f32, hipStream_t st) {
  return f32 ? route::backward<elem::F32>(A, st) : route::backward<elem::Bf16>(A, st);
}

}  // namespace tmk
