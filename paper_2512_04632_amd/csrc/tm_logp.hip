// Log probabilities of given tokens, entropies and the most likely alternatives of
// rows of logits, forward and backward, for gfx950.
//
// A row has logits l over a vocabulary of V and a target y (negative: the row takes no
// part).  With the temperature tau, u_v = (l_v - m) / tau and m the largest logit:
//
//   s = sum exp u_v,  logp = u_y - log s,  H = log s - sum u_v exp u_v / s
//   alternatives: the `top` largest l_v, of equal ones the lowest v, with u_v - log s
//   dl_v = (g ([v = y] - p_v) - h p_v (log p_v + H)) / tau,  p_v = exp(u_v) / s,
//          g and h the gradients by logp and H
//
// The logits are read once.  Each thread keeps a running maximum and, in powers of 2,
// the sums of e and of e u of what it has seen; they are joined at the end of a row.
// p log p of an entry without probability is zero: u is held at -200 there, where e
// is zero.  Sums are fp32; backwards p comes from m and s themselves, not from a rounded
// logarithm.
//
// Alternatives: an entry is a 64-bit key, its value's bits in an order of whole numbers above
// the complement of its place, so that keys are unique and the order is the wanted one.
// While the row goes by, the maximum of every 16 vectors (one of 16 neighbouring lanes each) is
// put down in LDS.  The `top` best entries lie in the `top` groups with the best maxima: if
// one lay outside, `top` groups would hold better ones.  One wave picks these groups, reads
// them again and picks the entries, both times from those that reach a bound that `top` of
// them are known to reach.  -inf and NaN are no alternatives.
#include <algorithm>

#include "tm_elem.h"
#include "tm_ops.h"

namespace tmk {
namespace logp {

using namespace elem;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFar = -200.f;   // a power of 2 that is zero in fp32

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// ---------------------------------------------------------------- sums
// m the maximum, s the sum of e = exp2((l - m) c), t the sum of e (l - m) c.
struct Sums {
  float m, s, t;
};
__device__ inline Sums nothing() { return Sums{-INFINITY, 0.f, 0.f}; }

// The sums of `a` about the maximum m.
__device__ inline void move_to(Sums& a, float m, float c) {
  const float by = (a.m - m) * c;
  const float f = a.m == -INFINITY ? 0.f : exp2_fast(by);   // nothing was summed about -inf
  a.t = (a.t + a.s * fmaxf(by, kFar)) * f;
  a.s *= f;
  a.m = m;
}

__device__ inline Sums join(Sums a, Sums b, float c) {
  const float m = fmaxf(a.m, b.m);
  const bool nan = a.s != a.s || b.s != b.s;   // one about -inf would vanish
  move_to(a, m, c);
  move_to(b, m, c);
  return Sums{m, nan ? NAN : a.s + b.s, a.t + b.t};
}

template <int N>
__device__ inline float largest(const float* v) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
  return m;
}

// Adds N logits whose maximum is m.
template <int N>
__device__ inline void add_terms(Sums& a, const float* v, float m, float c) {
  if (m > a.m) move_to(a, m, c);
  const float at = a.m == -INFINITY ? 0.f : a.m;   // terms of -inf are exp(-inf - 0) = 0
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float u = (v[i] - at) * c, e = exp2_fast(u);
    a.s += e;
    a.t += e * fmaxf(u, kFar);
  }
}

__device__ inline Sums wave_join(Sums a, float c) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    Sums b;
    b.m = __shfl_xor(a.m, o);
    b.s = __shfl_xor(a.s, o);
    b.t = __shfl_xor(a.t, o);
    a = join(a, b, c);
  }
  return a;
}

template <class T>
__device__ inline void write_row(const LogpArgs& A, int64_t r, int64_t y, Sums a) {
  const float log_sum = logf(a.s);
  const float ly = y < A.vocab ? T::load1(A.logits + (r * A.ld + y) * T::kBytes) : NAN;
  A.logp[r] = (ly - a.m) * A.inv_temp - log_sum;
  A.entropy[r] = log_sum - a.t * kLn2 / a.s;
  A.stats[r] = make_float2(a.m, a.s);
}

// ---------------------------------------------------------------- alternatives
typedef uint64_t Key;

__device__ inline uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);   // -0 and 0 are equal
  return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ inline float value_of(Key k) {
  const uint32_t b = uint32_t(k >> 32);
  return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ inline int place_of(Key k) { return int(~uint32_t(k)); }
// 0, less than every entry's, for what is no alternative.
__device__ inline Key key_of(float v, int place) {
  return v > -INFINITY ? Key(ordered(v)) << 32 | uint32_t(~place) : Key(0);
}

// LDS of one wave: what one lane has written the others read.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int kListed = 320;
struct List {
  Key keys[kListed], best[64];
};

// A wave's picking of the `top` best of the keys that it is given.
struct Picker {
  List& list;
  int top, n = 0;
  Key floor = 1;   // keys below it are out

  __device__ Picker(List& l, int k) : list(l), top(k) {}

  // The best `top` of the listed keys, in order.
  __device__ void settle() {
    const int lane = threadIdx.x & 63;
    wave_sync();
    for (int i = lane; i < n; i += 64) {
      const Key mine = list.keys[i];
      int better = 0;
      for (int j = 0; j < n; ++j) better += list.keys[j] > mine ? 1 : 0;
      if (better < top) list.best[better] = mine;
    }
    wave_sync();
    n = min(n, top);
    if (lane < n) list.keys[lane] = list.best[lane];
    wave_sync();
    if (n == top) floor = list.keys[top - 1];
  }
  // One key of each lane (0: none).
  __device__ void push(Key key) {
    const bool in = key >= floor;
    const uint64_t who = __ballot(in);
    if (who == 0) return;
    const int lane = threadIdx.x & 63;
    if (in) list.keys[n + __popcll(who & ((uint64_t(1) << lane) - 1))] = key;
    n += __popcll(who);
    if (n > kListed - 64) settle();
  }
  // Raises the floor to the `top`-th best of the lanes' own best keys: of each lane one
  // entry, and `top` of them reach it.
  __device__ void start(Key lanes_best) {
    push(lanes_best);
    settle();
    n = 0;
    wave_sync();
  }
};

template <class T>
__device__ inline void write_top(const LogpArgs& A, int64_t r, const Key* keys, int n, float m, float s) {
  const int lane = threadIdx.x & 63;
  if (lane < A.top) {
    const bool there = lane < n;
    const float v = there ? value_of(keys[lane]) : -INFINITY;
    A.top_logp[r * A.top + lane] = (v - m) * A.inv_temp - logf(s);
    A.top_ids[r * A.top + lane] = there ? place_of(keys[lane]) : -1;
  }
}

// A row that takes no part; `lanes` threads of it.
__device__ inline void write_none(const LogpArgs& A, int64_t r, int t) {
  if (t == 0) {
    A.logp[r] = 0.f;
    A.entropy[r] = 0.f;
    A.stats[r] = make_float2(0.f, 0.f);
  }
  if (t < A.top) {
    A.top_logp[r * A.top + t] = 0.f;
    A.top_ids[r * A.top + t] = -1;
  }
}

// ---------------------------------------------------------------- forward
// A wave per row, which holds it in registers, K vectors a lane.
template <class T, int K, bool TOP>
__global__ __launch_bounds__(256) void k_logp_held(const LogpArgs A) {
  constexpr int W = T::W;
  __shared__ List lists[TOP ? 4 : 1];
  const int lane = threadIdx.x & 63, n = A.vocab;
  const int64_t r = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (r >= A.rows) return;
  const int64_t y = A.targets[r];
  if (y < 0) return write_none(A, r, lane);
  const char* l = A.logits + r * A.ld * T::kBytes;
  const float c = A.inv_temp * kLog2e;
  float v[K * W];
#pragma unroll
  for (int j = 0; j < K; ++j) load_vec<T>(l, (j * 64 + lane) * W, n, -INFINITY, v + j * W);
  Sums a = nothing();
  add_terms<K * W>(a, v, largest<K * W>(v), c);
  a = wave_join(a, c);
  if (lane == 0) write_row<T>(A, r, y, a);
  if constexpr (TOP) {
    Picker pick(lists[threadIdx.x >> 6], A.top);
    Key best = 0;
#pragma unroll
    for (int e = 0; e < K * W; ++e) best = max(best, key_of(v[e], ((e / W) * 64 + lane) * W + e % W));
    pick.start(best);
#pragma unroll
    for (int e = 0; e < K * W; ++e) pick.push(key_of(v[e], ((e / W) * 64 + lane) * W + e % W));
    pick.settle();
    write_top<T>(A, r, pick.list.keys, pick.n, a.m, a.s);
  }
}

// Most groups of a chunk.
constexpr int kGroups = 2048;
template <class T>
constexpr int group_size() { return 16 * T::W; }

// The maximum over 16 neighbouring lanes, in each of them.
__device__ inline float max16(float v) {
  auto step = [&](auto ctrl) {
    v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, false)));
  };
  step(std::integral_constant<int, 0x128>{});   // row_ror:8, :4, :2, :1
  step(std::integral_constant<int, 0x124>{});
  step(std::integral_constant<int, 0x122>{});
  step(std::integral_constant<int, 0x121>{});
  return v;
}

// The best entries of l[first .. last) from its groups' maxima, by one wave.
template <class T>
__device__ inline void pick_entries(Picker& pick, const float* maxima, const char* l, int first, int last) {
  constexpr int W = T::W, GROUP = group_size<T>();
  const int lane = threadIdx.x & 63, groups = (last - first + GROUP - 1) / GROUP;
  Key best = 0;
  for (int g = lane; g < groups; g += 64) best = max(best, key_of(maxima[g], g));
  pick.start(best);
  for (int base = 0; base < groups; base += 64) {
    const int g = base + lane;
    pick.push(g < groups ? key_of(maxima[g], g) : Key(0));
  }
  pick.settle();
  // the picked groups, a lane each; their best entries reach the last one's maximum
  const int found = pick.n;
  const Key mine = lane < found ? pick.list.keys[lane] : Key(0);
  wave_sync();
  pick.floor = found == pick.top ? pick.floor >> 32 << 32 : Key(1);
  pick.n = 0;
  for (int base = 0; base < found; base += 4) {
    const int from = base + (lane >> 4), g = place_of(__shfl((unsigned long long)mine, from & 63));
    const int at = from < found ? first + g * GROUP + (lane & 15) * W : last;
    float v[W];
    load_vec<T>(l, at, last, -INFINITY, v);
#pragma unroll
    for (int i = 0; i < W; ++i) pick.push(key_of(v[i], at + i));
  }
  pick.settle();
}

// NT threads for a row, or a chunk of one.
template <class T, int NT, bool TOP>
__global__ __launch_bounds__(NT) void k_logp_rows(const LogpArgs A) {
  constexpr int W = T::W, STEP = NT * W, G = 4;
  __shared__ Sums slots[NT / 64];
  __shared__ float maxima[TOP ? kGroups : 1];
  __shared__ List list[1];
  const int64_t r = blockIdx.x / A.chunks;
  const int64_t y = A.targets[r];
  if (y < 0) {
    if (A.chunks == 1) write_none(A, r, threadIdx.x);
    return;
  }
  const int first = int(blockIdx.x - r * A.chunks) * A.chunk, last = min(A.vocab, first + A.chunk);
  const char* l = A.logits + r * A.ld * T::kBytes;
  const float c = A.inv_temp * kLog2e;
  Sums a = nothing();
  auto take = [&](const float* v, int at) __attribute__((always_inline)) {
    const float m = largest<W>(v);
    add_terms<W>(a, v, m, c);
    if constexpr (TOP) {
      const float g = max16(m);
      if ((threadIdx.x & 15) == 0 && at < last) maxima[(at - first) / group_size<T>()] = g;
    }
  };
  int base = first;
  for (; base + G * STEP <= last; base += G * STEP) {
    u32x4_t q[G];
#pragma unroll
    for (int g = 0; g < G; ++g) q[g] = T::load(l + int64_t(base + g * STEP + int(threadIdx.x) * W) * T::kBytes);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float v[W];
      T::unpack(q[g], v);
      take(v, base + g * STEP + int(threadIdx.x) * W);
    }
  }
  for (; base < last; base += STEP) {   // every lane, those past the end with -inf
    const int at = base + int(threadIdx.x) * W;
    float v[W];
    load_vec<T>(l, at, last, -INFINITY, v);
    take(v, at);
  }
  a = wave_join(a, c);
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = a;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  a = slots[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) a = join(a, slots[w], c);
  if (threadIdx.x == 0) {
    if (A.chunks == 1) write_row<T>(A, r, y, a);
    else A.part[blockIdx.x] = make_float4(a.m, a.s, a.t, 0.f);
  }
  if constexpr (TOP) {
    Picker pick(list[0], A.top);
    pick_entries<T>(pick, maxima, l, first, last);
    if (A.chunks == 1) {
      write_top<T>(A, r, pick.list.keys, pick.n, a.m, a.s);
    } else if (int(threadIdx.x) < A.top) {
      A.keys[int64_t(blockIdx.x) * A.top + threadIdx.x] = int(threadIdx.x) < pick.n ? pick.list.keys[threadIdx.x] : Key(0);
    }
  }
}

// A wave joins the chunks of a row.
template <class T, bool TOP>
__global__ __launch_bounds__(256) void k_logp_join(const LogpArgs A) {
  __shared__ List lists[TOP ? 4 : 1];
  const int lane = threadIdx.x & 63;
  const int64_t r = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (r >= A.rows) return;
  const int64_t y = A.targets[r];
  if (y < 0) return write_none(A, r, lane);
  const float c = A.inv_temp * kLog2e;
  Sums a = nothing();
  for (int q = lane; q < A.chunks; q += 64) {
    const float4 p = A.part[r * A.chunks + q];
    a = join(a, Sums{p.x, p.y, p.z}, c);
  }
  a = wave_join(a, c);
  if (lane == 0) write_row<T>(A, r, y, a);
  if constexpr (TOP) {
    const Key* keys = A.keys + r * A.chunks * A.top;
    const int n = A.chunks * A.top;
    Picker pick(lists[threadIdx.x >> 6], A.top);
    Key best = 0;
    for (int i = lane; i < n; i += 64) best = max(best, keys[i]);
    pick.start(best);
    for (int base = 0; base < n; base += 64) pick.push(base + lane < n ? keys[base + lane] : Key(0));
    pick.settle();
    write_top<T>(A, r, pick.list.keys, pick.n, a.m, a.s);
  }
}

// ---------------------------------------------------------------- backward
// A workgroup per chunk of a row.  Rows without a gradient are not read.
template <class T>
__global__ __launch_bounds__(256) void k_logp_gradient(const LogpArgs A) {
  const int64_t r = blockIdx.x / A.chunks;
  const int first = int(blockIdx.x - r * A.chunks) * A.chunk, last = min(A.vocab, first + A.chunk);
  const int64_t y = A.targets[r];
  float g = A.dlogp != nullptr ? A.dlogp[r] : 0.f;
  const float h = A.dentropy != nullptr ? A.dentropy[r] : 0.f;
  const bool none = y < 0 || (g == 0.f && h == 0.f);
  if (y >= A.vocab) g = NAN;
  const char* l = A.logits + r * A.ld * T::kBytes;
  char* d = A.dlogits + r * A.ldd * T::kBytes;
  const float c = A.inv_temp * kLog2e;
  const float2 st = A.stats[r];
  const float inv = 1.f / st.y, shift = A.entropy[r] - logf(st.y);
  const int target = y < A.vocab ? int(y) : INT32_MAX;   // a vocabulary ends before 2^30
  for (int at = first + int(threadIdx.x) * T::W; at < last; at += 256 * T::W) {
    float v[T::W];
    if (none) {
#pragma unroll
      for (int i = 0; i < T::W; ++i) v[i] = 0.f;
    } else {
      load_vec<T>(l, at, last, 0.f, v);
#pragma unroll
      for (int i = 0; i < T::W; ++i) {
        const float u = (v[i] - st.x) * c, p = exp2_fast(u) * inv;
        const float to = g + h * (fmaxf(u, kFar) * kLn2 + shift);
        v[i] = ((i == target - at ? g : 0.f) - p * to) * A.inv_temp;
      }
    }
    store_vec<T>(d, at, last, v);
  }
}

template <class T, bool TOP>
hipError_t forward_t(const LogpArgs& A, hipStream_t st) {
  const dim3 quads(uint32_t((A.rows + 3) / 4)), each(uint32_t(A.rows) * uint32_t(A.chunks));
  switch (logp_threads(A, T::kBytes == 4)) {
    case 64:
      if (A.vocab <= 128 * T::W) hipLaunchKernelGGL((k_logp_held<T, 2, TOP>), quads, dim3(256), 0, st, A);
      else hipLaunchKernelGGL((k_logp_held<T, 4, TOP>), quads, dim3(256), 0, st, A);
      break;
    case 256: hipLaunchKernelGGL((k_logp_rows<T, 256, TOP>), each, dim3(256), 0, st, A); break;
    case 512: hipLaunchKernelGGL((k_logp_rows<T, 512, TOP>), each, dim3(512), 0, st, A); break;
    default: hipLaunchKernelGGL((k_logp_rows<T, 1024, TOP>), each, dim3(1024), 0, st, A);
  }
  if (A.chunks > 1) hipLaunchKernelGGL((k_logp_join<T, TOP>), quads, dim3(256), 0, st, A);
  return hipGetLastError();
}

}  // namespace logp

void plan_logp(LogpArgs& A, bool f32) {
  const int64_t rows = std::max(A.rows, 1), group = f32 ? 64 : 128, most = group * logp::kGroups;
  int64_t chunks = rows < 256 ? std::min<int64_t>(512 / rows, A.vocab / 4096) : 1;
  chunks = std::max<int64_t>({chunks, 1, (A.vocab + most - 1) / most});
  A.chunk = int32_t(((A.vocab + chunks - 1) / chunks + group - 1) / group * group);
  A.chunks = (A.vocab + A.chunk - 1) / A.chunk;
}

// 64: a wave holds the row, four rows a workgroup.
int logp_threads(const LogpArgs& A, bool f32) {
  const int64_t bytes = int64_t(A.chunk) * (f32 ? 4 : 2);
  if (A.chunks == 1 && int64_t(A.vocab) * (f32 ? 4 : 2) <= 4096) return 64;
  return bytes <= 48 * 1024 ? 256 : bytes <= 160 * 1024 ? 512 : 1024;
}

hipError_t launch_logp(const LogpArgs& A, bool f32, hipStream_t st) {
  if (A.top > 0) return f32 ? logp::forward_t<elem::F32, true>(A, st) : logp::forward_t<elem::Bf16, true>(A, st);
  return f32 ? logp::forward_t<elem::F32, false>(A, st) : logp::forward_t<elem::Bf16, false>(A, st);
}

hipError_t launch_logp_backward(const LogpArgs& A, bool f32, hipStream_t st) {
  const dim3 grid(uint32_t(A.rows) * uint32_t(A.chunks));
  if (f32) hipLaunchKernelGGL((logp::k_logp_gradient<elem::F32>), grid, dim3(256), 0, st, A);
  else hipLaunchKernelGGL((logp::k_logp_gradient<elem::Bf16>), grid, dim3(256), 0, st, A);
  return hipGetLastError();
}

}  // namespace tmk
