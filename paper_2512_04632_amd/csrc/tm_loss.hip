// Clipped policy loss with a KL term, from the logits, for gfx950.
//
// Row t has logits l of a vocabulary of V, a target y, a weight m (0: the row
// takes no part), an advantage A and log probabilities of the sampling and of a
// reference policy.  With the temperature tau
//
//   logp  = l_y / tau - lse,  lse = log sum_v exp(l_v / tau)
//   r     = exp(logp - old),  q = exp(ref - logp)
//   loss += m (-min(r A, clip(r, 1 - low, 1 + high) A) + kl (q - log q - 1))
//   slope = d loss / d logp = m (-[r within the bound on A's side] r A + kl (1 - q))
//   dlogits_v = slope ([v = y] - exp(l_v / tau - lse)) / tau
//
// The passes are bound by HBM: the logits are read once for the value, and once
// more where they are not still in a cache for the gradient, which is as large.
// The running maximum and sum of exponentials of each thread are joined at the
// end of a row.  Sums and statistics are fp32, exponentials are taken of the
// distance from the maximum; only dlogits is rounded to the logits' type.
// Rows of weight 0 or with a negative target are not read: their gradient is
// written as zeros whatever their logits hold.
#include <algorithm>

#include "tm_elem.h"
#include "tm_ops.h"

namespace tmk {
namespace loss {

using namespace elem;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// v_exp_f32: 1 ulp, results below the smallest normal number are zero
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Running maximum m and sum s of exp2((l - m) c).
struct Soft {
  float m, s;
};
__device__ inline Soft nothing() { return Soft{-INFINITY, 0.f}; }

// exp2((l - m) c) of a part's terms when its maximum moves from `from` to
// `to`; nothing was summed while the maximum was -inf.
__device__ inline float rescale(float from, float to, float c) {
  return from == -INFINITY ? 0.f : exp2_fast((from - to) * c);
}

__device__ inline Soft join(Soft a, Soft b, float c) {
  Soft o;
  o.m = fmaxf(a.m, b.m);
  o.s = a.s * rescale(a.m, o.m, c) + b.s * rescale(b.m, o.m, c);
  // a NaN in either maximum must not vanish in fmaxf
  if (a.s != a.s || b.s != b.s) o.s = NAN;
  return o;
}

template <int N>
__device__ inline void add_terms(Soft& a, const float* v, float c) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
  if (m > a.m) {
    a.s *= rescale(a.m, m, c);
    a.m = m;
  }
  // while every value is -inf the terms are taken as exp(-inf - 0) = 0
  const float at = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
  for (int i = 0; i < N; ++i) a.s += exp2_fast((v[i] - at) * c);
}

__device__ inline Soft wave_join(Soft a, float c) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    Soft b;
    b.m = __shfl_xor(a.m, o);
    b.s = __shfl_xor(a.s, o);
    a = join(a, b, c);
  }
  return a;
}

template <int NT>
__device__ inline Soft block_join(Soft a, float c, Soft* slots) {
  a = wave_join(a, c);
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = a;
  __syncthreads();
  a = slots[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) a = join(a, slots[w], c);
  return a;
}

__device__ inline bool active(const LossArgs& A, int64_t r) {
  return A.weights[r] != 0.f && A.targets[r] >= 0;
}

struct Row {
  float logp, lse, slope, loss;
};

// em = e^gap - 1 and d = e^gap - 1 - gap of the KL term.  Policies that are close to
// each other have gaps of 10^-2 and less, where differences from 1 keep few of d's digits or
// none: below 1 d is its power series, gap^2 (1 / 2! + gap / 3! + ..), off by 6e-9 of itself
// where it ends.
struct Gap {
  float em, d;
};
__device__ inline Gap gap_terms(float gap) {
  if (!(fabsf(gap) < 1.f)) {
    const float em = expf(gap) - 1.f;
    return Gap{em, em - gap};
  }
  float p = 1.f / 39916800.f;   // 1 / 11!
  p = fmaf(p, gap, 1.f / 3628800.f);
  p = fmaf(p, gap, 1.f / 362880.f);
  p = fmaf(p, gap, 1.f / 40320.f);
  p = fmaf(p, gap, 1.f / 5040.f);
  p = fmaf(p, gap, 1.f / 720.f);
  p = fmaf(p, gap, 1.f / 120.f);
  p = fmaf(p, gap, 1.f / 24.f);
  p = fmaf(p, gap, 1.f / 6.f);
  p = fmaf(p, gap, 0.5f);
  const float d = gap * gap * p;
  return Gap{gap + d, d};
}

// What a row gives once its maximum and sum are known.
template <class T>
__device__ inline Row finish(const LossArgs& A, int64_t r, Soft s) {
  const int64_t y = A.targets[r];
  const float log_sum = logf(s.s);
  const float ly = y < A.vocab ? T::load1(A.logits + (r * A.ld + y) * T::kBytes) : NAN;
  Row o;
  o.lse = s.m * A.inv_temp + log_sum;
  o.logp = (ly - s.m) * A.inv_temp - log_sum;
  const float m = A.weights[r], adv = A.advantages[r];
  const float ratio = expf(o.logp - A.old_logp[r]);
  const float lo = 1.f - A.clip_low, hi = 1.f + A.clip_high;
  const bool clipped = adv >= 0.f ? ratio > hi : ratio < lo;
  const float at = clipped ? (adv >= 0.f ? hi : lo) : ratio;
  float value = -at * adv, grad = clipped ? 0.f : -ratio * adv;
  if (A.ref_logp != nullptr) {
    const Gap g = gap_terms(A.ref_logp[r] - o.logp);
    value += A.kl * g.d;
    grad -= A.kl * g.em;
  }
  o.loss = m * value;
  o.slope = m * grad;
  return o;
}

__device__ inline void write_row(const LossArgs& A, int64_t r, const Row& o) {
  A.logp[r] = o.logp;
  A.lse[r] = o.lse;
  A.slope[r] = o.slope;
  A.row_loss[r] = o.loss;
}

// Gradient of a vector of logits, the target `target` entries on from its first:
// p = exp2((l - m) c) inv, out = f ([v = y] - p).
template <class T>
__device__ inline void gradient_vec(float* v, int target, float m, float c, float inv, float f) {
#pragma unroll
  for (int i = 0; i < T::W; ++i) {
    const float p = exp2_fast((v[i] - m) * c) * inv;
    v[i] = f * ((i == target ? 1.f : 0.f) - p);
  }
}

// The row's target, or a place that no entry has: a vocabulary ends before 2^30.
__device__ inline int target_of(const LossArgs& A, int64_t r) {
  const int64_t y = A.targets[r];
  return y < A.vocab ? int(y) : INT32_MAX;
}

template <class T, int NT>
__device__ inline void zero_row(char* row, int n, int t) {
  float z[T::W];
#pragma unroll
  for (int i = 0; i < T::W; ++i) z[i] = 0.f;
  for (int c = t * T::W; c < n; c += NT * T::W) store_vec<T>(row, c, n, z);
}

// -inf in the elements of a vector that lie past the row's end.
template <class T>
__device__ inline u32x4_t fill_past(u32x4_t q, int first, int n) {
#pragma unroll
  for (int i = 0; i < T::W; ++i) {
    if (first + i < n) continue;
    if constexpr (T::kBytes == 2) q[i / 2] = i % 2 ? (q[i / 2] & 0xffffu) | 0xff800000u : (q[i / 2] & 0xffff0000u) | 0xff80u;
    else q[i] = 0xff800000u;
  }
  return q;
}

// The vector as it is, behind a fence: without it the compiler unpacks a held
// row of bf16 once and keeps the fp32 values, twice the registers.
__device__ inline u32x4_t afresh(u32x4_t q) {
  asm volatile("" : "+v"(q));
  return q;
}

// Between the vectors of a long held row: unpacked values of several at once
// have no registers.
template <int K>
__device__ inline void keep_order() {
  if constexpr (K >= 8) __builtin_amdgcn_sched_barrier(0);
}

// NT threads per row (64: four rows a workgroup), which hold the whole row in
// registers, K vectors each: it is read once, its maximum is known before the
// first exponential is taken, and the gradient is formed from the registers.
// Bound by the exponentials and the unpacking for short rows (10140 x 1731 bf16 with
// gradient: 25 us), by HBM for long ones (4096 x 32001 fp32 with gradient: 196 us).
template <class T, int NT, int K, bool GRAD>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void k_loss_held(const LossArgs A) {
  constexpr int RB = NT < 256 ? 256 / NT : 1, W = T::W, NW = NT / 64;
  __shared__ Soft slots[NT > 64 ? NW : 1];
  const int t = threadIdx.x % NT, n = A.vocab;
  const int64_t r = int64_t(blockIdx.x) * RB + threadIdx.x / NT;
  if (r >= A.rows) return;
  char* d = GRAD ? A.dlogits + r * A.ldd * T::kBytes : nullptr;
  if (!active(A, r)) {
    if (t == 0) write_row(A, r, Row{0.f, 0.f, 0.f, 0.f});
    if constexpr (GRAD) zero_row<T, NT>(d, n, t);
    return;
  }
  const char* l = A.logits + r * A.ld * T::kBytes;
  const float c = A.inv_temp * kLog2e;
  u32x4_t q[K];
#pragma unroll
  for (int j = 0; j < K; ++j) q[j] = load_ahead<T, true>(l, (j * NT + t) * W, n);
#pragma unroll
  for (int j = 0; j < K; ++j) {
    const int first = (j * NT + t) * W;
    if (first + W > n) q[j] = fill_past<T>(settle<T, true>(q[j], first, n), first, n);
  }
  Soft s = nothing();
  bool nan = false;
#pragma unroll
  for (int j = 0; j < K; ++j) {
    float v[W];
    T::unpack(afresh(q[j]), v);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      s.m = fmaxf(s.m, v[i]);
      nan |= v[i] != v[i];
    }
    keep_order<K>();
  }
  // while every value is -inf the terms are taken as exp(-inf - 0) = 0
  const float at = s.m == -INFINITY ? 0.f : s.m;
#pragma unroll
  for (int j = 0; j < K; ++j) {
    float v[W];
    T::unpack(afresh(q[j]), v);
#pragma unroll
    for (int i = 0; i < W; ++i) s.s += exp2_fast((v[i] - at) * c);
    keep_order<K>();
  }
  if (nan) s.s = NAN;
  s = wave_join(s, c);
  Row row;
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = s;
    __syncthreads();
    s = slots[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) s = join(s, slots[w], c);
  }
  row = finish<T>(A, r, s);   // every thread: what it reads is in a cache, and nothing waits for another
  if constexpr (NT > 64) {
    // the target's logit has been read by everyone before any of the row is overwritten
    if constexpr (GRAD) __syncthreads();
  }
  if (t == 0) write_row(A, r, row);
  if constexpr (GRAD) {
    const float f = row.slope * A.inv_temp, inv = 1.f / s.s;
    const int y = target_of(A, r);
    if (f == 0.f) {
      zero_row<T, NT>(d, n, t);
      return;
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
      const int first = (j * NT + t) * W;
      if (first >= n) continue;
      float v[W];
      T::unpack(afresh(q[j]), v);
      gradient_vec<T>(v, y - first, s.m, c, inv, f);
      store_vec<T>(d, first, n, v);
      keep_order<K>();
    }
  }
}

// f(values, first entry) for each vector of entries first .. last - 1 of a row
// that falls to this thread of NT, -inf past the end; four loads at a time.
template <class T, int NT, class F>
__device__ inline void each_group(const char* l, int first, int last, F f) {
  constexpr int G = 4, STEP = NT * T::W;
  int at = first + int(threadIdx.x) * T::W;
  for (; at + (G - 1) * STEP + T::W <= last; at += G * STEP) {
    u32x4_t q[G];
#pragma unroll
    for (int g = 0; g < G; ++g) q[g] = T::load(l + int64_t(at + g * STEP) * T::kBytes);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float v[T::W];
      T::unpack(q[g], v);
      f(v, at + g * STEP);
    }
  }
  for (; at < last; at += STEP) {
    float v[T::W];
    load_vec<T>(l, at, last, -INFINITY, v);
    f(v, at);
  }
}

// Longer rows: one workgroup per row, which reads it twice (the second time
// mostly from the memory-side cache).  Bound by HBM: 8192 x 131072 bf16 with gradient,
// a quarter of the rows without part, 783 us, 4.8 TB/s of what has to move (a large copy
// reaches 5.0); 4096 x 50257 bf16 with gradient 223 us.
template <class T, int NT, bool GRAD>
__global__ __launch_bounds__(NT) void k_loss_rows(const LossArgs A) {
  __shared__ Soft slots[NT / 64];
  __shared__ Row row;
  const int64_t r = blockIdx.x;
  const int n = A.vocab;
  if (!active(A, r)) {
    if (threadIdx.x == 0) write_row(A, r, Row{0.f, 0.f, 0.f, 0.f});
    if constexpr (GRAD) zero_row<T, NT>(A.dlogits + r * A.ldd * T::kBytes, n, threadIdx.x);
    return;
  }
  const char* l = A.logits + r * A.ld * T::kBytes;
  const float c = A.inv_temp * kLog2e;
  Soft s = nothing();
  each_group<T, NT>(l, 0, n, [&](float* v, int) { add_terms<T::W>(s, v, c); });
  s = block_join<NT>(s, c, slots);
  if (threadIdx.x == 0) {
    row = finish<T>(A, r, s);
    write_row(A, r, row);
  }
  if constexpr (GRAD) {
    __syncthreads();
    char* d = A.dlogits + r * A.ldd * T::kBytes;
    const float f = row.slope * A.inv_temp, inv = 1.f / s.s;
    const int y = target_of(A, r);
    if (f == 0.f) {
      zero_row<T, NT>(d, n, threadIdx.x);
      return;
    }
    each_group<T, NT>(l, 0, n, [&](float* v, int at) {
      gradient_vec<T>(v, y - at, s.m, c, inv, f);
      store_vec<T>(d, at, n, v);
    });
  }
}

// Few rows (loss_chunks): a workgroup per chunk of a row.  Bound by latency: 16 x
// 50257 bf16 4.9 us, and 3.6 us for the join, of the call's 14 us on the host.
template <class T>
__global__ __launch_bounds__(256) void k_loss_part(const LossArgs A) {
  __shared__ Soft slots[4];
  const int64_t r = blockIdx.x / A.chunks;
  if (!active(A, r)) return;
  const int q = blockIdx.x - int(r) * A.chunks;
  const int first = q * A.chunk, last = min(A.vocab, first + A.chunk);
  const char* l = A.logits + r * A.ld * T::kBytes;
  const float c = A.inv_temp * kLog2e;
  Soft s = nothing();
  each_group<T, 256>(l, first, last, [&](float* v, int) { add_terms<T::W>(s, v, c); });
  s = block_join<256>(s, c, slots);
  if (threadIdx.x == 0) A.part[blockIdx.x] = make_float2(s.m, s.s);
}

// One wave per row joins its chunks, and the one workgroup adds the loss up as well.
template <class T>
__global__ __launch_bounds__(1024) void k_loss_join(const LossArgs A) {
  __shared__ double sums[16];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const float c = A.inv_temp * kLog2e;
  double total = 0.0;
  for (int64_t r = wave; r < A.rows; r += 16) {
    Row o{0.f, 0.f, 0.f, 0.f};
    if (active(A, r)) {
      Soft s = nothing();
      for (int q = lane; q < A.chunks; q += 64) {
        const float2 p = A.part[r * A.chunks + q];
        s = join(s, Soft{p.x, p.y}, c);
      }
      s = wave_join(s, c);
      o = finish<T>(A, r, s);
      if (lane == 0) A.stats[r] = make_float2(s.m, 1.f / s.s);
    }
    if (lane == 0) write_row(A, r, o);
    total += double(o.loss);
  }
  if (lane == 0) sums[wave] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) total += sums[w];
    *A.loss = float(total);
  }
}

// The rows' shares added up in a fixed order, in 64 bits (8192 rows: 5.6 us, bound by
// latency; a loss of parts per workgroup added by the last one would need a counter
// that is cleared for every call).
__global__ __launch_bounds__(1024) void k_loss_sum(const float* row_loss, int rows, float* out) {
  __shared__ double sums[1024];
  double s = 0.0;
  for (int r = threadIdx.x; r < rows; r += 1024) s += double(row_loss[r]);
  sums[threadIdx.x] = s;
  __syncthreads();
  for (int o = 512; o > 0; o >>= 1) {
    if (int(threadIdx.x) < o) sums[threadIdx.x] += sums[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) *out = float(sums[0]);
}

// dlogits of the rows' slopes, a workgroup per chunk of a row.  Rows without a
// slope are not read.
//   STATS = true   of rows that k_loss_join has just joined: from their maximum
//                  and sum, as where one workgroup has the whole row.
//   STATS = false  from lse, which is all that is left of an earlier call: l / tau -
//                  lse is rounded once (fma), but carries the rounding of lse.
//                  Bound by HBM: 3000 x 32001 fp32, a tenth of the rows without
//                  part, 125 us, 5.8 TB/s.
template <class T, bool STATS>
__global__ __launch_bounds__(256) void k_loss_gradient(const LossArgs A) {
  const int64_t r = blockIdx.x / A.chunks;
  const int q = blockIdx.x - int(r) * A.chunks;
  const int first = q * A.chunk, last = min(A.vocab, first + A.chunk);
  const float slope = A.slope[r];
  const char* l = A.logits + r * A.ld * T::kBytes;
  char* d = A.dlogits + r * A.ldd * T::kBytes;
  const float f = slope * A.inv_temp * (!STATS && A.grad != nullptr ? *A.grad : 1.f);
  const bool none = STATS ? f == 0.f : slope == 0.f;
  const float c = A.inv_temp * kLog2e;
  float2 stats = make_float2(0.f, 0.f);
  float lse = 0.f;
  if constexpr (STATS) {
    if (!none) stats = A.stats[r];
  } else {
    lse = A.lse[r];
  }
  const int y = target_of(A, r);
  for (int at = first + threadIdx.x * T::W; at < last; at += 256 * T::W) {
    float v[T::W];
    if (none) {
#pragma unroll
      for (int i = 0; i < T::W; ++i) v[i] = 0.f;
    } else {
      load_vec<T>(l, at, last, 0.f, v);
      if constexpr (STATS) {
        gradient_vec<T>(v, y - at, stats.x, c, stats.y, f);
      } else {
#pragma unroll
        for (int i = 0; i < T::W; ++i) {
          const float p = exp2_fast(fmaf(v[i], A.inv_temp, -lse) * kLog2e);
          v[i] = f * ((i == y - at ? 1.f : 0.f) - p);
        }
      }
    }
    store_vec<T>(d, at, last, v);
  }
}

template <class T, int NT, int K>
void launch_held(const LossArgs& A, hipStream_t st) {
  constexpr int RB = NT < 256 ? 256 / NT : 1;
  const dim3 grid(uint32_t((A.rows + RB - 1) / RB)), block(NT < 256 ? 256 : NT);
  if (A.dlogits != nullptr) hipLaunchKernelGGL((k_loss_held<T, NT, K, true>), grid, block, 0, st, A);
  else hipLaunchKernelGGL((k_loss_held<T, NT, K, false>), grid, block, 0, st, A);
}

template <class T, int NT>
void launch_twice(const LossArgs& A, hipStream_t st) {
  const dim3 grid(uint32_t(A.rows));
  if (A.dlogits != nullptr) hipLaunchKernelGGL((k_loss_rows<T, NT, true>), grid, dim3(NT), 0, st, A);
  else hipLaunchKernelGGL((k_loss_rows<T, NT, false>), grid, dim3(NT), 0, st, A);
}

// Rows held in registers or read twice, and by how many threads; the same with
// and without the gradient, so that the value has the same bits (4096 rows unless
// said otherwise).
//   Held by a wave: up to 256 vectors (10140 x 1731 bf16 with gradient: 25 us, 36
//   when read twice).
//   Held by a workgroup: fp32 from 16384 to 32768 entries (32001: 196 us with
//   gradient, 230 when read twice).  Below, what the gradient gains the value alone
//   loses (15000: 100 against 118 us, 67 against 41), and bf16 rows, which are
//   unpacked anew in every pass, are better read twice (20000: 160 against 75).
//   Read twice: 256 threads, so that many rows overlap, as long as the rows under
//   way stay in the memory-side cache until their second reading: 512 threads from
//   48 KB a row and 1024 from 160 KB (with gradient, 50257 bf16: 251, 223 and 276 us
//   with 256, 512 and 1024 threads; 8192 x 131072: 1185, 1047, 881).
template <class T>
void launch_rows(const LossArgs& A, hipStream_t st) {
  const int vecs = (A.vocab + T::W - 1) / T::W;
  if (vecs <= 64 * 2) return launch_held<T, 64, 2>(A, st);
  if (vecs <= 64 * 4) return launch_held<T, 64, 4>(A, st);
  if constexpr (T::kBytes == 4) {
    if (vecs > 1024 * 4 && vecs <= 1024 * 8) return launch_held<T, 1024, 8>(A, st);
  }
  const int64_t bytes = int64_t(A.vocab) * T::kBytes;
  if (bytes <= 48 * 1024) return launch_twice<T, 256>(A, st);
  if (bytes <= 160 * 1024) return launch_twice<T, 512>(A, st);
  launch_twice<T, 1024>(A, st);
}

template <class T>
hipError_t forward_t(const LossArgs& A, hipStream_t st) {
  if (A.chunks > 1) {
    const dim3 grid(uint32_t(A.rows) * A.chunks);
    hipLaunchKernelGGL((k_loss_part<T>), grid, dim3(256), 0, st, A);
    hipLaunchKernelGGL((k_loss_join<T>), dim3(1), dim3(1024), 0, st, A);
    if (A.dlogits != nullptr) hipLaunchKernelGGL((k_loss_gradient<T, true>), grid, dim3(256), 0, st, A);
    return hipGetLastError();
  }
  if (A.rows > 0) launch_rows<T>(A, st);
  hipLaunchKernelGGL(k_loss_sum, dim3(1), dim3(1024), 0, st, A.row_loss, A.rows, A.loss);
  return hipGetLastError();
}

}  // namespace loss

// Parts that each row is cut into where there are fewer rows than the card needs
// workgroups (us of the value and with gradient, bf16, whole against cut: 16 x
// 50257 9.6, 15.4 and 7.7, 10.6; 16 x 32768 7.9, 11.3 and 7.5, 9.7; 16 x 16384 6.8, 8.9 and 7.4, 9.9;
// 32 x 131072 14.9, 26.5 and 10.4, 15.5; 32 x 50257 9.5, 15.8 and 9.9, 13.2; 48 x 131072 15.6, 27.4
// and 15.4, 20.2: the one workgroup that joins the parts then has three rows a wave;
// 1 x 131072 14.1, 16.8 and 6.7, 8.8 in 64 parts).
int loss_chunks(int64_t rows, int64_t vocab) {
  if (rows > 32 || vocab < (rows > 16 ? 65536 : 32768)) return 1;
  return int(std::min<int64_t>({512 / rows, vocab / 2048, 64}));
}

hipError_t launch_loss(const LossArgs& A, bool f32, hipStream_t st) {
  return f32 ? loss::forward_t<elem::F32>(A, st) : loss::forward_t<elem::Bf16>(A, st);
}

hipError_t launch_loss_backward(const LossArgs& A, bool f32, hipStream_t st) {
  const dim3 grid(uint32_t(A.rows) * uint32_t(A.chunks));
  if (f32) hipLaunchKernelGGL((loss::k_loss_gradient<elem::F32, false>), grid, dim3(256), 0, st, A);
  else hipLaunchKernelGGL((loss::k_loss_gradient<elem::Bf16, false>), grid, dim3(256), 0, st, A);
  return hipGetLastError();
}

}  // namespace tmk
