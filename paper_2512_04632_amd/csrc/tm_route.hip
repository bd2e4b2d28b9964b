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
// Forward: rows are held in the registers of 16, 32, 64 or 256 lanes, which take the maximum `top` times; a block of 64
// rows marks a choice with the row's bit in a word of 64 per expert, so that a choice's place among the block's is a
// count of the bits below it, and no order of atomics shows.  Up to 64 rows are one block, which knows all places, ends
// and the loss at once.  Else a second launch adds up the blocks' counts (16 bits each) and moves every choice by what lies
// before its block.  Sums of probabilities are fp32 over a block's rows, 64-bit over the blocks, in a fixed order.
//
// Bound by instructions and by latency, not by memory: 32768 x 256 fp32, 8 chosen, has 34 MB to read and 3 to write (7 us at
// the rate of a copy) and takes 27 us, 18 of it the choices and 10 the second launch, whose steps wait for one another.
// The choices take 53 vector instructions for each score of 256: 18 the nine rounds, 6 the keys, the others exponentials and
// sums, the end of each row (the chosen's shares, their marks) and of the block.  The rows of 129 to 1024 experts
// stand at the 128 registers of four waves a SIMD, 2 to 4 of them kept in memory (3 of the 7 MB that the choices write).
// 64 rows x 8 take 10 us of the host for 6 of the kernel.  65 to some 2000 rows are a few workgroups, each with four
// rows or more to a group one after the other, and the second launch: 100 x 384 22 us, 17 and 6 in the kernels; 1000 x 512
// 23, 17 and 7; 512 x 64 14, 7 and 7.
#include <algorithm>

#include "tm_elem.h"
#include "tm_ops.h"

namespace tmk {
namespace route {

using namespace elem;

constexpr int kRows = kRouteRows;
constexpr float kLog2e = 1.4426950408889634f;

// A reduction over the 16 lanes of a data-parallel row, the same in each of them.
template <class V, class F>
__device__ inline V over16(V v, F f) {
  auto step = [&](auto ctrl) {
    const int b = __builtin_bit_cast(int, v);
    v = f(v, __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(b, b, decltype(ctrl)::value, 0xf, 0xf, true)));
  };
  using std::integral_constant;
  step(integral_constant<int, 0x128>{});   // row_ror:8, :4, :2, :1
  step(integral_constant<int, 0x124>{});
  step(integral_constant<int, 0x122>{});
  step(integral_constant<int, 0x121>{});
  return v;
}

// A reduction over the L lanes of a row of logits, the same in each of them.  `slot`: LDS for a row of 256.
template <int L, class V, class F>
__device__ inline V over_row(V v, V* slot, F f) {
  v = over16(v, f);
  // rows of 16 lanes in pairs, then halves of the wave: a swap leaves one of the two in each operand, which the compiler
  // must not take for the same value
  auto swap = [&](auto how) __attribute__((always_inline)) {
    uint32_t x = __builtin_bit_cast(uint32_t, v), y = x;
    asm("" : "+v"(y));
    const auto both = how(x, y);
    v = f(__builtin_bit_cast(V, uint32_t(both[0])), __builtin_bit_cast(V, uint32_t(both[1])));
  };
  if constexpr (L >= 32) swap([](uint32_t x, uint32_t y) { return __builtin_amdgcn_permlane16_swap(x, y, false, false); });
  if constexpr (L >= 64) swap([](uint32_t x, uint32_t y) { return __builtin_amdgcn_permlane32_swap(x, y, false, false); });
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
  static constexpr int N = L > 64 ? L / 64 : 1;
  float f[N];
  int i[N];
  uint32_t u[N];
};
template <int L>
__device__ inline float row_max(float v, Slots<L>& s) { return over_row<L>(v, s.f, [](float a, float b) { return fmaxf(a, b); }); }
template <int L>
__device__ inline float row_sum(float v, Slots<L>& s) { return over_row<L>(v, s.f, [](float a, float b) { return a + b; }); }
template <int L>
__device__ inline int row_max(int v, Slots<L>& s) { return over_row<L>(v, s.i, [](int a, int b) { return max(a, b); }); }
template <int L>
__device__ inline int row_min(int v, Slots<L>& s) { return over_row<L>(v, s.i, [](int a, int b) { return min(a, b); }); }
template <int L>
__device__ inline uint32_t row_min(uint32_t v, Slots<L>& s) { return over_row<L>(v, s.u, [](uint32_t a, uint32_t b) { return min(a, b); }); }

// Whole numbers in the order of the floats; -0 is 0, NaN is -inf.
__device__ inline int ordered(float v) {
  const int b = __float_as_int(v > -INFINITY ? v + 0.f : -INFINITY);
  return b ^ ((b >> 31) & 0x7fffffff);
}

// L lanes a row, J vectors each: element (j L + t) W + i of the row is number j W + i of lane t.
template <class T, int L, int J>
struct Held {
  static constexpr int W = T::W, N = J * W, MOST = L * N;
  __device__ static int place(int t, int n) { return ((n / W) * L + t) * W + n % W; }
  // Read ahead, and in place; past the row's end -inf.
  __device__ static void load(const char* row, int t, int experts, u32x4_t (&q)[J]) {
    if (experts % W == 0) {
#pragma unroll
      for (int j = 0; j < J; ++j) q[j] = load_ahead<T, false>(row, (j * L + t) * W, experts);
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) q[j] = load_ahead<T, true>(row, (j * L + t) * W, experts);
    }
  }
  __device__ static void values(const u32x4_t (&q)[J], int t, int experts, float (&v)[N]) {
    if (experts % W == 0) {
#pragma unroll
      for (int j = 0; j < J; ++j) T::unpack(q[j], v + j * W);
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) T::unpack(settle<T, true>(q[j], (j * L + t) * W, experts), v + j * W);
    }
    if (experts < MOST) {
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] = place(t, n) < experts ? v[n] : -INFINITY;
    }
  }
};

// The row's `top` best, exactly, by value and, of equal values, by place: the row is read again for each of them.
// put(j, place) is called by one lane for each j.
template <class T, int L, int J, class F>
__device__ inline void pick_exact(const char* row, int t, int experts, int top, Slots<L>& slots, F put) {
  int last = INT32_MAX, at = -1;   // the last one's order and place
  for (int j = 0; j < top; ++j) {
    int best = INT32_MIN, first = INT32_MAX;
#pragma unroll 1
    for (int u = 0; u < J; ++u) {
      float v[T::W];
      load_vec<T>(row, (u * L + t) * T::W, experts, -INFINITY, v);
#pragma unroll
      for (int i = 0; i < T::W; ++i) {
        const int place = (u * L + t) * T::W + i, k = ordered(v[i]);
        const bool better = place < experts && k > best && (k < last || (k == last && place > at));
        best = better ? k : best;
        first = better ? place : first;
      }
    }
    last = row_max<L>(best, slots);
    at = row_min<L>(best == last ? first : INT32_MAX, slots);
    if (t == 0) put(j, at);
  }
}

// The same by keys of 32 bits: the value's order above the complement of the place, so that no two are the same and
// a key tells its place (past the row's end they are those of -inf, behind all others).  The next best is the one that
// is least below the last: one subtraction and half a minimum for each value.  Not for rows with NaN.  A bf16 value has its 16 bits beside a place of 16.  Of an fp32 value the last bits make way for
// the place: one key more is taken, and where two neighbours in the list are the same in what is left, keys are taken
// until the list's end is clear and its entries ranked by their whole values (256 scores: one row in 200).  Rows whose
// list would pass the L lanes are picked exactly: many of the same value, all of them for a router that starts at zero, and
// all fp32 rows with as many choices as lanes or more: 16 of up to 256 experts, 32 of up to 512, 64 of up to 1024 (32768 x
// 256, 15 and 16 of fp32 49 and 83 us, of bf16 29 each).
template <class T, int L, int J>
struct Keys {
  static constexpr int N = Held<T, L, J>::N;
  static constexpr bool EXACT = T::kBytes == 2;
  static constexpr uint32_t places = EXACT ? 0xffffu : uint32_t(Held<T, L, J>::MOST - 1);   // of a power of two
  static_assert(((places + 1) & places) == 0 && places >= uint32_t(Held<T, L, J>::MOST - 1), "a bit for each");
  uint32_t key[N];
  __device__ Keys(const float (&v)[N], int t) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int b = __float_as_int(v[n] + 0.f);
      const uint32_t u = uint32_t(b) ^ (uint32_t(b >> 31) | 0x80000000u);
      key[n] = ((u & ~places) | (places - uint32_t(Held<T, L, J>::place(t, 0)))) - uint32_t(Held<T, L, J>::place(0, n));
    }
  }
  template <class F>
  __device__ bool pick(const char* row, int t, int experts, int top, Slots<L>& slots, F put) const;
};

template <class T, int L, int J>
template <class F>
__device__ inline bool Keys<T, L, J>::pick(const char* row, int t, int experts, int top, Slots<L>& slots, F put) const {
  if constexpr (!EXACT) {
    if (L > 64 || top >= L) return false;
  }
  uint32_t below = 0xffffffffu;   // the next key is this or less
  auto next = [&]() __attribute__((always_inline)) {
    uint32_t least = below - key[0];
#pragma unroll
    for (int n = 1; n < N; ++n) least = min(least, below - key[n]);
    const uint32_t found = below - row_min<L>(least, slots);
    below = found - 1u;
    return found;
  };
  uint32_t mine = 0u;   // key t of the list (of a long bf16 list, of the last L)
  if constexpr (EXACT) {
    for (int from = 0; from < top; from += L) {
      const int here = min(top - from, L);
      for (int j = 0; j < here; ++j) {
        const uint32_t found = next();
        mine = t == j ? found : mine;
      }
      if (t < here) put(from + t, int(places - (mine & places)));
    }
  } else {
    int n = min(top + 1, experts);
    uint32_t end = 0u, last = 0u;   // the last two keys
    for (int j = 0; j < n; ++j) {
      last = end;
      end = next();
      mine = t == j ? end : mine;
    }
    const uint32_t before = __shfl_up(mine, 1);   // of lane t - 1
    const bool same = t > 0 && t < n && ((before ^ mine) & ~places) == 0u;
    if (row_min<L>(same ? 0 : 1, slots) != 0) {
      if (t < top) put(t, int(places - (mine & places)));
      return true;
    }
    while (n < L && n < experts && ((end ^ last) & ~places) == 0u) {
      last = end;
      end = next();
      mine = t == n ? end : mine;
      ++n;
    }
    if (n < experts && ((end ^ last) & ~places) == 0u) return false;
    const int place = int(places - (mine & places));
    const int order = t < n && place < experts ? ordered(T::load1(row + int64_t(place) * T::kBytes)) : INT32_MIN;
    int rank = 0;
    for (int i = 0; i < n; ++i) {
      const int from = int(threadIdx.x & 63) - t + i, other = __shfl(order, from), there = __shfl(place, from);
      rank += other > order || (other == order && there < place) ? 1 : 0;
    }
    if (t < n && rank < top) put(rank, place);
  }
  return true;
}

// LDS of one wave: what one lane has written the others read.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Exclusive sums of the experts' bits, by one wave.
__device__ inline void starts(const uint64_t* mask, int* before, int experts) {
  const int lane = threadIdx.x & 63;
  int sum = 0;
  for (int base = 0; base < experts; base += 64) {
    const int e = base + lane, n = e < experts ? __popcll(mask[e]) : 0;
    int scan = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(scan, o);
      if (lane >= o) scan += up;
    }
    if (e < experts) before[e] = sum + scan - n;
    sum += __shfl(scan, 63);
  }
}

// The balance loss from sum_e c_e (sum of the rows' p_e) and the number of choices.
__device__ inline float balance_of(const RouteArgs& A, double dot, int used) {
  return used > 0 ? float(double(A.experts) * dot * double(A.top) / (double(used) * double(used))) : 0.f;
}

// Threads of a block of rows.
template <int L>
constexpr int route_threads() { return L > 64 ? 256 : 512; }

template <class T, int L, int J>
__global__ __launch_bounds__(route_threads<L>(), L > 64 ? 1 : 4) void k_route(const RouteArgs A) {
  using H = Held<T, L, J>;
  constexpr int N = H::N, NT = route_threads<L>(), G = NT / L;
  __shared__ uint64_t mask[H::MOST];
  __shared__ int before[H::MOST];
  __shared__ float sums[L > 64 ? 1 : NT / 64][H::MOST];
  __shared__ __attribute__((aligned(8))) float share[kRows * TM_MAX_TOP], whole[kRows];
  __shared__ uint16_t sel[kRows * TM_MAX_TOP];
  __shared__ Slots<L> slots;
  const int t = threadIdx.x % L, grp = threadIdx.x / L, experts = A.experts, top = A.top;
  float acc[N];
#pragma unroll
  for (int n = 0; n < N; ++n) acc[n] = 0.f;
  for (int e = threadIdx.x; e < experts; e += NT) before[e] = 0;
  for (int turn = 0; turn < A.turns; ++turn) {
    const int64_t first = (int64_t(blockIdx.x) * A.turns + turn) * kRows;
    const int rows = int(min(int64_t(kRows), A.rows - first));
    if (rows <= 0) break;
    for (int e = threadIdx.x; e < experts; e += NT) mask[e] = 0;
    __syncthreads();
    auto active = [&](int at) { return at < rows && (A.active == nullptr || A.active[first + at] != 0); };
    u32x4_t q[J];
    constexpr bool AHEAD = T::kBytes == 2 || J < 4;   // registers
    bool on = active(grp);
    if (AHEAD && on) H::load(A.logits + (first + grp) * A.ld * T::kBytes, t, experts, q);
    for (int at = grp; at < rows; at += G) {
      const bool now = on;
      float v[N];
      if (!AHEAD && now) H::load(A.logits + (first + at) * A.ld * T::kBytes, t, experts, q);
      if (now) H::values(q, t, experts, v);
      // the next row is on its way while this one is worked on
      on = active(at + G);
      if (AHEAD && on) H::load(A.logits + (first + at + G) * A.ld * T::kBytes, t, experts, q);
      if (!now) {
        if (t == 0) whole[at] = -1.f;
        continue;
      }
      const char* row = A.logits + (first + at) * A.ld * T::kBytes;
      float m = v[0];
#pragma unroll
      for (int n = 1; n < N; ++n) m = fmaxf(m, v[n]);
      m = row_max<L>(m, slots);
      const Keys<T, L, J> keys(v, t);
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        v[n] = __builtin_amdgcn_exp2f((v[n] - m) * kLog2e);
        sum += v[n];
      }
      sum = row_sum<L>(sum, slots);
      const float inv = 1.f / sum;
#pragma unroll
      for (int n = 0; n < N; ++n) acc[n] += v[n] * inv;
      auto put = [&](int j, int place) { sel[at * top + j] = uint16_t(place); };
      if (sum != sum || !keys.pick(row, t, experts, top, slots, put)) pick_exact<T, L, J>(row, t, experts, top, slots, put);
      wave_sync();
      float chosen = 0.f;
      for (int j = t; j < top; j += L) {
        const int e = sel[at * top + j];
        const float p = __builtin_amdgcn_exp2f((T::load1(row + int64_t(e) * T::kBytes) - m) * kLog2e);
        share[at * top + j] = p;
        chosen += p;
        atomicOr((unsigned long long*)&mask[e], 1ull << at);
      }
      chosen = row_sum<L>(chosen, slots);
      // a sum that is not a number shows in the weights either way
      if (t == 0) whole[at] = A.renormalize ? chosen + 0.f * sum : sum;
    }
    __syncthreads();
    if (A.blocks == 1) {   // one turn: what stands before the experts' choices is known at once
      if (threadIdx.x < 64) starts(mask, before, experts);
      __syncthreads();
    }
    for (int i = threadIdx.x; i < rows * top; i += NT) {
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
    for (int e = threadIdx.x; e < experts; e += NT) before[e] += __popcll(mask[e]);
  }
  // the groups of a wave, then the waves
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int o = L; o < 64; o *= 2) acc[n] += __shfl_xor(acc[n], o);
  if (L > 64 || (threadIdx.x & 63) < L) {
#pragma unroll
    for (int n = 0; n < N; ++n) sums[L > 64 ? 0 : threadIdx.x / 64][H::place(t, n)] = acc[n];
  }
  __syncthreads();
  if (A.blocks == 1) {
    // the counts have been added to what stands before them; the choices are their differences
    double dot = 0.0;
    for (int e = threadIdx.x; e < experts; e += NT) {
      float s = 0.f;
      for (int w = 0; w < (L > 64 ? 1 : NT / 64); ++w) s += sums[w][e];
      A.ends[e] = before[e];
      dot += double(s) * double(before[e] - (e > 0 ? before[e - 1] : 0));
    }
    const int used = before[experts - 1];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
    double* parts = reinterpret_cast<double*>(share);
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < NT / 64; ++w) dot += parts[w];
      *A.balance = balance_of(A, dot, used);
    }
    return;
  }
  const int width = (experts + 7) / 8 * 8;
  for (int e = threadIdx.x; e < width; e += NT) {
    float s = 0.f;
    if (e < experts)
      for (int w = 0; w < (L > 64 ? 1 : NT / 64); ++w) s += sums[w][e];
    A.counts[int64_t(blockIdx.x) * width + e] = uint16_t(e < experts ? before[e] : 0);
    A.shares[int64_t(blockIdx.x) * width + e] = s;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *A.arrived = 0;   // for k_route_place
}

constexpr int kPlace = 1024;

typedef uint16_t u16x8_t __attribute__((ext_vector_type(8)));

// SPAN blocks of k_route a workgroup, as many as leave one workgroup a CU or so, each a share of its threads (us of the
// call by one, two and four: 32768 x 256 in 512 blocks 32, 28, 28; 16384 x 512 in 256 25, 25, 26; 45000 x 128 in 704
// two 27, four 24); the first workgroup writes ends.  The balance loss is
// added up by vectors of eight experts, dealt out among the workgroups, and by the last of these to arrive.
template <int MOST, int SPAN>
__global__ __launch_bounds__(kPlace) void k_route_place(const RouteArgs A) {
  // expert 8 v + i at i vecs + v: neighbouring lanes, neighbouring words
  __shared__ int total[MOST], base[SPAN][MOST], waves[kPlace / 64];
  __shared__ double parts[kPlace / 64];
  constexpr int PER = (MOST + kPlace - 1) / kPlace, SHARE = kPlace / SPAN;
  const int experts = A.experts, width = (experts + 7) / 8 * 8, tid = threadIdx.x, lane = tid & 63;
  const int own = int(blockIdx.x) * SPAN, vecs = width / 8;
  auto word = [&](int e) { return (e % 8) * vecs + e / 8; };
  // what is needed last is asked for first: this thread's choices, its experts' counts in the blocks, and the first of
  // the sums of probabilities that it adds up (vector blockIdx.x + m gridDim.x, block, half)
  const int share = tid / SHARE, block = own + share;
  const int64_t entries = int64_t(A.turns) * kRows * A.top, first = int64_t(block) * entries + tid % SHARE;
  const int64_t last = block < A.blocks ? min(int64_t(block + 1) * entries, int64_t(A.rows) * A.top) : 0;
  constexpr int EARLY = 2;
  int chosen[EARLY], at[EARLY];
#pragma unroll
  for (int i = 0; i < EARLY; ++i) {
    chosen[i] = first + i * SHARE < last ? A.chosen[first + i * SHARE] : -1;
    at[i] = first + i * SHARE < last ? A.slots[first + i * SHARE] : 0;
  }
  int count[PER > 1 ? 1 : SPAN];
  if constexpr (PER == 1) {
#pragma unroll
    for (int u = 0; u < SPAN; ++u)
      count[u] = own + u < A.blocks && tid < experts ? A.counts[int64_t(own + u) * width + tid] : 0;
  }
  const int grid = int(gridDim.x), summers = min(grid, vecs);   // workgroups that have sums to add up
  const int64_t sums = int(blockIdx.x) < vecs ? int64_t((vecs - 1 - int(blockIdx.x)) / grid + 1) * A.blocks * 2 : 0;
  auto expert_of = [&](int64_t i) { return (int(blockIdx.x) + int(i / 2 / A.blocks) * grid) * 8 + int(i % 2) * 4; };
  auto sums_at = [&](int64_t i) {
    return *reinterpret_cast<const float4*>(A.shares + (i / 2) % A.blocks * width + expert_of(i));
  };
  float4 early = make_float4(0.f, 0.f, 0.f, 0.f);
  if (tid < sums) early = sums_at(tid);
  for (int e = tid; e < width; e += kPlace) total[e] = base[0][e] = 0;
  __syncthreads();
  // the blocks' counts: vectors of eight experts, `pitch` lanes for them, the blocks dealt out among the rest
  int pitch = 16;
  while (pitch < vecs && pitch < kPlace) pitch *= 2;
  const int step = kPlace / pitch, each = A.turns <= 65535 / (8 * kRows) ? 8 : 1;   // counts that 16 bits hold the sum of
  for (int v = tid % pitch; v < (vecs + pitch - 1) / pitch * pitch; v += pitch) {
    int all[8] = {}, low[8] = {};
    for (int b = tid / pitch; v < vecs && b < A.blocks; b += 8 * step) {
      u16x8_t q[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        q[u] = u16x8_t{0, 0, 0, 0, 0, 0, 0, 0};
        if (b + u * step < A.blocks) q[u] = *reinterpret_cast<const u16x8_t*>(A.counts + int64_t(b + u * step) * width + v * 8);
      }
      auto add = [&](u16x8_t every, u16x8_t before) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          all[i] += every[i];
          low[i] += before[i];
        }
      };
      const u16x8_t none = u16x8_t{0, 0, 0, 0, 0, 0, 0, 0};
      u16x8_t every = none, before = none;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        every += q[u];
        before += b + u * step < own ? q[u] : none;
        if (each == 1) {
          add(every, before);
          every = before = none;
        }
      }
      add(every, before);
    }
    for (int o = pitch; o < 64; o *= 2)   // lanes of the same experts
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        all[i] += __shfl_xor(all[i], o);
        low[i] += __shfl_xor(low[i], o);
      }
    if (v < vecs && lane < pitch) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        atomicAdd(&total[i * vecs + v], all[i]);
        atomicAdd(&base[0][i * vecs + v], low[i]);
      }
    }
  }
  __syncthreads();
  // exclusive sums of the totals: PER neighbouring experts a thread
  int mine[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    mine[i] = tid * PER + i < experts ? total[word(tid * PER + i)] : 0;
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
  // where each block's choices of an expert begin
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = tid * PER + i;
    if (e >= experts) continue;
    int from = base[0][word(e)] + start;
    if constexpr (PER > 1) {
      static_assert(PER == 1 || SPAN == 1, "one block's");
      base[0][word(e)] = from;
    } else {
#pragma unroll
      for (int u = 0; u < SPAN; ++u) {
        base[u][word(e)] = from;
        from += count[u];
      }
    }
    start += mine[i];
    if (blockIdx.x == 0) A.ends[e] = start;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < EARLY; ++i)
    if (chosen[i] >= 0) A.slots[first + i * SHARE] = at[i] + base[share][word(chosen[i])];
  for (int64_t i = first + EARLY * SHARE; i < last; i += SHARE) {
    const int e = A.chosen[i];
    if (e >= 0) A.slots[i] += base[share][word(e)];
  }
  if (int(blockIdx.x) >= summers) return;
  double dot = 0.0;
  for (int64_t i = tid; i < sums; i += kPlace) {
    const float4 p = i == tid ? early : sums_at(i);
    const int e = expert_of(i);
    dot += double(p.x) * double(total[word(e)]) + double(p.y) * double(total[word(e + 1)]) +
           double(p.z) * double(total[word(e + 2)]) + double(p.w) * double(total[word(e + 3)]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
  if (lane == 0) parts[tid >> 6] = dot;
  __syncthreads();
  if (tid >= 64) return;
  dot = 0.0;
  for (int w = 0; w < kPlace / 64; ++w) dot += parts[w];
  if (summers > 1) {
    // The part is written through to memory and waited for before the count goes up; the one who finds the count full
    // reads the parts from memory.  A release would write back the whole cache for one value.
    int arrived = 0;
    if (tid == 0) {
      __hip_atomic_store(&A.dots[blockIdx.x], dot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      arrived = __hip_atomic_fetch_add(A.arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (__builtin_amdgcn_readfirstlane(arrived) + 1 != summers) return;
    asm volatile("" ::: "memory");   // no part is read before
    dot = 0.0;
    for (int i = tid; i < summers; i += 64)   // in the workgroups' order
      dot += __hip_atomic_load(&A.dots[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
  }
  if (tid == 0) *A.balance = balance_of(A, dot, used);
}

constexpr int kThreads = 256;

// What the lanes of a row have written in LDS the others read.
template <int L>
__device__ inline void group_sync() {
  if constexpr (L > 64) __syncthreads();
  else wave_sync();
}

// Backward: the row's lanes take a choice each (L at a time) and put its share of the gradient where the expert's lane
// finds it.  A choice that the caller names twice counts twice, in the order of the choices.  32768 rows of 256 experts,
// 8 of fp32, 21 us and 67 MB: bound by the row's chain of loads, six reductions and LDS, about 600 vector
// instructions a wave for four rows; 73% of the waves' time was waiting with nothing of the next row read ahead (24 us).
template <class T, int L, int J>
__global__ __launch_bounds__(kThreads, L > 64 ? 1 : 4) void k_route_backward(const RouteGradArgs A) {
  using H = Held<T, L, J>;
  constexpr int N = H::N, G = kThreads / L;
  __shared__ Slots<L> slots;
  __shared__ __attribute__((aligned(16))) float extra[G][H::MOST];
  __shared__ __attribute__((aligned(16))) int2 picks[G][TM_MAX_TOP];   // expert and gradient, to whole runs of four
  const int t = threadIdx.x % L, grp = threadIdx.x / L, experts = A.experts, top = A.top, wide = (top + 3) / 4 * 4;
  const float used = float(A.ends[experts - 1]), taking = used / float(top);
  const float per = A.dbalance != nullptr && used > 0.f ? *A.dbalance * float(experts) / (used * taking) : 0.f;
  float u[N];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int first = (j * L + t) * T::W;
    int last = first > 0 && first <= experts ? A.ends[first - 1] : 0;
#pragma unroll
    for (int i = 0; i < T::W; ++i) {
      const int end = first + i < experts ? A.ends[first + i] : last;
      u[j * T::W + i] = per * float(end - last);
      last = end;
    }
  }
  constexpr bool AHEAD = T::kBytes == 2 || J < 4;   // registers
  const int64_t step = int64_t(gridDim.x) * G;
  int64_t r = int64_t(blockIdx.x) * G + grp;
  // a row's values, whether it takes part, and this lane's first choice: its expert (-1: none) and, of the gradients,
  // dw scale.  The next row's are on their way while this one is worked on.
  u32x4_t q[J];
  int part = -1, own = -1;
  float own_at = 0.f;
  const bool gradients = A.dweights != nullptr, shared = gradients && A.renormalize;
  auto read = [&](int64_t at) __attribute__((always_inline)) {
    part = A.chosen[at * top];
    if (gradients && t < top) {
      own = A.chosen[at * top + t];
      own_at = A.dweights[at * top + t];
    }
    if constexpr (AHEAD) H::load(A.logits + at * A.ld * T::kBytes, t, experts, q);
  };
  if (r < A.rows) read(r);
  for (; r < A.rows; r += step) {
    const char* row = A.logits + r * A.ld * T::kBytes;
    char* out = A.dlogits + r * A.ldd * T::kBytes;
    float v[N];
    if constexpr (!AHEAD) H::load(row, t, experts, q);
    const bool on = part >= 0;
    const int first = own >= 0 && own < experts ? own : -1;
    const float first_at = A.scale * own_at;
    float first_l = -INFINITY;
    if (on && shared && first >= 0) first_l = T::load1(row + int64_t(first) * T::kBytes);
    H::values(q, t, experts, v);
    if (r + step < A.rows) read(r + step);
    if (!on) {
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] = 0.f;
    } else {
      // choice j of this lane
      auto choice = [&](int j, float& at, float& l) __attribute__((always_inline)) {
        if (j < L) {
          at = first_at;
          l = first_l;
          return first;
        }
        const int e = A.chosen[r * top + j];
        const bool there = e >= 0 && e < experts;
        at = A.scale * A.dweights[r * top + j];
        l = there && shared ? T::load1(row + int64_t(e) * T::kBytes) : -INFINITY;
        return there ? e : -1;
      };
      float most = -INFINITY, whole = 0.f, mean = 0.f;
      if (shared) {   // the chosen's softmax, about their own maximum
        float at, l;
        for (int j = t; j < top; j += L)
          if (choice(j, at, l) >= 0) most = fmaxf(most, l);
        most = row_max<L>(most, slots);
        for (int j = t; j < top; j += L) {
          if (choice(j, at, l) < 0) continue;
          const float p = expf(l - most);
          whole += p;
          mean += p * at;
        }
        whole = row_sum<L>(whole, slots);
        mean = row_sum<L>(mean, slots) / whole;
      }
      if (gradients) {
#pragma unroll
        for (int n = 0; n < N; ++n) extra[grp][H::place(t, n)] = 0.f;
        for (int j = t; j < wide; j += L) {
          float at = 0.f, l;
          const int e = j < top ? choice(j, at, l) : -1;
          if (e >= 0 && shared) at = expf(l - most) / whole * (at - mean);
          picks[grp][j] = make_int2(e, __float_as_int(at));
        }
        group_sync<L>();
        for (int j = t; j < top; j += L) {
          const int e = picks[grp][j].x;
          float sum = 0.f;
          for (int i = 0; i < wide; i += 4) {
            const int4 p = *reinterpret_cast<const int4*>(&picks[grp][i]), q = *reinterpret_cast<const int4*>(&picks[grp][i + 2]);
            sum += p.x == e ? __int_as_float(p.y) : 0.f;
            sum += p.z == e ? __int_as_float(p.w) : 0.f;
            sum += q.x == e ? __int_as_float(q.y) : 0.f;
            sum += q.z == e ? __int_as_float(q.w) : 0.f;
          }
          if (e >= 0) extra[grp][e] = sum;
        }
        group_sync<L>();
      }
      float m = v[0];
#pragma unroll
      for (int n = 1; n < N; ++n) m = fmaxf(m, v[n]);
      m = row_max<L>(m, slots);
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        v[n] = H::place(t, n) < experts ? __builtin_amdgcn_exp2f((v[n] - m) * kLog2e) : 0.f;
        sum += v[n];
      }
      sum = row_sum<L>(sum, slots);
      const float inv = 1.f / sum;
      auto more = [&](int n) __attribute__((always_inline)) { return gradients ? extra[grp][H::place(t, n)] : 0.f; };
      float dot = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        v[n] *= inv;
        dot += v[n] * (A.renormalize ? u[n] : u[n] + more(n));
      }
      dot = row_sum<L>(dot, slots);
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] = A.renormalize ? v[n] * (u[n] - dot) + more(n) : v[n] * (u[n] + more(n) - dot);
      if (gradients) group_sync<L>();   // before the next row's zeros
    }
#pragma unroll
    for (int j = 0; j < J; ++j) store_vec<T>(out, (j * L + t) * T::W, experts, v + j * T::W);
  }
}

// f(L, J) with the lanes of a row and vectors of each that hold `experts`: the fewest lanes whose registers hold a row, as
// the reductions over them cost more than the rounds in a lane (us, with twice the lanes: forward 32768 x 256, 8 of fp32,
// 28 and 30, bf16 25 and 28, 16384 x 512 29 and 33, bf16 26 and 30, 65536 x 128, 6 of fp32, 27 and 34; 8192 x 1024 42, by
// 256 lanes, which meet at barriers and pick fp32 exactly, 604; backward alike up to 512, 20 and 25 for 65536 x 128).
template <class T, class F>
void with_shape(int experts, F f) {
  using std::integral_constant;
  constexpr int W = T::W;
  if (experts <= 16 * W) f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  else if (experts <= 128) f(integral_constant<int, 16>{}, integral_constant<int, 8 / W>{});
  else if (experts <= 256) f(integral_constant<int, 16>{}, integral_constant<int, 16 / W>{});
  else if (experts <= 512) f(integral_constant<int, 32>{}, integral_constant<int, 16 / W>{});
  else if (experts <= 1024) f(integral_constant<int, 64>{}, integral_constant<int, 16 / W>{});
  else f(integral_constant<int, 256>{}, integral_constant<int, 32 / W>{});
}

template <class T>
hipError_t forward(const RouteArgs& A, hipStream_t st) {
  with_shape<T>(A.experts, [&](auto l, auto j) {
    constexpr int L = decltype(l)::value;
    hipLaunchKernelGGL((k_route<T, L, decltype(j)::value>), dim3(A.blocks), dim3(route_threads<L>()), 0, st, A);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || A.blocks == 1) return e;
  if (A.experts > 1024) {
    hipLaunchKernelGGL((k_route_place<TM_MAX_EXPERTS, 1>), dim3(A.blocks), dim3(kPlace), 0, st, A);
  } else if (A.blocks <= 256) {
    hipLaunchKernelGGL((k_route_place<1024, 1>), dim3(A.blocks), dim3(kPlace), 0, st, A);
  } else if (A.blocks <= 512) {
    hipLaunchKernelGGL((k_route_place<1024, 2>), dim3((A.blocks + 1) / 2), dim3(kPlace), 0, st, A);
  } else {
    hipLaunchKernelGGL((k_route_place<1024, 4>), dim3((A.blocks + 3) / 4), dim3(kPlace), 0, st, A);
  }
  return hipGetLastError();
}

template <class T>
hipError_t backward(const RouteGradArgs& A, hipStream_t st) {
  with_shape<T>(A.experts, [&](auto l, auto j) {
    constexpr int G = kThreads / decltype(l)::value;
    // as many as are resident, each of which reads `ends` once (us by 512, 1024 and 2048: 32768 x 256, 8 of fp32, 26, 24,
    // 29; 65536 x 128, 6 of bf16, 32, 23, 27)
    const dim3 grid(uint32_t(std::min<int64_t>((int64_t(A.rows) + G - 1) / G, 1024)));
    hipLaunchKernelGGL((k_route_backward<T, decltype(l)::value, decltype(j)::value>), grid, dim3(kThreads), 0, st, A);
  });
  return hipGetLastError();
}

}  // namespace route

void plan_route(RouteArgs& A) {
  // Every workgroup of the second launch reads all counts: fewer blocks, of more turns, where there are many experts or
  // rows (us with about 256, 512 and 1024 blocks: 65536 x 128, 6 of bf16, 28, 26, 29; 131072 x 64, 6 of bf16, 44, 37, 40;
  // 32768 x 256, 8 of fp32, 27 each); 40000 x 200, 8 of fp32, in 625 blocks of one turn 35, in 313 of two 37.
  const int64_t runs = std::max<int64_t>((int64_t(A.rows) + kRouteRows - 1) / kRouteRows, 1);
  const int64_t about = std::clamp<int64_t>((1 << 18) / A.experts, 64, 512);
  const int64_t turns = std::clamp<int64_t>((runs + about / 2) / about, 1, 65535 / kRouteRows);
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
