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
// The logits are read once.  Each thread keeps the maximum of what it has seen and, in
// powers of 2, the sums of e and of e u about a value that follows the maximum at a
// distance: they are moved to another value only when a logit is 2^24 times as likely as
// it, so that hardly a row moves them twice.  (With a move for every vector 4096 x 131072
// took 335 us, so 152.)  They are joined at the end of a row.
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
//
// Long rows and the backward pass are bound by HBM (in brackets the bytes at the 5.04 TB/s of
// a large copy): 4096 x 131072 bf16, 5 alternatives, a quarter of the rows without target,
// 152 us (160).  Short rows by instructions: 32768 x 1000 bf16 16 us (13), with 5
// alternatives 27, as picking is half of a row's instructions.  A few rows by chains of
// waits: 16 x 50257 bf16 7 us in the kernel, with 20 alternatives 14, picked by one wave.
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
// What a thread has seen: `m` the maximum; s the sum of e = exp2((l - at) c) and t that of e (l - at) c, about a value
// `at` that follows the maximum at a distance: it moves when a logit passes `limit`, where e is 2^kAbove.
constexpr float kAbove = 24.f;
struct Sums {
  float m = -INFINITY, at = -INFINITY, limit = -INFINITY, s = 0.f, t = 0.f;
};

// The sums about another value.
__device__ inline void move_to(Sums& a, float at, float c) {
  const float by = (a.at - at) * c;
  const float f = a.at == -INFINITY ? 0.f : exp2_fast(by);   // nothing was summed about -inf
  a.t = (a.t + a.s * fmaxf(by, kFar)) * f;
  a.s *= f;
  a.at = at;
}

// The largest of N values; NaN counts as -inf.
template <int N>
__device__ inline float largest(const float* v) {
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, v[i]);
  return m;
}

// Adds N logits whose maximum is m.  FILLED: some of them may be the -inf past a row's end, where e u is held at 0;
// else that is done only where one is met.
template <int N, bool FILLED>
__device__ inline void add_terms(Sums& a, const float* v, float m, float c, float above) {
  a.m = fmaxf(a.m, m);
  if (m > a.limit) {
    move_to(a, m, c);
    a.limit = m + above;
  }
  const float at = a.at == -INFINITY ? 0.f : a.at;   // terms of -inf are exp(-inf - 0) = 0
  float s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float u = (v[i] - at) * c, e = exp2_fast(u);
    s[i % 2] += e;
    t[i % 2] += e * (FILLED ? fmaxf(u, kFar) : u);
  }
  t[0] += t[1];
  if (!FILLED && __ballot(t[0] != t[0]) != 0) {   // 0 (-inf), which is 0; a value that is not a number shows in s
    float from = at;
    asm volatile("" : "+v"(from));   // keeps this out of the way that all other terms take
    t[0] = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float u = (v[i] - from) * c;
      t[0] += exp2_fast(u) * fmaxf(u, kFar);
    }
  }
  a.s += s[0] + s[1];
  a.t += t[0];
}

// Entries at .. at + W - 1 of a row that ends at `last`, at a multiple of W, and what they are; -inf past the end.
template <class T>
__device__ inline u32x4_t load_to(const char* l, int at, int last) {
  return last % T::W == 0 ? load_ahead<T, false>(l, at, last) : load_ahead<T, true>(l, at, last);
}
template <class T>
__device__ inline void values_to(u32x4_t q, int at, int last, float* v) {
  if (last % T::W == 0) {   // whole, or wholly past the end
    T::unpack(q, v);
    if (at >= last)
#pragma unroll
      for (int i = 0; i < T::W; ++i) v[i] = -INFINITY;
  } else {
    T::unpack(settle<T, true>(q, at, last), v);
    if (at + T::W > last)
#pragma unroll
      for (int i = 0; i < T::W; ++i) v[i] = at + i < last ? v[i] : -INFINITY;
  }
}

// m, and the sums about it.
struct Joined {
  float m, s, t;
};

template <class T>
__device__ inline void write_row(const LogpArgs& A, int64_t r, int64_t y, Joined a) {
  const float log_sum = logf(a.s);
  const float ly = y < A.vocab ? T::load1(A.logits + (r * A.ld + y) * T::kBytes) : NAN;
  A.logp[r] = (ly - a.m) * A.inv_temp - log_sum;
  A.entropy[r] = log_sum - a.t * kLn2 / a.s;
  A.stats[r] = make_float2(a.m, a.s);
}

// ---------------------------------------------------------------- alternatives
typedef uint64_t Key;

// Whole numbers in the order of the floats.
__device__ inline int ordered(float v) {
  const int b = __float_as_int(v + 0.f);   // -0 and 0 are equal
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ inline float value_of(int order) { return __int_as_float(order ^ ((order >> 31) & 0x7fffffff)); }
__device__ inline Key key_of(float v, int place) { return Key(uint32_t(ordered(v)) ^ 0x80000000u) << 32 | uint32_t(~place); }
__device__ inline float value_of(Key k) { return value_of(int(uint32_t(k >> 32) ^ 0x80000000u)); }
__device__ inline int place_of(Key k) { return int(~uint32_t(k)); }

// That of -inf, for what is not there.
constexpr Key kNone = Key(0x007fffffu) << 32;
// Every number but -inf is at least this.
constexpr float kLowest = -3.402823466e38f;

// LDS of one wave: what one lane has written the others read.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The maximum over the wave, the same in every lane: as wave_sum, by data-parallel moves.
__device__ inline int wave_max(int v) {
  auto step = [&](auto ctrl, auto rows) {
    v = max(v, __builtin_amdgcn_update_dpp(v, v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
  };
  using std::integral_constant;
  step(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});   // row_shr:1, :2, :4, :8
  step(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // row_bcast:15, :31
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
  return __builtin_amdgcn_readlane(v, 63);
}

constexpr int kListed = 320;
struct List {
  Key keys[kListed + 8], best[64];
};

// A wave's picking of the `top` best of the entries that it is given.
struct Picker {
  List& list;
  int top, n = 0;
  Key floor = 0;         // keys below it are out
  float low = kLowest;   // and so are values below this

  __device__ Picker(List& l, int k) : list(l), top(k) {}

  // The best `top` of the listed keys, in order.
  __device__ void settle() {
    const int lane = threadIdx.x & 63;
    if (lane < 8) list.keys[n + lane] = 0;   // whole runs of eight
    wave_sync();
    for (int i = lane; i < n; i += 64) {
      const Key mine = list.keys[i];
      int better = 0;
      for (int j = 0; j < n; j += 8)
#pragma unroll
        for (int u = 0; u < 8; ++u) better += list.keys[j + u] > mine ? 1 : 0;
      if (better < top) list.best[better] = mine;
    }
    wave_sync();
    n = min(n, top);
    if (lane < n) list.keys[lane] = list.best[lane];
    wave_sync();
    if (n == top) floor = list.keys[top - 1];
  }
  // One entry of each lane (-inf: none).
  __device__ void push(float v, int place) {
    bool in = v >= low;
    if (__ballot(in) == 0) return;
    const Key key = key_of(v, place);
    in = in && key >= floor;
    const uint64_t who = __ballot(in);
    const int lane = threadIdx.x & 63;
    if (in) list.keys[n + __popcll(who & ((uint64_t(1) << lane) - 1))] = key;
    n += __popcll(who);
    if (n > kListed - 64) settle();
  }
  // Raises the bound to the `top`-th best of values of which each lane has one (of different entries), where there
  // are so many: for a few the best is taken away top - 1 times, else it is the least value that fewer than `top` are
  // above.
  __device__ void start(float lanes_best) {
    if (top <= 8) {
      int v = ordered(lanes_best);
      for (int i = 1; i < top; ++i) {
        const uint64_t who = __ballot(v == wave_max(v));
        if ((threadIdx.x & 63) == __ffsll((unsigned long long)who) - 1) v = INT32_MIN;
      }
      low = fmaxf(value_of(wave_max(v)), kLowest);
      return;
    }
    float* values = reinterpret_cast<float*>(list.keys);
    values[threadIdx.x & 63] = lanes_best;
    wave_sync();
    int above = 0;
#pragma unroll
    for (int i = 0; i < 64; ++i) above += values[i] > lanes_best ? 1 : 0;
    wave_sync();
    low = fmaxf(value_of(~wave_max(above < top ? ~ordered(lanes_best) : INT32_MIN)), kLowest);
  }
};

// What was picked of row r, by the lanes of a wave.
__device__ inline void write_top(const LogpArgs& A, int64_t r, const Picker& pick, Joined row) {
  const int lane = threadIdx.x & 63;
  if (lane < A.top) {
    const bool there = lane < pick.n;
    const float v = there ? value_of(pick.list.keys[lane]) : -INFINITY;
    A.top_logp[r * A.top + lane] = (v - row.m) * A.inv_temp - logf(row.s);
    A.top_ids[r * A.top + lane] = there ? place_of(pick.list.keys[lane]) : -1;
  }
}

// The same of a whole row, or of chunk `id` for k_logp_join.
template <class T>
__device__ inline void write_sums(const LogpArgs& A, int64_t id, int64_t r, int64_t y, Joined row) {
  if (A.chunks == 1) write_row<T>(A, r, y, row);
  else A.part[id] = make_float4(row.m, row.s, row.t, 0.f);
}
template <class T>
__device__ inline void write_picked(const LogpArgs& A, int64_t id, int64_t r, const Picker& pick, Joined row) {
  const int lane = threadIdx.x & 63;
  if (A.chunks == 1) write_top(A, r, pick, row);
  else if (lane < A.top) A.keys[id * A.top + lane] = lane < pick.n ? pick.list.keys[lane] : kNone;
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
// The values of the lanes that hold alternatives.
constexpr int kStaged = 24;
template <int N>
struct Staged {
  __attribute__((aligned(16))) float value[kStaged][N];
  int lane[kStaged];
};

// A wave per row, which holds it in registers, K vectors a lane.  The alternatives lie in the lanes whose own best
// reaches the bound (by all lanes' values one after the other 32768 x 1000 with 5 took 30 us, so 27).  (Waves that go on to other rows, the next one on its
// way, are slower: what the compiler keeps from row to row takes the registers of half the waves.)
template <class T, int K, bool TOP>
__global__ __launch_bounds__(256) void k_logp_held(const LogpArgs A) {
  constexpr int W = T::W;
  __shared__ List lists[TOP ? 4 : 1];
  __shared__ Staged<TOP ? K * W : 4> staged[TOP ? 4 : 1];
  const int lane = threadIdx.x & 63, n = A.vocab;
  const int64_t r = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (r >= A.rows) return;
  const int64_t y = A.targets[r];
  if (y < 0) return write_none(A, r, lane);
  const char* l = A.logits + r * A.ld * T::kBytes;
  const float c = A.inv_temp * kLog2e;
  float v[K * W];
  u32x4_t q[K];
#pragma unroll
  for (int j = 0; j < K; ++j) q[j] = load_to<T>(l, (j * 64 + lane) * W, n);
#pragma unroll
  for (int j = 0; j < K; ++j) values_to<T>(q[j], (j * 64 + lane) * W, n, v + j * W);
  const float mine = largest<K * W>(v);
  Sums a;
  a.m = value_of(wave_max(ordered(mine)));
  add_terms<K * W, true>(a, v, a.m, c, 0.f);
  const Joined row{a.m, wave_sum(a.s), wave_sum(a.t)};
  if (lane == 0) write_row<T>(A, r, y, row);
  if constexpr (TOP) {
    Picker pick(lists[threadIdx.x >> 6], A.top);
    pick.start(mine);
    const uint64_t who = __ballot(mine >= pick.low);
    const int lanes = __popcll(who);
    if (lanes <= kStaged) {
      // as few lanes as alternatives reach the bound, but for equal values: theirs alone, dealt out to all
      Staged<K * W>& to = staged[threadIdx.x >> 6];
      if (mine >= pick.low) {
        const int at = __popcll(who & ((uint64_t(1) << lane) - 1));
        to.lane[at] = lane;
#pragma unroll
        for (int e = 0; e < K * W; e += 4) *reinterpret_cast<float4*>(&to.value[at][e]) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
      }
      wave_sync();
      for (int base = 0; base < lanes * K * W; base += 64) {
        const int i = base + lane, at = i / (K * W), e = i % (K * W);
        const bool there = at < lanes;
        const float value = there ? to.value[at][e] : -INFINITY;
        pick.push(value, ((e / W) * 64 + (there ? to.lane[at] : 0)) * W + e % W);
      }
    } else {
#pragma unroll
      for (int e = 0; e < K * W; ++e) pick.push(v[e], ((e / W) * 64 + lane) * W + e % W);
    }
    pick.settle();
    write_top(A, r, pick, row);
  }
}

// Most groups of a chunk; a wave has rows of kWaveBytes at most, and the less LDS, the more of them there are.
constexpr int kGroups = 2048, kWaveBytes = 24 * 1024;
template <class T>
constexpr int group_size() { return 16 * T::W; }

// The maximum over 16 neighbouring lanes, in each of them.
__device__ inline int max16(int v) {
  auto step = [&](auto ctrl) { v = max(v, __builtin_amdgcn_update_dpp(v, v, decltype(ctrl)::value, 0xf, 0xf, true)); };
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
  float best = -INFINITY;
  for (int g = lane; g < groups; g += 64) best = fmaxf(best, maxima[g]);
  pick.start(best);
  for (int base = 0; base < groups; base += 64) {
    const int g = base + lane;
    pick.push(g < groups ? maxima[g] : -INFINITY, g);
  }
  pick.settle();
  // the picked groups, a lane each
  const int found = pick.n;
  const Key mine = lane < found ? pick.list.keys[lane] : Key(0);
  const float worst = found > 0 ? value_of(pick.list.keys[found - 1]) : 0.f;
  wave_sync();
  pick.floor = 0;
  pick.n = 0;
  auto read = [&](int base, float* v) __attribute__((always_inline)) {
    const int from = base + (lane >> 4), g = place_of(__shfl((unsigned long long)mine, from & 63));
    const int at = from < found ? first + g * GROUP + (lane & 15) * W : last;
    values_to<T>(load_to<T>(l, at, last), at, last, v);
    return at;
  };
  float v[W];
  if (found == pick.top) {
    pick.low = worst;   // the groups' best entries reach it
  } else {
    pick.low = kLowest;
    best = -INFINITY;
    for (int base = 0; base < found; base += 4) {
      read(base, v);
      best = fmaxf(best, largest<W>(v));
    }
    pick.start(best);
  }
  for (int base = 0; base < found; base += 4) {
    const int at = read(base, v);
#pragma unroll
    for (int i = 0; i < W; ++i) pick.push(v[i], at + i);
  }
  pick.settle();
}

// NT threads for a row, or a chunk of one.  The next G vectors of a thread are on their way while G are summed.
template <class T, int NT, bool TOP>
__global__ __launch_bounds__(NT) void k_logp_rows(const LogpArgs A) {
  constexpr int W = T::W, STEP = NT * W, G = 4, NW = NT / 64;
  __shared__ float slots[3][NW];
  constexpr int GROUPS = NT > 64 ? kGroups : kWaveBytes / 256;   // of 256 bytes
  __shared__ float maxima[TOP ? GROUPS : 1];
  __shared__ List list[1];
  const int64_t r = blockIdx.x / A.chunks;
  const int64_t y = A.targets[r];
  if (y < 0) {
    if (A.chunks == 1) write_none(A, r, threadIdx.x);
    return;
  }
  const int tid = threadIdx.x;
  const int first = int(blockIdx.x - r * A.chunks) * A.chunk, last = min(A.vocab, first + A.chunk);
  const char* l = A.logits + r * A.ld * T::kBytes;
  const float c = A.inv_temp * kLog2e, above = kAbove / c;
  Sums a;
  u32x4_t q[G];
  auto load = [&](int base) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < G; ++g) q[g] = T::load(l + int64_t(base + g * STEP + tid * W) * T::kBytes);
  };
  int base = first;
  bool more = base + G * STEP <= last;
  if (more) load(base);
  while (more) {
    float v[G * W], m[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      T::unpack(q[g], v + g * W);
      m[g] = largest<W>(v + g * W);
    }
    const int at = (base - first) / group_size<T>();
    base += G * STEP;
    more = base + G * STEP <= last;
    if (more) load(base);
    add_terms<G * W, false>(a, v, largest<G>(m), c, above);
    if constexpr (TOP) {
      int mine = 0;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int best = max16(ordered(m[g]));
        mine = (tid & 15) == g ? best : mine;
      }
      if ((tid & 15) < G) maxima[at + (tid & 15) * (NT / 16) + tid / 16] = value_of(mine);
    }
  }
  for (; base < last; base += STEP) {   // every lane, those past the end with -inf
    const int at = base + tid * W;
    float v[W];
    values_to<T>(load_to<T>(l, at, last), at, last, v);
    const float m = largest<W>(v);
    add_terms<W, true>(a, v, m, c, above);
    if constexpr (TOP) {
      const int best = max16(ordered(m));
      if ((tid & 15) == 0 && at < last) maxima[(at - first) / group_size<T>()] = value_of(best);
    }
  }
  // about the row's maximum, then plain sums
  a.m = value_of(wave_max(ordered(a.m)));
  if ((tid & 63) == 0) slots[0][tid >> 6] = a.m;
  __syncthreads();
  Joined row{largest<NW>(slots[0]), 0.f, 0.f};
  move_to(a, row.m, c);
  a.s = wave_sum(a.s);
  a.t = wave_sum(a.t);
  if ((tid & 63) == 0) {
    slots[1][tid >> 6] = a.s;
    slots[2][tid >> 6] = a.t;
  }
  __syncthreads();
  if (tid >= 64) return;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    row.s += slots[1][w];
    row.t += slots[2][w];
  }
  if (tid == 0) write_sums<T>(A, blockIdx.x, r, y, row);
  if constexpr (TOP) {
    Picker pick(list[0], A.top);
    pick_entries<T>(pick, maxima, l, first, last);
    write_picked<T>(A, blockIdx.x, r, pick, row);
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
  const float4* part = A.part + r * A.chunks;
  const float4 none = make_float4(-INFINITY, 0.f, 0.f, 0.f);
  const float4 own = lane < A.chunks ? part[lane] : none;   // more than 64 chunks are read a second time
  Sums a;
  a.m = own.x;
  for (int q = lane + 64; q < A.chunks; q += 64) a.m = fmaxf(a.m, part[q].x);
  a.m = value_of(wave_max(ordered(a.m)));
  for (int q = lane; q < A.chunks; q += 64) {   // about the row's maximum
    const float4 p = q == lane ? own : part[q];
    Sums b;
    b.at = p.x;
    b.s = p.y;
    b.t = p.z;
    move_to(b, a.m, c);
    a.s += b.s;
    a.t += b.t;
  }
  const Joined row{a.m, wave_sum(a.s), wave_sum(a.t)};
  if (lane == 0) write_row<T>(A, r, y, row);
  if constexpr (TOP) {
    const Key* keys = A.keys + r * A.chunks * A.top;
    const int n = A.chunks * A.top;
    Picker pick(lists[threadIdx.x >> 6], A.top);
    float best = -INFINITY;
    for (int i = lane; i < n; i += 64) best = fmaxf(best, value_of(keys[i]));
    pick.start(best);
    for (int base = 0; base < n; base += 64) {
      const Key key = base + lane < n ? keys[base + lane] : kNone;
      pick.push(value_of(key), place_of(key));
    }
    pick.settle();
    write_top(A, r, pick, row);
  }
}

// ---------------------------------------------------------------- backward
// A workgroup per chunk of a row.  Rows without a gradient are not read.  3000 x 32001 fp32, a tenth without one, 134 us
// for 730 MB, 5.4 TB/s.
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
    case 0:
      if (A.vocab <= 1024) hipLaunchKernelGGL((k_logp_held<T, 16 / T::W, TOP>), quads, dim3(256), 0, st, A);
      else hipLaunchKernelGGL((k_logp_held<T, 32 / T::W, TOP>), quads, dim3(256), 0, st, A);
      break;
    case 64: hipLaunchKernelGGL((k_logp_rows<T, 64, TOP>), each, dim3(64), 0, st, A); break;
    default: hipLaunchKernelGGL((k_logp_rows<T, 256, TOP>), each, dim3(256), 0, st, A);
  }
  if (A.chunks > 1) hipLaunchKernelGGL((k_logp_join<T, TOP>), quads, dim3(256), 0, st, A);
  return hipGetLastError();
}

}  // namespace logp

// A few long rows are cut, about 32 KB a part (us, 5 to 20 alternatives, whole and cut: 1 x 131072 bf16 21 and 15, 64 of
// them 22 and 18, 200 23 and 25; 16 x 50257 14 and 16); and rows beyond a workgroup's list of groups.
void plan_logp(LogpArgs& A, bool f32) {
  const int64_t rows = std::max(A.rows, 1), group = f32 ? 64 : 128, most = group * logp::kGroups;
  const int64_t bytes = int64_t(A.vocab) * (f32 ? 4 : 2);
  int64_t chunks = rows <= 128 && bytes > 200 * 1024 ? std::min<int64_t>(bytes / 32768, 64) : 1;
  chunks = std::max<int64_t>({chunks, 1, (A.vocab + most - 1) / most});
  A.chunk = int32_t(((A.vocab + chunks - 1) / chunks + group - 1) / group * group);
  A.chunks = (A.vocab + A.chunk - 1) / A.chunk;
}

// Threads of a row; 0: a wave holds it, four rows a workgroup (us, with alternatives: 20000 x 2000 fp32 held 40, by
// 64 threads 58, by 256 55).  One wave up to 24 KB a row, as each wave has its share of joins and of work on less than a
// whole step (10000 rows of bf16 by 64, 128 and 256 threads: 4099 29, 35, 51; 8000 45, 52, 66; 10000 53, 52, 60; 16384
// 70, 64, 67; 6000 x 6000 fp32 33 each).  Not more than 256 (4096 x 131072 bf16 by 256 152, by 1024 250; a few
// rows by 256 to 1024 alike).
int logp_threads(const LogpArgs& A, bool f32) {
  const int64_t bytes = int64_t(A.chunk) * (f32 ? 4 : 2);
  if (A.chunks == 1 && A.vocab <= 2048) return 0;
  return bytes <= logp::kWaveBytes ? 64 : 256;
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
