// Expert products through registers: operands of any alignment and stride,
// fp32, and groups of a few rows.  Tiles of TM x TN by four waves in a WM x WN
// grid.
//
// A stage is 128 bytes of the summed index (64 bf16 or 32 fp32 values) of both
// operands.  Its 16-byte chunks go global -> registers -> LDS, at any address
// (the memory path takes 16-byte loads at an element's alignment).  Rows and
// columns past the tile's end are read from the last row or the first chunk
// that is there and dropped when the tile is stored; a stage that reaches the
// summed index's end, or the last seven rows of a matrix (where 16 bytes could
// end outside), is loaded with a check of every chunk, and what is past the
// summed index comes out as zeros.  While a stage is multiplied from one LDS
// buffer, the next D wait in registers, and the first of them is written to the
// other buffer afterwards: one barrier a stage.
//
// Layouts in LDS: an operand whose summed index is contiguous as rows of 128
// bytes, chunks XORed by (row / 2) % 8; a row-major one as rows of the tile's
// columns, for bf16 32-byte chunks XORed by swz_y and read with the transposing
// instruction, for fp32 64-byte blocks XORed by (row / 4) % 4 and read 4 bytes
// a lane.  None of these reads has bank conflicts.  fp32 multiplies with
// v_mfma_f32_16x16x4_f32, four at a time: lane group g of step j takes summed
// value 16 s + 4 g + j of both operands, so that a contiguous operand is read
// 16 bytes a lane.
//
// fp32 on the 128 tile goes as three bf16 parts, x = hi + mid + lo, each rounded to
// nearest from what the ones before it leave: 8 bits each, all 24 of x together.
// A product is hi hi + hi mid + mid hi + mid mid + hi lo + lo hi in one fp32 accumulator,
// small terms first; mid lo, lo mid and lo lo, at most 2^-23 of it, are left out.  Six
// bf16 instructions take 96 clocks where the eight of fp32 for the same 32 values
// take 256 (16384 rows over 8 experts of 2048 x 2048: 0.75-0.80 ms, 172-184 TFLOP/s, against
// 1.03 ms of fp32 instructions).  A tile with a value that three parts do not hold exactly (NaN,
// infinities, the few that round to one, those below about 2^-110 whose last bits lie below
// the smallest bf16) or with a result that is not finite is done again with fp32
// instructions (where every tile is: 1.74 ms).  On the smaller tiles the splitting costs what the
// instructions save (2048 rows of 1024 x 1024: 45 us, 40 without; 80 rows over 5 experts
// of 7960 x 1970: 111 against 95), and fp32 multiplies as it is.
//
// Rows that only fill a tile cost as much as real ones: groups of a few rows take
// tiles of 16 or 32 rows, which are bound by the reading of the matrices: 24 rows over
// 8 experts of 768 x 2048 bf16 8.0 us a call, 3.1 TB/s (9.6 where the matrices of thirty calls
// in turn come from HBM; 8.5 in the kernel under the tracer); 192 rows over 16 of
// 2048 x 4096 64 us, 4.2 TB/s.  The larger tiles are bound by their fp32 instructions (3001 rows
// over 5 of 515 x 777 fp32: 33.8 us, 71 TFLOP/s of 153) or, for bf16 of odd strides, by
// the way through the registers (2048 rows of 2049 x 2048: 36 us, 0.48 PFLOP/s).
#include "tm_elem.h"
#include "tm_expert.h"
#include "tm_tile.h"

namespace tmk {
namespace expert {

using namespace tile;
using elem::Bf16;
using elem::F32;
using elem::u32x4_t;

constexpr int kStageBytes = 128;   // of the summed index, per row or column of a tile

// One operand of a tile.  KC: its rows are the tile's, the summed index runs
// along them; otherwise (row-major) its rows are the summed index.
struct Source {
  const char* p;   // first element of the tile's part
  int64_t ld;
  int limit;       // the tile's rows (row-major: columns) that are there
  int left;        // rows from p's to the matrix's last
};

// The 16 bytes at p, of which the first n elements are wanted and the others
// come out as zeros.  `inside`: all 16 bytes belong to the matrix.
template <class T>
__device__ inline u32x4_t load_chunk(const char* p, int n, bool inside) {
  u32x4_t q = {0u, 0u, 0u, 0u};
  if (n <= 0) return q;
  if (n >= T::W || inside) {
    q = T::load(p);
    if (n < T::W) {
      const int bytes = n * T::kBytes;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        q[j] &= bytes >= 4 * j + 4 ? 0xffffffffu : bytes > 4 * j ? 0xffffu : 0u;
    }
  } else {
#pragma unroll
    for (int i = 0; i < T::W; ++i)
      if (i < n) T::put1(q, i, p + i * T::kBytes);
  }
  return q;
}

// One operand's way into LDS.  TS: the tile's rows (row-major: columns).
template <class T, int TS, bool KC>
struct Stager {
  static constexpr int BK = kStageBytes / T::kBytes, CHUNKS = TS * kStageBytes / 16, Q = (CHUNKS + 255) / 256;
  static constexpr int PER = KC ? 8 : TS * T::kBytes / 16;   // chunks of a stored row
  const char* p[Q];
  int64_t step;
  int limit, left, K, whole;   // whole: values of the summed index that need no check

  __device__ static int id(int i) { return i * 256 + int(threadIdx.x); }
  __device__ static int row(int i) { return id(i) / PER; }
  __device__ static int chunk(int i) { return id(i) % PER; }
  __device__ static bool mine(int i) { return CHUNKS % 256 == 0 || id(i) < CHUNKS; }

  __device__ void start(const Source& s, int summed) {
    limit = s.limit;
    left = s.left;
    K = summed;
    whole = KC ? K : min(K, left - 7);
    step = KC ? kStageBytes : BK * s.ld * T::kBytes;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      const int64_t r = KC ? min(row(i), limit - 1) : row(i);
      const int c = KC || chunk(i) * T::W < limit ? chunk(i) : 0;
      p[i] = s.p + (r * s.ld + c * T::W) * T::kBytes;
    }
  }
  // Stage at k0, in steps of BK.  FAST: known to need no check (the main loops'
  // way: with the checked loads' branches beside them, every wait for a stage that
  // was loaded long ago would be a wait for all loads under way).
  template <bool FAST>
  __device__ void load(int k0, u32x4_t (&v)[Q]) {
    if (FAST || k0 + BK <= whole) {
#pragma unroll
      for (int i = 0; i < Q; ++i)
        if (mine(i)) v[i] = T::load(p[i]);
    } else {
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        if (!mine(i)) continue;
        // seven rows before the last one, 16 bytes from an element of a row end within the matrix
        if constexpr (KC)
          v[i] = load_chunk<T>(p[i], K - k0 - chunk(i) * T::W, min(row(i), limit - 1) + 7 < left);
        else
          v[i] = load_chunk<T>(p[i], k0 + row(i) < K ? limit - chunk(i) * T::W : 0, k0 + row(i) + 7 < left);
      }
    }
#pragma unroll
    for (int i = 0; i < Q; ++i) p[i] += step;
  }
  __device__ void store(char* lds, const u32x4_t (&v)[Q]) const {
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      if (!mine(i)) continue;
      const int r = row(i), c = chunk(i);
      int at;
      if constexpr (KC) at = r * kStageBytes + 16 * (c ^ ((r / 2) % 8));
      else if constexpr (T::kBytes == 2) at = r * 2 * TS + 32 * ((c >> 1) ^ swz_y<TS>(r)) + 16 * (c & 1);
      else at = r * 4 * TS + 64 * ((c >> 2) ^ ((r >> 2) & 3)) + 16 * (c & 3);
      *reinterpret_cast<u32x4_t*>(lds + at) = v[i];
    }
  }
};

// Operands of slice s of a stage, rows or columns 16 (w F + f) + lane % 16 of a
// tile side of TS (g: lane / 16).  bf16: 8 values 32 s + 8 g .. + 7.
template <int TS, bool KC, int F>
__device__ inline void load_slice(Bf16, uint4 (&v)[F], const char* st, int s, int w) {
  const int lr = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  if constexpr (KC) {
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const int r = (w * F + f) * 16 + lr;
      v[f] = *reinterpret_cast<const uint4*>(st + r * kStageBytes + 16 * ((4 * s + g) ^ ((r / 2) % 8)));
    }
  } else {
    const int rl = 8 * g + (lr >> 2);
    const char* base = st + (32 * s + rl) * (2 * TS) + 8 * (lr & 3);
    const int chunk = (w * F) ^ swz_y<TS>(rl);
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const char* p = base + 32 * (chunk ^ f);
      s16x4_t h[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
        h[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4_t*)(lds_addr(p + u * 4 * (2 * TS))));
      v[f] = __builtin_bit_cast(uint4, h);
    }
  }
}
// fp32: 4 values 16 s + 4 g .. + 3.
template <int TS, bool KC, int F>
__device__ inline void load_slice(F32, f32x4_t (&v)[F], const char* st, int s, int w) {
  const int lr = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int f = 0; f < F; ++f) {
    if constexpr (KC) {
      const int r = (w * F + f) * 16 + lr;
      v[f] = *reinterpret_cast<const f32x4_t*>(st + r * kStageBytes + 16 * ((4 * s + g) ^ ((r / 2) % 8)));
    } else {
      const char* p = st + (16 * s + 4 * g) * 4 * TS + 64 * ((w * F + f) ^ g) + 4 * lr;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[f][j] = *reinterpret_cast<const float*>(p + j * 4 * TS);
    }
  }
}

// The operands are fed the other way round: each lane holds four consecutive columns of a row.
template <int FM, int FN>
__device__ inline void mma_slice(Bf16, f32x4_t (&acc)[FM][FN], const uint4 (&a)[FM], const uint4 (&b)[FN]) {
#pragma unroll
  for (int fm = 0; fm < FM; ++fm)
#pragma unroll
    for (int fn = 0; fn < FN; ++fn)
      acc[fm][fn] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, b[fn]),
                                                            __builtin_bit_cast(bf16x8_t, a[fm]), acc[fm][fn], 0, 0, 0);
}
template <int FM, int FN>
__device__ inline void mma_slice(F32, f32x4_t (&acc)[FM][FN], const f32x4_t (&a)[FM], const f32x4_t (&b)[FN]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int fm = 0; fm < FM; ++fm)
#pragma unroll
      for (int fn = 0; fn < FN; ++fn)
        acc[fm][fn] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[fn][j], a[fm][j], acc[fm][fn], 0, 0, 0);
}

template <class T>
struct SliceOf;
template <>
struct SliceOf<Bf16> { typedef uint4 V; };
template <>
struct SliceOf<F32> { typedef f32x4_t V; };

// A tile's shape: FM x FN blocks of 16 x 16 a wave; D stages wait in registers
// (a load takes longer than a stage of a small tile).
template <int TM_, int TN_, int WM_, int D_>
struct Shape {
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = 4 / WM_, D = D_;
  static constexpr int FM = TM / 16 / WM, FN = TN / 16 / WN;
  static constexpr int A_BYTES = TM * kStageBytes, STAGE = (TM + TN) * kStageBytes;
  static constexpr int ROW = 2 * TN + 16;   // of the bf16 output stage
  static constexpr int LDS = 2 * STAGE > TM * ROW ? 2 * STAGE : TM * ROW;
  static constexpr bool kParts = TM >= 128;   // fp32 as three bf16 parts
  static_assert(3 * 64 * (TM + TN) <= 2 * STAGE, "a stage of their planes takes less than two stages");
  static constexpr int kWaves = TM >= 128 ? 2 : 3;   // per SIMD, for the register allocation
  static_assert(FM >= 1 && FN >= 1, "a block for every wave");
};

// Row and first of the four columns that a lane holds of block (fm, fn).
template <class S>
__device__ inline int staged_row(int fm) {
  return (int(threadIdx.x >> 6) / S::WN * S::FM + fm) * 16 + int(threadIdx.x & 15);
}
template <class S>
__device__ inline int staged_col(int fn) {
  return (int(threadIdx.x >> 6) % S::WN * S::FN + fn) * 16 + 4 * (int(threadIdx.x & 63) >> 4);
}

// begin(fast), then step(kt, kt % D, fast) for each stage kt < nk; fast (a constant)
// while the stages that they load, at most D for begin and kt + D for a step, are
// among the first `unchecked` (steps that load one further say one less).  The
// fast steps follow a beginning of their own: with the other's branches in front of
// them the compiler would wait for every load under way before each use.
template <int D, class FB, class F>
__device__ inline void staged_loop(int nk, int unchecked, FB begin, F step) {
  int kt = 0;
  if (unchecked >= D) {
    begin(std::true_type{});
    for (; kt + 2 * D <= unchecked; kt += D)
#pragma unroll
      for (int u = 0; u < D; ++u) step(kt + u, u, std::true_type{});
  } else {
    begin(std::false_type{});
  }
  for (; kt < nk; kt += D)
#pragma unroll
    for (int u = 0; u < D; ++u)
      if (kt + u < nk) step(kt + u, u, std::false_type{});
}

// acc = the tile's product over K values.
template <class T, class S, bool AKC, bool BKC>
__device__ inline void product_staged(f32x4_t (&acc)[S::FM][S::FN], char* smem, const Source& a, const Source& b, int K) {
  using SA = Stager<T, S::TM, AKC>;
  using SB = Stager<T, S::TN, BKC>;
  constexpr int BK = SA::BK, D = S::D;
  const int wave = threadIdx.x >> 6, wm = wave / S::WN, wn = wave % S::WN;
#pragma unroll
  for (int i = 0; i < S::FM; ++i)
#pragma unroll
    for (int j = 0; j < S::FN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (K <= 0) return;
  SA sa;
  SB sb;
  u32x4_t va[D][SA::Q], vb[D][SB::Q];
  sa.start(a, K);
  sb.start(b, K);
  const int nk = (K + BK - 1) / BK;
  auto begin = [&](auto fast) __attribute__((always_inline)) {
    constexpr bool FAST = decltype(fast)::value;
    sa.template load<FAST>(0, va[0]);
    sb.template load<FAST>(0, vb[0]);
    sa.store(smem, va[0]);
    sb.store(smem + S::A_BYTES, vb[0]);
#pragma unroll
    for (int u = 0; u < D; ++u)
      if (FAST || u + 1 < nk) {
        sa.template load<FAST>((u + 1) * BK, va[u]);
        sb.template load<FAST>((u + 1) * BK, vb[u]);
      }
    __syncthreads();
  };
  auto step = [&](int kt, int u, auto fast) __attribute__((always_inline)) {
    constexpr bool FAST = decltype(fast)::value;
    const char* st = smem + (kt & 1) * S::STAGE;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      typename SliceOf<T>::V fa[S::FM], fb[S::FN];
      load_slice<S::TM, AKC, S::FM>(T{}, fa, st, s, wm);
      load_slice<S::TN, BKC, S::FN>(T{}, fb, st + S::A_BYTES, s, wn);
      mma_slice<S::FM, S::FN>(T{}, acc, fa, fb);
    }
    if (FAST || kt + 1 < nk) {
      char* nx = smem + ((kt + 1) & 1) * S::STAGE;   // last read before the previous barrier
      sa.store(nx, va[u]);
      sb.store(nx + S::A_BYTES, vb[u]);
      if (FAST || kt + 1 + D < nk) {
        sa.template load<FAST>((kt + 1 + D) * BK, va[u]);
        sb.template load<FAST>((kt + 1 + D) * BK, vb[u]);
      }
    }
    __syncthreads();
  };
  staged_loop<D>(nk, min(sa.whole, sb.whole) / BK - 1, begin, step);
}

// The three parts of four values, each as four bf16 (hi first).  The third is what the
// others leave, `rest` its bits: where the lower 16 of them are not zero, it has bits below
// the smallest bf16 (2^-133; values from about 2^-110 down) and is no bf16 itself.  An
// infinity, a NaN or a value that rounds past the largest bf16 has a part that is not finite.
__device__ inline void split3(u32x4_t q, uint2 (&part)[3], uint32_t (&rest)[4]) {
  float x[4];
  F32::unpack(q, x);
#pragma unroll
  for (int p = 0; p < 3; ++p) {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[i] = f2bf(x[i]);
      if (p < 2) x[i] -= __uint_as_float(h[i] << 16);   // exact
    }
    part[p] = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) rest[i] = __float_as_uint(x[i]);
}

// A stage of 32 fp32 values as three planes in LDS, TS * 64 bytes each: a
// contiguous operand as rows of 64 bytes, 16-byte chunks XORed by (row / 4) % 4;
// a row-major one as rows of the tile's columns, as for bf16.
template <int TS, bool KC>
struct Planes {
  using St = Stager<F32, TS, KC>;
  static_assert(TS * kStageBytes % 4096 == 0 && 256 % St::PER == 0, "a chunk for every thread, the same of every row");
  uint32_t low[2] = {0u, 0u};   // lower bits of the third parts seen: of columns 0 and 1, 2 and 3 of the thread's chunk

  __device__ void store(char* lds, const u32x4_t (&v)[St::Q]) {
#pragma unroll
    for (int i = 0; i < St::Q; ++i) {
      const int r = St::row(i), c = St::chunk(i);
      const int at = KC ? r * 64 + 16 * ((c >> 1) ^ ((r / 4) % 4)) + 8 * (c & 1)
                        : r * 2 * TS + 32 * ((c >> 2) ^ swz_y<TS>(r)) + 8 * (c & 3);
      uint2 part[3];
      uint32_t x[4];
      split3(v[i], part, x);
      if constexpr (KC) {
        low[0] |= x[0] | x[1] | x[2] | x[3];
      } else {
        low[0] |= __builtin_amdgcn_perm(x[1], x[0], 0x05040100u);
        low[1] |= __builtin_amdgcn_perm(x[3], x[2], 0x05040100u);
      }
#pragma unroll
      for (int p = 0; p < 3; ++p) *reinterpret_cast<uint2*>(lds + p * TS * 64 + at) = part[p];
    }
  }
  // Whether a value lost bits.  What was read beside a row-major operand's last column
  // (`limit` are there) is not part of it, and must not decide how the tile is done.
  __device__ bool lost(int limit) const {
    if constexpr (KC) return (low[0] & 0xffffu) != 0u;
    const int n = limit - 4 * St::chunk(0);
    return ((low[0] & 0xffffu) != 0u && n > 0) || ((low[0] >> 16) != 0u && n > 1) ||
           ((low[1] & 0xffffu) != 0u && n > 2) || ((low[1] >> 16) != 0u && n > 3);
  }
};

// One plane's operands: 8 values 8 g .. + 7 of row or column 16 (w F + f) + lane % 16.
template <int TS, bool KC, int F>
__device__ inline void load_plane(uint4 (&v)[F], const char* st, int w) {
  if constexpr (KC) {
    const int lr = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const int r = (w * F + f) * 16 + lr;
      v[f] = *reinterpret_cast<const uint4*>(st + r * 64 + 16 * (g ^ ((r / 4) % 4)));
    }
  } else {
    load_slice<TS, false, F>(Bf16{}, v, st, 0, w);
  }
}

// fp32 as three parts, in one LDS buffer with two barriers a stage, so that two
// workgroups share a compute unit.  False if a value has no parts: its third one has
// lost bits, or a result is not finite (a part was not, or the product of two high parts,
// each up to 2^-8 above its value, passed the largest fp32 where that of the values does
// not).
template <class S, bool AKC, bool BKC>
__device__ inline bool product_parts(f32x4_t (&acc)[S::FM][S::FN], char* smem, const Source& a, const Source& b, int K) {
  using SA = Stager<F32, S::TM, AKC>;
  using SB = Stager<F32, S::TN, BKC>;
  constexpr int BK = SA::BK, D = S::D, PA = S::TM * 64, PB = S::TN * 64;
  const int wave = threadIdx.x >> 6, wm = wave / S::WN, wn = wave % S::WN;
#pragma unroll
  for (int i = 0; i < S::FM; ++i)
#pragma unroll
    for (int j = 0; j < S::FN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (K <= 0) return true;
  SA sa;
  SB sb;
  u32x4_t va[D][SA::Q], vb[D][SB::Q];
  sa.start(a, K);
  sb.start(b, K);
  const int nk = (K + BK - 1) / BK;
  Planes<S::TM, AKC> planes_a;
  Planes<S::TN, BKC> planes_b;
  auto store = [&](char* lds, const u32x4_t (&qa)[SA::Q], const u32x4_t (&qb)[SB::Q]) __attribute__((always_inline)) {
    planes_a.store(lds, qa);
    planes_b.store(lds + 3 * PA, qb);
  };
  auto multiply = [&](const char* lds) __attribute__((always_inline)) {
    uint4 fb[3][S::FN];
#pragma unroll
    for (int p = 0; p < 3; ++p) load_plane<S::TN, BKC, S::FN>(fb[p], lds + 3 * PA + p * PB, wn);
#pragma unroll
    for (int p = 2; p >= 0; --p) {   // a's parts, small ones first, each with those of b that count
      uint4 fa[S::FM];
      load_plane<S::TM, AKC, S::FM>(fa, lds + p * PA, wm);
#pragma unroll
      for (int q = 2 - p; q >= 0; --q) mma_slice<S::FM, S::FN>(Bf16{}, acc, fa, fb[q]);
    }
  };
  const int unchecked = min(sa.whole, sb.whole) / BK;
  auto begin = [&](auto fast) __attribute__((always_inline)) {
    constexpr bool FAST = decltype(fast)::value;
#pragma unroll
    for (int u = 0; u < D; ++u)
      if (FAST || u < nk) {
        sa.template load<FAST>(u * BK, va[u]);
        sb.template load<FAST>(u * BK, vb[u]);
      }
  };
  staged_loop<D>(nk, unchecked, begin, [&](int kt, int u, auto fast) __attribute__((always_inline)) {
    constexpr bool FAST = decltype(fast)::value;
    if (kt > 0) __syncthreads();   // the stage before has been read
    store(smem, va[u], vb[u]);
    if (FAST || kt + D < nk) {
      sa.template load<FAST>((kt + D) * BK, va[u]);
      sb.template load<FAST>((kt + D) * BK, vb[u]);
    }
    __syncthreads();
    multiply(smem);
  });
  bool bad = planes_a.lost(a.limit) || planes_b.lost(b.limit);
#pragma unroll
  for (int i = 0; i < S::FM; ++i)
#pragma unroll
    for (int j = 0; j < S::FN; ++j)
#pragma unroll
      for (int u = 0; u < 4; ++u)   // of contiguous operands every row is one that is there
        bad |= (AKC || staged_row<S>(i) < a.limit) && (BKC || staged_col<S>(j) + u < b.limit) && !(fabsf(acc[i][j][u]) < INFINITY);
  return !__syncthreads_or(bad);
}

// bf16 through LDS (free after the product's last barrier): 16 bytes a lane along the rows.
template <class S>
__device__ inline void store_tile(Bf16, const f32x4_t (&acc)[S::FM][S::FN], char* smem, char* out, int64_t ld, int rows,
                                  int cols) {
#pragma unroll
  for (int fm = 0; fm < S::FM; ++fm)
#pragma unroll
    for (int fn = 0; fn < S::FN; ++fn) {
      uint32_t o[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) o[u] = f2bf(acc[fm][fn][u]);
      *reinterpret_cast<uint2*>(smem + staged_row<S>(fm) * S::ROW + staged_col<S>(fn) * 2) =
          make_uint2(o[0] | o[1] << 16, o[2] | o[3] << 16);
    }
  __syncthreads();
  constexpr int LPR = S::TN / 8;   // lanes per row
  const int c = int(threadIdx.x % LPR) * 8;
  for (int r = threadIdx.x / LPR; r < rows; r += 256 / LPR) {
    const char* from = smem + r * S::ROW + c * 2;
    char* to = out + (r * ld + c) * 2;
    if (c + 8 <= cols) {
      Bf16::store(to, *reinterpret_cast<const u32x4_t*>(from));
    } else {
      for (int i = 0; i < cols - c; ++i)
        reinterpret_cast<uint16_t*>(to)[i] = reinterpret_cast<const uint16_t*>(from)[i];
    }
  }
}

// add: to what this thread stored there before.
template <class S>
__device__ inline void store_tile(F32, const f32x4_t (&acc)[S::FM][S::FN], char*, char* out, int64_t ld, int rows, int cols,
                                  bool add = false) {
#pragma unroll
  for (int fm = 0; fm < S::FM; ++fm) {
    const int r = staged_row<S>(fm);
    if (r >= rows) continue;
#pragma unroll
    for (int fn = 0; fn < S::FN; ++fn) {
      float v[4] = {acc[fm][fn][0], acc[fm][fn][1], acc[fm][fn][2], acc[fm][fn][3]};
      if (add) {
        float before[4];
        elem::load_vec<F32>(out + r * ld * 4, staged_col<S>(fn), cols, 0.f, before);
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] += before[u];
      }
      elem::store_vec<F32>(out + r * ld * 4, staged_col<S>(fn), cols, v);
    }
  }
}

// `s` from value `at` of the summed index on.
template <class T, bool KC>
__device__ inline Source from(const Source& s, int at) {
  return Source{s.p + (KC ? int64_t(at) : at * s.ld) * T::kBytes, s.ld, s.limit, KC ? s.left : s.left - at};
}

// The product in the type's way, and its result to `out`.  RUNS: sums may be longer than
// kLongest; those of fp32 instructions are then taken in runs of it, each added to what
// the ones before left in `out` (16 KB of a 64 tile for 1.4 MB of operands).
template <class T, class TO, class S, bool AKC, bool BKC, bool RUNS>
__device__ inline void product_tile(char* smem, const Source& a, const Source& b, int K, char* out, int64_t ld, int rows,
                                    int cols) {
  f32x4_t acc[S::FM][S::FN];
  if constexpr (T::kBytes == 4 && S::kParts) {
    if (product_parts<S, AKC, BKC>(acc, smem, a, b, K)) {
      store_tile<S>(TO{}, acc, smem, out, ld, rows, cols);
      return;
    }
  }
  if constexpr (T::kBytes == 4 && RUNS) {
    static_assert(kLongest % (kStageBytes / 4) == 0, "runs of whole stages");
    if (K > int(kLongest)) {
      for (int at = 0; at < K; at += int(kLongest)) {
        // a zero that the compiler does not know: addresses are formed anew in every run, and
        // do not take registers beside the product's
        int64_t zero = 0;
        asm volatile("" : "+s"(zero));
        const Source ra{a.p + zero, a.ld + zero, a.limit, a.left}, rb{b.p + zero, b.ld + zero, b.limit, b.left};
        product_staged<T, S, AKC, BKC>(acc, smem, from<T, AKC>(ra, at), from<T, BKC>(rb, at), min(K - at, int(kLongest)));
        asm volatile("" : "+s"(zero));
        store_tile<S>(TO{}, acc, smem, out + zero, ld + zero, rows, cols, at > 0);
      }
      return;
    }
  }
  product_staged<T, S, AKC, BKC>(acc, smem, a, b, K);
  store_tile<S>(TO{}, acc, smem, out, ld, rows, cols);
}

// The rows' product.  TO: type of the result, F32 for slices of the summed index.
template <class T, class TO, class S, bool TRANS>
__global__ __launch_bounds__(256, S::kWaves) void k_rows_staged(const ExpertArgs A, int row_tiles) {
  __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
  const int nJ = (A.n + S::TN - 1) / S::TN;
  const Slice sl = slice_of(A, int(blockIdx.x), int(gridDim.x));
  const Place at = place_of(sl.id, row_tiles, nJ);
  Group g;
  if (!find_tile(A, S::TM, at.I, g)) return;
  const int c0 = at.J * S::TN, rows = g.last - g.first, cols = min(S::TN, A.n - c0);
  int k0 = 0, K = 0;
  if (g.e < A.experts) sl.range(A.k, kStageBytes / T::kBytes, k0, K);
  const Source a{A.a + (g.first * A.lda + k0) * T::kBytes, A.lda, rows, A.rows - g.first};
  const char* w = A.b + (K > 0 ? g.e * A.stride_b : 0) * T::kBytes;
  const Source b = TRANS ? Source{w + (c0 * A.ldb + k0) * T::kBytes, A.ldb, cols, A.n - c0}
                         : Source{w + (k0 * A.ldb + c0) * T::kBytes, A.ldb, cols, A.k - k0};
  // the smaller tiles' sums are cut into slices (plan_expert_matmul)
  product_tile<T, TO, S, true, TRANS, S::kParts>(smem, a, b, K, A.out + (sl.z * A.slice_out + g.first * A.ldo + c0) * TO::kBytes,
                                                 A.ldo, rows, cols);
}

// The weight gradient: 2048 rows over 4 experts of 2048 x 768, bf16 of odd strides, 21 us,
// 0.31 PFLOP/s.  The fp32 64 tile's registers are held to what its five workgroups a compute unit
// (32 KB of LDS each) leave: the runs of long fp32 sums would take more from every call (4096
// rows over 16 of 512 x 512, fp32: 27.2 us, 32.1 without the bound; 27080 rows, 10295 of them one
// expert's, over 63 of 256 x 192: 30.3 evenly, 211 unevenly, 190 in one run).
template <class T, class TO, class S>
__global__ __launch_bounds__(256, T::kBytes == 4 && S::TM == 64 ? 5 : S::kWaves) void k_wgrad_staged(const ExpertArgs A) {
  __shared__ __attribute__((aligned(1024))) char smem[S::LDS];
  const int nI = (A.k + S::TM - 1) / S::TM, nJ = (A.n + S::TN - 1) / S::TN;
  GradTile t;
  if (!grad_tile(A, int(blockIdx.x), int(gridDim.x), nI * nJ, t)) return;
  const Place at = place_of(t.tile, nI, nJ);
  const int r0 = at.I * S::TM, c0 = at.J * S::TN, rows = min(S::TM, A.k - r0), cols = min(S::TN, A.n - c0);
  const Source a{A.a + (t.first * A.lda + r0) * T::kBytes, A.lda, rows, A.rows - t.first};
  const Source b{A.b + (t.first * A.ldb + c0) * T::kBytes, A.ldb, cols, A.rows - t.first};
  product_tile<T, TO, S, false, false, true>(smem, a, b, t.K, A.out + (t.out * A.stride_b + r0 * A.ldo + c0) * TO::kBytes,
                                             A.ldo, rows, cols);
}

template <class T, class TO, class S>
hipError_t rows_staged(const ExpertArgs& A, bool transposed, hipStream_t st) {
  const uint64_t tiles = row_tiles(A, S::TM);
  const uint64_t blocks = tiles * col_tiles(A, S::TN) * uint64_t(A.slices);
  if (!launchable(blocks, 256)) return hipErrorInvalidConfiguration;
  const dim3 grid{uint32_t(blocks)};
  if (transposed) hipLaunchKernelGGL((k_rows_staged<T, TO, S, true>), grid, dim3(256), 0, st, A, int(tiles));
  else hipLaunchKernelGGL((k_rows_staged<T, TO, S, false>), grid, dim3(256), 0, st, A, int(tiles));
  return hipGetLastError();
}

template <class T, class TO, class S>
hipError_t wgrad_staged(const ExpertArgs& A, hipStream_t st) {
  const uint64_t blocks = wgrad_blocks(A, S::TM, S::TN);
  if (!launchable(blocks, 256)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((k_wgrad_staged<T, TO, S>), dim3(uint32_t(blocks)), dim3(256), 0, st, A);
  return hipGetLastError();
}

using Tile16 = Shape<16, 64, 1, 3>;
using Tile32 = Shape<32, 64, 2, 3>;
using Tile64 = Shape<64, 64, 2, 2>;
using Tile128 = Shape<128, 128, 2, 1>;

template <class T, class TO>
hipError_t rows_tile(const ExpertArgs& A, int tile, bool transposed, hipStream_t st) {
  switch (tile) {
    case 16: return rows_staged<T, TO, Tile16>(A, transposed, st);
    case 32: return rows_staged<T, TO, Tile32>(A, transposed, st);
    case 64: return rows_staged<T, TO, Tile64>(A, transposed, st);
  }
  return rows_staged<T, TO, Tile128>(A, transposed, st);
}

template <class T, class TO>
hipError_t wgrad_tile(const ExpertArgs& A, int tile, hipStream_t st) {
  return tile == 64 ? wgrad_staged<T, TO, Tile64>(A, st) : wgrad_staged<T, TO, Tile128>(A, st);
}

}  // namespace expert

using elem::Bf16;
using elem::F32;

hipError_t launch_rows_staged(const ExpertArgs& A, const ExpertPlan& P, bool f32, bool transposed, hipStream_t st) {
  if (f32) return expert::rows_tile<F32, F32>(A, P.tile, transposed, st);
  return P.slices > 1 ? expert::rows_tile<Bf16, F32>(A, P.tile, transposed, st)
                      : expert::rows_tile<Bf16, Bf16>(A, P.tile, transposed, st);
}

hipError_t launch_wgrad_staged(const ExpertArgs& A, const ExpertPlan& P, bool f32, bool out_f32, hipStream_t st) {
  if (f32) return expert::wgrad_tile<F32, F32>(A, P.tile, st);
  return out_f32 || P.chunk > 0 ? expert::wgrad_tile<Bf16, F32>(A, P.tile, st)
                                 : expert::wgrad_tile<Bf16, Bf16>(A, P.tile, st);
}

}  // namespace tmk
