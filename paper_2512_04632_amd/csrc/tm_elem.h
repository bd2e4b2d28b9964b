// Element access shared by the streaming operators (layer norm, policy loss):
// rows of bf16 or fp32 read and written 16 bytes at a time at the element's own
// alignment (the global memory path takes 16-byte accesses at any), values in
// fp32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace tmk {
namespace elem {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef u32x4_t u32x4_a2 __attribute__((aligned(2)));   // at a bf16 element's alignment
typedef u32x4_t u32x4_a4 __attribute__((aligned(4)));

struct Bf16 {
  static constexpr int kBytes = 2, W = 8;   // W: elements of a 16-byte vector
  __device__ static u32x4_t load(const char* p) { return *reinterpret_cast<const u32x4_a2*>(p); }
  __device__ static void store(char* p, u32x4_t v) { *reinterpret_cast<u32x4_a2*>(p) = v; }
  __device__ static void unpack(u32x4_t q, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(q[i] << 16);
      v[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
    }
  }
  __device__ static u32x4_t pack(const float* v) {   // rounds to nearest even
    u32x4_t q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[2 * i]));
      const uint32_t hi = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[2 * i + 1]));
      q[i] = lo | hi << 16;
    }
    return q;
  }
  // element i of a vector that is zero there, from memory
  __device__ static void put1(u32x4_t& q, int i, const char* p) {
    q[i / 2] |= uint32_t(*reinterpret_cast<const uint16_t*>(p)) << (16 * (i % 2));
  }
  __device__ static float load1(const char* p) {
    return __uint_as_float(uint32_t(*reinterpret_cast<const uint16_t*>(p)) << 16);
  }
  __device__ static void store1(char* p, float v) {
    *reinterpret_cast<uint16_t*>(p) = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
  }
};

struct F32 {
  static constexpr int kBytes = 4, W = 4;
  __device__ static u32x4_t load(const char* p) { return *reinterpret_cast<const u32x4_a4*>(p); }
  __device__ static void store(char* p, u32x4_t v) { *reinterpret_cast<u32x4_a4*>(p) = v; }
  __device__ static void unpack(u32x4_t q, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(q[i]);
  }
  __device__ static u32x4_t pack(const float* v) {
    u32x4_t q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = __float_as_uint(v[i]);
    return q;
  }
  __device__ static void put1(u32x4_t& q, int i, const char* p) { q[i] = *reinterpret_cast<const uint32_t*>(p); }
  __device__ static float load1(const char* p) { return *reinterpret_cast<const float*>(p); }
  __device__ static void store1(char* p, float v) { *reinterpret_cast<float*>(p) = v; }
};

// Elements first .. first + W - 1 of a row of n (`fill` past its end).
template <class T>
__device__ inline void load_vec(const char* row, int first, int n, float fill, float* v) {
  if (first + T::W <= n) {
    T::unpack(T::load(row + int64_t(first) * T::kBytes), v);
  } else {
#pragma unroll
    for (int i = 0; i < T::W; ++i)
      v[i] = first + i < n ? T::load1(row + int64_t(first + i) * T::kBytes) : fill;
  }
}

// Elements first .. first + W - 1 of a row of n as stored, for a row that is read
// ahead: a load whose value nothing waits for.  What comes back past the row's
// end is for `settle` to put right when the row's turn comes.
//   TAIL = false  n is a multiple of W: a vector is whole or wholly past the end
//                 (then the row's last one is read again).
//   TAIL          a vector that would end past the row is read from the row's
//                 last W elements; rows of less than W are read one by one.
template <class T, bool TAIL>
__device__ inline u32x4_t load_ahead(const char* row, int first, int n) {
  if constexpr (!TAIL) return T::load(row + int64_t(min(first, n - T::W)) * T::kBytes);
  u32x4_t q = {0u, 0u, 0u, 0u};
  if (n >= T::W) {
    if (first < n) q = T::load(row + int64_t(min(first, n - T::W)) * T::kBytes);
    return q;
  }
#pragma unroll
  for (int i = 0; i < T::W; ++i)
    if (first + i < n) T::put1(q, i, row + int64_t(first + i) * T::kBytes);
  return q;
}

// The vector that load_ahead read, elements in their places and zeros past the end.
template <class T, bool TAIL>
__device__ inline u32x4_t settle(u32x4_t q, int first, int n) {
  if constexpr (!TAIL) {
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = first < n ? q[i] : 0u;
    return q;
  }
  const int by = first + T::W - n;   // elements past the end
  if (by <= 0 || n < T::W) return q;
  const int bits = min(by, T::W) * (8 * T::kBytes);   // down by this many of 128
  if (bits & 16) q = u32x4_t{q[0] >> 16 | q[1] << 16, q[1] >> 16 | q[2] << 16, q[2] >> 16 | q[3] << 16, q[3] >> 16};
  if (bits & 32) q = u32x4_t{q[1], q[2], q[3], 0u};
  if (bits & 64) q = u32x4_t{q[2], q[3], 0u, 0u};
  if (bits & 128) q = u32x4_t{0u, 0u, 0u, 0u};
  return q;
}

template <class T>
__device__ inline void store_vec(char* row, int first, int n, const float* v) {
  if (first + T::W <= n) {
    T::store(row + int64_t(first) * T::kBytes, T::pack(v));
  } else {
#pragma unroll
    for (int i = 0; i < T::W; ++i)
      if (first + i < n) T::store1(row + int64_t(first + i) * T::kBytes, v[i]);
  }
}

// Sum over the wave, in every lane: within rows of 16 lanes, then from row to
// row, with data-parallel moves (no trip through LDS); lane 63 holds the total.
__device__ inline float wave_sum(float v) {
  auto add = [&](auto ctrl, auto rows) {
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), decltype(ctrl)::value, decltype(rows)::value,
                                                     0xf, false));
  };
  using std::integral_constant;
  add(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});   // row_shr:1
  add(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});   // row_shr:2
  add(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});   // row_shr:4
  add(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});   // row_shr:8
  add(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // row_bcast:15
  add(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});   // row_bcast:31
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

}  // namespace elem
}  // namespace tmk
