// Operand fragments of the 16 x 16 matrix-core products, loads of rows of any
// alignment and length, and four-element stores, for bf16 and fp32 operands.
#pragma once

#include <type_traits>

#include "cci_device.hpp"

namespace cci {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// A device pointer out of a kernel's parameter struct, known to the compiler to point to global memory (such pointers
// are generic otherwise, and generic accesses also count as LDS operations).
template <typename T, typename V>
__device__ __forceinline__ T* global_ptr(V* p) {
  return (T*)(__attribute__((address_space(1))) T*)(p);
}

// The place of workgroup b of `grid` in an order in which those of one XCD
// (b % 8, as the dispatcher deals them out) follow each other.
__device__ __forceinline__ uint32_t xcd_order(uint32_t b, uint32_t grid) {
  const uint32_t x = b & 7u, rest = grid & 7u;
  return x * (grid >> 3) + (x < rest ? x : rest) + (b >> 3);
}

// Eight consecutive elements: a unit of a row, and an operand fragment's share of a lane.
template <typename T>
struct Unit {
  u32x4_t d[sizeof(T) / 2];
};

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// Two values as bf16, rounded to nearest even (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{lo, hi}), bf16x2_t));
}

// Element e of a unit, in fp32.
template <typename T>
__device__ __forceinline__ float elem(const Unit<T>& u, int e) {
  if constexpr (sizeof(T) == 2)
    return __uint_as_float(e & 1 ? u.d[0][e >> 1] & 0xffff0000u : u.d[0][e >> 1] << 16);
  else
    return __uint_as_float(u.d[e >> 2][e & 3]);
}

// A unit's eight entries in another order: what is entry e becomes entry e ^ m,
// m a lane's own.  The lanes of a wave write their entries one at a time; in
// the same order they would meet in few banks of the LDS.
struct Shuffle {
  uint32_t m, bytes, half;
};
__device__ __forceinline__ Shuffle make_shuffle(uint32_t m) {
  return Shuffle{m, 0x03020100u ^ (0x01010101u * (m & 3u)), 16u * (m & 1u)};
}
__device__ __forceinline__ void shuffle(const Shuffle& s, Unit<bf16_t>& v, u32x2_t& ix) {
  const bool s1 = (s.m & 2u) != 0, s2 = (s.m & 4u) != 0;
  u32x4_t a = v.d[0];
#pragma unroll
  for (int j = 0; j < 4; ++j) a[j] = __builtin_amdgcn_alignbit(a[j], a[j], s.half);
  const u32x4_t b = s1 ? u32x4_t{a[1], a[0], a[3], a[2]} : a;
  v.d[0] = s2 ? u32x4_t{b[2], b[3], b[0], b[1]} : b;
  const uint32_t lo = __builtin_amdgcn_perm(ix[0], ix[0], s.bytes), hi = __builtin_amdgcn_perm(ix[1], ix[1], s.bytes);
  ix = s2 ? u32x2_t{hi, lo} : u32x2_t{lo, hi};
}

// acc += A B over the 32 reduction elements of the wave's fragments: lane l holds elements 8 (l / 16) .. +7 of
// row (A) or column (B) l % 16, and rows 4 (l / 16) .. +3 of column l % 16 of acc.  fp32: MFMA e multiplies element
// e of each lane's eight, so the sum runs in another order over the same products.
__device__ __forceinline__ void mma(f32x4_t& acc, const Unit<bf16_t>& a, const Unit<bf16_t>& b) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a.d[0]),
                                                __builtin_bit_cast(bf16x8_t, b.d[0]), acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x4_t& acc, const Unit<float>& a, const Unit<float>& b) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.d[e >> 2][e & 3]), __uint_as_float(b.d[e >> 2][e & 3]),
                                               acc, 0, 0, 0);
}

// NE elements at p.  Rows need no alignment beyond their element's.
template <int NE, typename T, typename V>
__device__ __forceinline__ void load_full(V& v, const T* p) {
  static_assert(sizeof(V) == NE * sizeof(T));
  __builtin_memcpy(&v, p, sizeof(V));
}
// The same where only the first `left` exist and the others read as 0: one
// load per element, those past the row's end from its last element (which is
// p[left - 1], also for left <= 0), and no branch.
template <int NE, typename T, typename V>
__device__ __forceinline__ void load_tail(V& v, const T* p, int64_t left) {
  static_assert(sizeof(V) == NE * sizeof(T));
  T e[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) e[i] = p[i < left ? i : left - 1];
#pragma unroll
  for (int i = 0; i < NE; ++i) e[i] = i < left ? e[i] : T{};
  __builtin_memcpy(&v, e, sizeof(V));
}
// Either, by `whole`, which is uniform over a wave: a branch that no lane of a
// whole chunk pays for.
template <int NE, typename T, typename V>
__device__ __forceinline__ void load_part(V& v, const T* p, int64_t left, bool whole) {
  if (whole)
    load_full<NE>(v, p);
  else
    load_tail<NE>(v, p, left);
}
// By lane: all of them, a part, or none (left <= 0: nothing is read).
template <int NE, typename T, typename V>
__device__ __forceinline__ void load_elems(V& v, const T* p, int64_t left) {
  if (left >= NE) {
    load_full<NE>(v, p);
  } else {
    v = V{};
    if (left > 0) load_tail<NE>(v, p, left);
  }
}

template <typename YT>
__device__ __forceinline__ void store4(YT* p, const float (&v)[4], int64_t left, bool vec) {
  if (left <= 0) return;
  if (vec && left >= 4) {
    if constexpr (std::is_same<YT, float>::value) {
      *reinterpret_cast<f32x4_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
    } else {
      *reinterpret_cast<u32x2_t*>(p) = u32x2_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    }
    return;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (r < left) io<YT>::store(p, r, v[r]);
}

}  // namespace cci
