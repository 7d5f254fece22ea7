// Eight consecutive elements of a row as float32, and back with one rounding
// (to nearest even, NaN kept): the unit of the element-wise layer operators, 16
// bytes of bf16 or two 16-byte pieces of float32.
#pragma once

#include "common.h"

namespace pspo {

struct Bf16 {
  static constexpr int kBytes = 2;
};
struct F32 {
  static constexpr int kBytes = 4;
};

struct Vec8 {
  float v[8];
};

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

template <class T>
struct Raw8;   // the eight elements as they lie in memory
template <>
struct Raw8<Bf16> {
  u32x4 a;
};
template <>
struct Raw8<F32> {
  u32x4 a, b;
};

// p: the row's bytes; i: index of the group of eight in the row; kPast: past the caches.
template <class T, bool kPast = false>
__device__ __forceinline__ Raw8<T> load8(const unsigned char* p, int64_t i) {
  Raw8<T> r;
  const u32x4* q = reinterpret_cast<const u32x4*>(p + i * (8 * T::kBytes));
  if constexpr (kPast) {
    r.a = __builtin_nontemporal_load(q);
    if constexpr (T::kBytes == 4) r.b = __builtin_nontemporal_load(q + 1);
  } else {
    r.a = q[0];
    if constexpr (T::kBytes == 4) r.b = q[1];
  }
  return r;
}

__device__ __forceinline__ Vec8 unpack8(const Raw8<Bf16>& r) {
  Vec8 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x.v[2 * i] = __uint_as_float(r.a[i] << 16);
    x.v[2 * i + 1] = __uint_as_float(r.a[i] & 0xFFFF0000u);
  }
  return x;
}
__device__ __forceinline__ Vec8 unpack8(const Raw8<F32>& r) {
  Vec8 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x.v[i] = __uint_as_float(r.a[i]);
    x.v[4 + i] = __uint_as_float(r.b[i]);
  }
  return x;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const bf16x2 b = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, b);
}

template <bool kPast>
__device__ __forceinline__ void put16(u32x4* q, const u32x4& a) {
  if constexpr (kPast) __builtin_nontemporal_store(a, q);
  else *q = a;
}

template <class T, bool kPast = false>
__device__ __forceinline__ void store8(unsigned char* p, int64_t i, const Vec8& x) {
  u32x4* q = reinterpret_cast<u32x4*>(p + i * (8 * T::kBytes));
  if constexpr (T::kBytes == 2) {
    u32x4 a;
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] = pack_bf16(x.v[2 * k], x.v[2 * k + 1]);
    put16<kPast>(q, a);
  } else {
    u32x4 a, b;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      a[k] = __float_as_uint(x.v[k]);
      b[k] = __float_as_uint(x.v[4 + k]);
    }
    put16<kPast>(q, a);
    put16<kPast>(q + 1, b);
  }
}

}  // namespace pspo
