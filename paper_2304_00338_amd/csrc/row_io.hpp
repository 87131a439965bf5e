// Eight consecutive elements of a row tensor in registers: loads and stores
// that need no more than the element's own alignment, and a row's end.
#pragma once

#include "dev_common.hpp"

namespace mgn {
namespace dev {

template <typename T>
struct Raw8;
template <>
struct Raw8<float> {
  float v[8];
  __device__ __forceinline__ float get(int e) const { return v[e]; }
  __device__ __forceinline__ void put(int e, float f) { v[e] = f; }
};
template <>
struct Raw8<bf16> {
  uint32_t v[4];
  __device__ __forceinline__ float get(int e) const {
    const uint32_t w = v[e >> 1];
    return __uint_as_float((e & 1) ? (w & 0xffff0000u) : (w << 16));
  }
  __device__ __forceinline__ void put(int e, bf16 f) { v[e >> 1] |= (uint32_t)__builtin_bit_cast(uint16_t, f) << (16 * (e & 1)); }
};

__device__ __forceinline__ Raw8<float> raw8(const float (&f)[8], float) {
  Raw8<float> r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r.v[e] = f[e];
  return r;
}
// as vectors, for the instruction that rounds two at a time
__device__ __forceinline__ Raw8<bf16> raw8(const float (&f)[8], bf16) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  Raw8<bf16> r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r.v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){f[2 * i], f[2 * i + 1]}, bf16x2));
  return r;
}

// The eight elements from p on, of which the first n are inside the row (<= 0:
// none); the others are 0.
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p, int n) {
  Raw8<T> r;
  if (n >= 8) {
    __builtin_memcpy(&r, p, sizeof(r));
  } else {
    // bits, not values: a conversion here would be moved before the loads' wait
    r = Raw8<T>{};
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) r.put(e, p[e]);
  }
  return r;
}
// Elements [lo, hi) of the eight.
template <typename T>
__device__ __forceinline__ void store8(T* p, int lo, int hi, const float (&f)[8]) {
  if (hi - lo == 8) {
    const Raw8<T> r = raw8(f, T());
    __builtin_memcpy(p, &r, sizeof(r));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= lo && e < hi) p[e] = (T)f[e];
  }
}
// Elements outside of [lo, hi) become 0.
__device__ __forceinline__ void keep(Raw8<float>& r, int lo, int hi) {
#pragma unroll
  for (int e = 0; e < 8; ++e) r.v[e] = e >= lo && e < hi ? r.v[e] : 0.f;
}
__device__ __forceinline__ void keep(Raw8<bf16>& r, int lo, int hi) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r.v[i] &= (2 * i >= lo && 2 * i < hi ? 0xffffu : 0u) | (2 * i + 1 >= lo && 2 * i + 1 < hi ? 0xffff0000u : 0u);
}

}  // namespace dev
}  // namespace mgn
