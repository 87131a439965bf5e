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
  __device__ __forceinline__ void set(int e, float f) { v[e] = f; }
};
template <>
struct Raw8<bf16> {
  uint32_t v[4];
  __device__ __forceinline__ float get(int e) const {
    const uint32_t w = v[e >> 1];
    return __uint_as_float((e & 1) ? (w & 0xffff0000u) : (w << 16));
  }
  __device__ __forceinline__ void set(int e, float f) {
    const uint32_t h = (uint32_t)__builtin_bit_cast(uint16_t, (bf16)f);
    v[e >> 1] = (e & 1) ? ((v[e >> 1] & 0xffffu) | (h << 16)) : ((v[e >> 1] & 0xffff0000u) | h);
  }
};

// n: how many of the eight are inside the row (<= 0: none); the others are 0.
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p, int n) {
  Raw8<T> r;
  if (n >= 8) {
    __builtin_memcpy(&r, p, sizeof(r));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.set(e, 0.f);
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) r.set(e, tof(p[e]));
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, const float (&f)[8]) {
  if (n >= 8) {
    Raw8<T> r = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) r.set(e, f[e]);
    __builtin_memcpy(p, &r, sizeof(r));
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) p[e] = (T)f[e];
  }
}

}  // namespace dev
}  // namespace mgn
