// Eight consecutive elements of a row as fp32, from and to any element
// address: one or two 16-byte accesses (the hardware takes them unaligned),
// by element where the row ends first (n < 8; missing elements read as 0).
#pragma once

#include "device.h"

namespace ffmlp {

typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ u32x4 load8_bits(const uint16_t* p, int n) {
  if (n >= 8) return *reinterpret_cast<const u32x4_a2*>(p);
  u32x4 x = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int q = 0; q < 8; ++q)
    if (q < n) x[q / 2] |= (uint32_t)p[q] << (16 * (q & 1));
  return x;
}
__device__ __forceinline__ void widen8(const u32x4& x, float (&v)[8]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v[2 * q] = bf16_lo(x[q]);
    v[2 * q + 1] = bf16_hi(x[q]);
  }
}
__device__ __forceinline__ void load8(const uint16_t* p, int n, float (&v)[8]) { widen8(load8_bits(p, n), v); }
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
  if (n >= 8) {
    const f32x4 a = *reinterpret_cast<const f32x4_a4*>(p), b = *reinterpret_cast<const f32x4_a4*>(p + 4);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[q] = a[q];
      v[q + 4] = b[q];
    }
  } else {
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = q < n ? p[q] : 0.f;
  }
}
// eight floats in LDS, 16-byte aligned
__device__ __forceinline__ void lds8(const float* p, float (&v)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v[q] = a[q];
    v[q + 4] = b[q];
  }
}
template <bool NT = false>
__device__ __forceinline__ void store8(uint16_t* p, int n, const float (&v)[8]) {
  const u32x4 x = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  if (n >= 8) {
    if (NT) __builtin_nontemporal_store(x, reinterpret_cast<u32x4_a2*>(p));
    else *reinterpret_cast<u32x4_a2*>(p) = x;
  } else {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < n) p[q] = (uint16_t)(x[q / 2] >> (16 * (q & 1)));
  }
}
template <bool NT = false>
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    if (NT) {
      __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_a4*>(p));
      __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4_a4*>(p + 4));
    } else {
      *reinterpret_cast<f32x4_a4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4_a4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
  } else {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < n) p[q] = v[q];
  }
}

}  // namespace ffmlp
