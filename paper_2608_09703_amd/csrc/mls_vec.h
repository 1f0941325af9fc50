// Row chunks of bf16 or fp32 storage <-> fp32 registers, with the default or the
// non-temporal cache policy (NT).
#pragma once

#include "mls_device.h"

namespace mls {

// 16 bytes at an element's address (bf16 or fp32: any even one)
typedef unsigned int u32x4_any_t __attribute__((ext_vector_type(4), aligned(2)));
template <bool NT>
__device__ __forceinline__ uint4 load16_any(const void* p) {
  const u32x4_any_t* q = static_cast<const u32x4_any_t*>(p);
  const u32x4_any_t v = NT ? __builtin_nontemporal_load(q) : *q;
  return make_uint4(v.x, v.y, v.z, v.w);
}
template <bool NT>
__device__ __forceinline__ void store16_any(void* p, uint4 v) {
  const u32x4_any_t w = {v.x, v.y, v.z, v.w};
  if (NT)
    __builtin_nontemporal_store(w, static_cast<u32x4_any_t*>(p));
  else
    *static_cast<u32x4_any_t*>(p) = w;
}

typedef unsigned int u32x2j __attribute__((ext_vector_type(2)));
template <bool NT>
__device__ __forceinline__ uint2 ld8(const void* p) {
  if (NT) {
    const u32x2j v = __builtin_nontemporal_load(static_cast<const u32x2j*>(p));
    return make_uint2(v.x, v.y);
  }
  return *reinterpret_cast<const uint2*>(p);
}
template <bool NT>
__device__ __forceinline__ void st8(void* p, uint2 v) {
  if (NT)
    __builtin_nontemporal_store(u32x2j{v.x, v.y}, static_cast<u32x2j*>(p));
  else
    *reinterpret_cast<uint2*>(p) = v;
}
template <bool NT>
__device__ __forceinline__ uint4 ld16(const void* p) {
  return NT ? load16_nt(p) : *reinterpret_cast<const uint4*>(p);
}
template <bool NT>
__device__ __forceinline__ void st16(void* p, uint4 v) {
  if (NT)
    store16_nt(p, v);
  else
    *reinterpret_cast<uint4*>(p) = v;
}

// 8 consecutive elements <-> 8 floats, 16-byte accesses (the forward's lane
// mapping)
template <bool NT>
__device__ __forceinline__ void load8(const uint16_t* p, float* v) {
  const uint4 r = ld16<NT>(p);
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
template <bool NT>
__device__ __forceinline__ void load8(const float* p, float* v) {
  const uint4 a = ld16<NT>(p);
  const uint4 b = ld16<NT>(p + 4);
  v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y);
  v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
  v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y);
  v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
}
template <bool NT>
__device__ __forceinline__ void store8(uint16_t* p, const float* v) {
  uint4 r;
  r.x = (uint32_t)to_storage<Bf16>(v[0]) | ((uint32_t)to_storage<Bf16>(v[1]) << 16);
  r.y = (uint32_t)to_storage<Bf16>(v[2]) | ((uint32_t)to_storage<Bf16>(v[3]) << 16);
  r.z = (uint32_t)to_storage<Bf16>(v[4]) | ((uint32_t)to_storage<Bf16>(v[5]) << 16);
  r.w = (uint32_t)to_storage<Bf16>(v[6]) | ((uint32_t)to_storage<Bf16>(v[7]) << 16);
  st16<NT>(p, r);
}
template <bool NT>
__device__ __forceinline__ void store8(float* p, const float* v) {
  st16<NT>(p, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                         __float_as_uint(v[3])));
  st16<NT>(p + 4, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]),
                             __float_as_uint(v[7])));
}

// 4 consecutive elements <-> 4 floats, 8-byte (bf16) or 16-byte (fp32)
// accesses (the backward's lane mapping)
template <bool NT>
__device__ __forceinline__ void load4(const uint16_t* p, float* v) {
  const uint2 r = ld8<NT>(p);
  v[0] = __uint_as_float(r.x << 16);
  v[1] = __uint_as_float(r.x & 0xffff0000u);
  v[2] = __uint_as_float(r.y << 16);
  v[3] = __uint_as_float(r.y & 0xffff0000u);
}
template <bool NT>
__device__ __forceinline__ void load4(const float* p, float* v) {
  const uint4 r = ld16<NT>(p);
  v[0] = __uint_as_float(r.x);
  v[1] = __uint_as_float(r.y);
  v[2] = __uint_as_float(r.z);
  v[3] = __uint_as_float(r.w);
}
template <bool NT>
__device__ __forceinline__ void store4(uint16_t* p, const float* v) {
  st8<NT>(p, make_uint2((uint32_t)to_storage<Bf16>(v[0]) | ((uint32_t)to_storage<Bf16>(v[1]) << 16),
                        (uint32_t)to_storage<Bf16>(v[2]) | ((uint32_t)to_storage<Bf16>(v[3]) << 16)));
}
template <bool NT>
__device__ __forceinline__ void store4(float* p, const float* v) {
  st16<NT>(p, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                         __float_as_uint(v[3])));
}

template <typename T>
struct Elt;
template <>
struct Elt<Bf16> {
  typedef uint16_t type;
};
template <>
struct Elt<F32> {
  typedef float type;
};

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float widen(float v) { return v; }

// A chunk of 16 bytes: kN elements.
template <typename A>
struct Chunk;
template <>
struct Chunk<Bf16> {
  static constexpr int kN = 8;
  __device__ __forceinline__ static void unpack(uint4 r, float* v) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ static uint4 pack(const float* v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = (uint32_t)to_storage<Bf16>(v[2 * i]) | ((uint32_t)to_storage<Bf16>(v[2 * i + 1]) << 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Chunk<F32> {
  static constexpr int kN = 4;
  __device__ __forceinline__ static void unpack(uint4 r, float* v) {
    v[0] = __uint_as_float(r.x);
    v[1] = __uint_as_float(r.y);
    v[2] = __uint_as_float(r.z);
    v[3] = __uint_as_float(r.w);
  }
  __device__ __forceinline__ static uint4 pack(const float* v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};

}  // namespace mls
