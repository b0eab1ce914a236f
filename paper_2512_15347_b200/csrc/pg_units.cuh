// Units of eight logits: how the rules on logits read, convert and write them.  Of it the policy update on tokens uses pack2; its own units are
// 16 bytes of any type.
#pragma once

#include "pg_kv.cuh"

namespace pg {

constexpr int kUnit = 8;                      // tokens that a thread handles at a time

__device__ __forceinline__ void unpack8(const uint4& a, float (&x)[8], __nv_bfloat16) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack8(const uint4& a, float (&x)[8], __half) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
// Eight logits as they lie in memory.
template <typename T> struct Raw8 { uint4 v[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ void load8(const T* at, Raw8<T>& r) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = __ldcs((const uint4*)at + i);
}
template <typename T>
__device__ __forceinline__ void floats8(const Raw8<T>& r, float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[4 * i] = __uint_as_float(r.v[i].x);
      x[4 * i + 1] = __uint_as_float(r.v[i].y);
      x[4 * i + 2] = __uint_as_float(r.v[i].z);
      x[4 * i + 3] = __uint_as_float(r.v[i].w);
    }
  } else {
    unpack8(r.v[0], x, T());
  }
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T>
__device__ __forceinline__ void store8(T* at, const float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    __stcs((float4*)at, make_float4(x[0], x[1], x[2], x[3]));
    __stcs((float4*)at + 1, make_float4(x[4], x[5], x[6], x[7]));
  } else {
    __stcs((uint4*)at, make_uint4(pack2(x[0], x[1], T()), pack2(x[2], x[3], T()), pack2(x[4], x[5], T()), pack2(x[6], x[7], T())));
  }
}

}  // namespace pg
