// Two floats at a time (one instruction for two values), and vectors of values of either type.
#pragma once
#include "hbp_internal.h"

namespace hbp {

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair_of(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 floats_of(f32x2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 both(float a) { return pair_of(a, a); }

// The values of two neighbouring elements, and back
__device__ __forceinline__ f32x2 widen2(const float* v) { return pair_of(v[0], v[1]); }
__device__ __forceinline__ f32x2 widen2(const bf16* v) {
  const uint32_t w = *reinterpret_cast<const uint32_t*>(v);
  return pair_of(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ void narrow2(f32x2 x, float* v) {
  const float2 f = floats_of(x);
  v[0] = f.x;
  v[1] = f.y;
}
__device__ __forceinline__ void narrow2(f32x2 x, bf16* v) {
  const float2 f = floats_of(x);
  *reinterpret_cast<__nv_bfloat162*>(v) = __floats2bfloat162_rn(f.x, f.y);
}
// The values of a vector of 16 bytes, and back
template <int N, typename T>
__device__ __forceinline__ void widen(const T* v, float* f) {
#pragma unroll
  for (int e = 0; e < N; e += 2) {
    const float2 t = floats_of(widen2(v + e));
    f[e] = t.x;
    f[e + 1] = t.y;
  }
}
template <int N, typename T>
__device__ __forceinline__ void narrow(const float* f, T* v) {
#pragma unroll
  for (int e = 0; e < N; e += 2) narrow2(pair_of(f[e], f[e + 1]), v + e);
}

}  // namespace hbp
