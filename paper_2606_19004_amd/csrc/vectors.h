// Vectors of elements at the alignment of one element, which the memory unit allows (8, 4 or 2 at a time; math in fp32).
#pragma once
#include "internal.h"

namespace dit {

typedef unsigned u32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void unpack8(const uint32_t* w, float* f) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8_any(const u16* p, float* f) {
  const u32x4_any2 u = *(const u32x4_any2*)p;
  const uint32_t w[4] = {u[0], u[1], u[2], u[3]};
  unpack8(w, f);
}
__device__ __forceinline__ void load8_any(const float* p, float* f) {
  const f32x4_any4 u = *(const f32x4_any4*)p, v = *(const f32x4_any4*)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    f[i] = u[i];
    f[4 + i] = v[i];
  }
}
__device__ __forceinline__ void store8_any(u16* p, const float* f) {
  *(u32x4_any2*)p = u32x4_any2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
}
__device__ __forceinline__ void store8_any(float* p, const float* f) {
  *(f32x4_any4*)p = f32x4_any4{f[0], f[1], f[2], f[3]};
  *(f32x4_any4*)(p + 4) = f32x4_any4{f[4], f[5], f[6], f[7]};
}
typedef unsigned u32x2_any2 __attribute__((ext_vector_type(2), aligned(2)));
typedef unsigned u32_any2 __attribute__((aligned(2)));
typedef float f32x2_any4 __attribute__((ext_vector_type(2), aligned(4)));
__device__ __forceinline__ void store4_any(u16* p, const float* f) { *(u32x2_any2*)p = u32x2_any2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])}; }
__device__ __forceinline__ void store4_any(float* p, const float* f) { *(f32x4_any4*)p = f32x4_any4{f[0], f[1], f[2], f[3]}; }
__device__ __forceinline__ void store2_any(u16* p, const float* f) { *(u32_any2*)p = pack_bf16x2(f[0], f[1]); }
__device__ __forceinline__ void store2_any(float* p, const float* f) { *(f32x2_any4*)p = f32x2_any4{f[0], f[1]}; }

}  // namespace dit
