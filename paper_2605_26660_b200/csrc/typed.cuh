// Values of a runtime type (fp16, bf16, fp32) eight at a time.  The type is the same for a whole launch, so the
// branches are uniform; they cost nothing next to the memory access they choose.
#pragma once

#include <cuda_bf16.h>

#include "windq_internal.cuh"

namespace windq {

__host__ __device__ inline int dtype_bytes(int dt) { return dt == WINDQ_F32 ? 4 : 2; }

__device__ __forceinline__ float2 unpack2(uint32_t w, int dt) {
  if (dt == WINDQ_F16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pack2(float a, float b, int dt) {
  uint32_t w;
  if (dt == WINDQ_F16) {
    const __half2 h = __floats2half2_rn(a, b);
    w = *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    w = *reinterpret_cast<const uint32_t*>(&h);
  }
  return w;
}

// Eight consecutive values at a 16-byte aligned address (32 bytes of fp32, 16 of the others).
__device__ __forceinline__ void load8(const void* base, int64_t i, int dt, float (&x)[8]) {
  if (dt == WINDQ_F32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + i);
    const float4 a = p[0], b = p[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
    const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + i);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int k = 0; k < 4; k++) {
      const float2 f = unpack2(w[k], dt);
      x[2 * k] = f.x;
      x[2 * k + 1] = f.y;
    }
  }
}
__device__ __forceinline__ void store8(void* base, int64_t i, int dt, const float (&x)[8]) {
  if (dt == WINDQ_F32) {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + i);
    p[0] = make_float4(x[0], x[1], x[2], x[3]);
    p[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint4 a;
    a.x = pack2(x[0], x[1], dt);
    a.y = pack2(x[2], x[3], dt);
    a.z = pack2(x[4], x[5], dt);
    a.w = pack2(x[6], x[7], dt);
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + i) = a;
  }
}
// One value, for the ragged end of a tensor.
__device__ __forceinline__ float load1(const void* base, int64_t i, int dt) {
  if (dt == WINDQ_F32) return static_cast<const float*>(base)[i];
  return unpack2(static_cast<const uint16_t*>(base)[i], dt).x;
}
__device__ __forceinline__ void store1(void* base, int64_t i, int dt, float x) {
  if (dt == WINDQ_F32) static_cast<float*>(base)[i] = x;
  else static_cast<uint16_t*>(base)[i] = (uint16_t)pack2(x, 0.0f, dt);
}
// `live` (1..7) of the eight values; the others read as zero and are not written.
__device__ __forceinline__ void load_some(const void* base, int64_t i, int dt, int live, float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 8; k++) x[k] = k < live ? load1(base, i + k, dt) : 0.0f;
}
__device__ __forceinline__ void store_some(void* base, int64_t i, int dt, int live, const float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 8; k++)
    if (k < live) store1(base, i + k, dt, x[k]);
}

}  // namespace windq
