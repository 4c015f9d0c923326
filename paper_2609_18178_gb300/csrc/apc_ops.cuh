// Device helpers that the operators' kernels share: element types and 8-bit
// formats.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "apc_ops.h"

namespace apc {

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// Two values to 8 bits each, nearest even, `lo` in the low byte.  The
// instruction saturates: infinities are the caller's.
template <bool E5M2>
__device__ __forceinline__ uint32_t to_fp8x2(float lo, float hi) {
  uint16_t r;
  if (E5M2) asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// 2^x, to 2 ulp, subnormal results flushed to zero.
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// f(T{}) for the element type of an apc_dtype.
template <typename F>
int with_dtype(uint32_t dtype, F f) {
  switch (dtype) {
    case APC_F32: return f(float{});
    case APC_BF16: return f(__nv_bfloat16{});
    default: return f(__half{});
  }
}

}  // namespace apc
