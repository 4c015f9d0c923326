// Device helpers of the kernels that write 8-bit matrices (apc_quantize.cu,
// apc_rmsnorm.cu): elements in words, scales, conversions.
#pragma once

#include "apc_ops.cuh"
#include "apc_tcgen05.cuh"

namespace apc {

// A pair of 16-bit elements, or one of 32 bits, in a word.  Magnitudes compare
// as integers.
template <typename T>
struct Word {
  static constexpr int kPer = 4 / sizeof(T);
  static constexpr uint32_t kAbs = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
  static __device__ __forceinline__ uint32_t max(uint32_t a, uint32_t b) { return sizeof(T) == 4 ? ::max(a, b) : __vmaxu2(a, b); }
};

// The bits of T's infinity.
template <typename T>
__device__ __forceinline__ constexpr uint32_t inf_bits();
template <>
__device__ __forceinline__ constexpr uint32_t inf_bits<float>() { return 0x7f800000u; }
template <>
__device__ __forceinline__ constexpr uint32_t inf_bits<__nv_bfloat16>() { return 0x7f80u; }
template <>
__device__ __forceinline__ constexpr uint32_t inf_bits<__half>() { return 0x7c00u; }

template <typename T>
__device__ __forceinline__ float bits_to_float(uint32_t b);  // b: an element's bits, zero-extended
template <>
__device__ __forceinline__ float bits_to_float<float>(uint32_t b) { return __uint_as_float(b); }
template <>
__device__ __forceinline__ float bits_to_float<__nv_bfloat16>(uint32_t b) { return __uint_as_float(b << 16); }
template <>
__device__ __forceinline__ float bits_to_float<__half>(uint32_t b) { return __half2float(__ushort_as_half((unsigned short)b)); }

// Element i of some words.
template <typename T>
__device__ __forceinline__ uint32_t element_bits(const uint32_t *w, int i) {
  if (sizeof(T) == 4) return w[i];
  return i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
}

template <typename T>
__device__ __forceinline__ float element(const uint32_t *w, int i) {
  if (sizeof(T) == 4) return __uint_as_float(w[i]);
  if (inf_bits<T>() == 0x7f80u) return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  return bits_to_float<T>(element_bits<T>(w, i));
}

// The word with non-finite elements as zeros, magnitudes only.
template <typename T>
__device__ __forceinline__ uint32_t finite_abs(uint32_t w) {
  w &= Word<T>::kAbs;
  if (sizeof(T) == 4) return w >= 0x7f800000u ? 0 : w;
  if ((w & 0xffffu) >= inf_bits<T>()) w &= 0xffff0000u;
  if ((w >> 16) >= inf_bits<T>()) w &= 0xffffu;
  return w;
}

// The larger of a word's elements.
template <typename T>
__device__ __forceinline__ uint32_t larger(uint32_t w) {
  return sizeof(T) == 4 ? w : max(w & 0xffffu, w >> 16);
}

// The exponent e of the scale, biased by 127: 2^e * largest >= amax > 2^(e-1) *
// largest.  The largest value is 1.75 * 2^8 (E4M3) or 1.75 * 2^15 (E5M2), so only
// fractions above 1.75 need the next power.
template <bool E5M2>
__device__ __forceinline__ uint32_t scale_exponent(float amax) {
  const uint32_t b = __float_as_uint(amax) + 0x1fffffu;  // carries into the exponent above a fraction of 1.75
  const int e = (int)(b >> 23) - (E5M2 ? 15 : 8);        // a subnormal amax is below 2^-126 * largest as it is
  return amax == 0.0f ? 127u : (uint32_t)max(e, 1);
}

__device__ __forceinline__ float power(uint32_t biased) { return __uint_as_float(biased << 23); }
// 2^-e: 2^127 (e = -127) does not occur, 2^-126 does.
__device__ __forceinline__ float inverse_power(uint32_t biased) { return __uint_as_float((254u - biased) << 23); }

// The 8-bit value of x times a power of two; non-finite values with their sign.
template <bool E5M2>
__device__ __forceinline__ uint8_t any_to_fp8(float x, float inv) {
  const uint32_t b = __float_as_uint(x), m = b & 0x7fffffffu;
  if (m >= 0x7f800000u) return (uint8_t)((E5M2 && m == 0x7f800000u ? 0x7cu : 0x7fu) | (b >> 24 & 0x80u));
  return (uint8_t)to_fp8x2<E5M2>(x * inv, 0.0f);
}

// Pairs (lo, hi) of finite values times inv, 8 in a row, little-endian.
template <bool E5M2>
__device__ __forceinline__ uint2 to_fp8x8(const uint64_t (&v)[4], uint64_t inv) {
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = unpack2(mul2(v[i], inv));
    h[i] = to_fp8x2<E5M2>(y.x, y.y);
  }
  return {__byte_perm(h[0], h[1], 0x5410), __byte_perm(h[2], h[3], 0x5410)};
}

// How memory is read.  The read-only path is for what nothing writes while the kernel runs;
// a matrix that an output may replace is read plainly; and what a kernel that is still running
// when this one starts has written, from L2, behind the wait for that kernel.
enum class Read { kOnly, kPlain, kL2 };

template <Read HOW, typename U>
__device__ __forceinline__ U read(const U *p) {
  if (HOW == Read::kOnly) return __ldg(p);
  if (HOW == Read::kL2) return __ldcg(p);
  return *p;
}

// 8 elements from x, of which the first n exist, as words; `wide`: x is 16-byte aligned.
template <typename T, Read HOW = Read::kOnly>
__device__ __forceinline__ void load8(uint32_t *w, const T *x, int n, bool wide) {
  constexpr int kWords = 8 / Word<T>::kPer;
  if (wide && n >= 8) {
#pragma unroll
    for (int i = 0; i < kWords; i += 4) {
      const uint4 v = read<HOW>(reinterpret_cast<const uint4 *>(x) + i / 4);
      w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if (sizeof(T) == 4) {
        w[i] = i < n ? read<HOW>(reinterpret_cast<const uint32_t *>(x) + i) : 0;
      } else {
        const uint32_t lo = 2 * i < n ? read<HOW>(reinterpret_cast<const uint16_t *>(x) + 2 * i) : 0;
        const uint32_t hi = 2 * i + 1 < n ? read<HOW>(reinterpret_cast<const uint16_t *>(x) + 2 * i + 1) : 0;
        w[i] = hi << 16 | lo;
      }
    }
  }
}

// The first n of 8 bytes to 8-byte aligned memory.
__device__ __forceinline__ void store8(uint8_t *at, uint2 v, int n) {
  if (n >= 8) {
    *reinterpret_cast<uint2 *>(at) = v;
  } else {
    for (int i = 0; i < n; ++i) at[i] = (uint8_t)((i < 4 ? v.x : v.y) >> (i % 4 * 8));
  }
}

}  // namespace apc
