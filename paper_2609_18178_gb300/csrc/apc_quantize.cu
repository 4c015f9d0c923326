// Quantization to 8 bits with a power-of-two scale per block (apc_quantize_fp8).
//
//   scale = 2^e, the smallest with max |x| <= 2^e * largest, e >= -126
//   q     = x / scale rounded to nearest even; the division by a power of two
//           is exact, so it is a multiplication by 2^-e
//
// One read of x and one write of each output: bound by memory.  Two kernels:
// rows alone, where half a warp owns a block of 128, and tiles of 128 x 128,
// for square blocks and for the transpose, whose blocks run down the columns.
#include <cuda_runtime.h>

#include "apc_ops.cuh"

namespace apc {

namespace {

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
__device__ __forceinline__ uint32_t scale_exponent(float amax, bool e5m2) {
  const uint32_t b = __float_as_uint(amax) + 0x1fffffu;  // carries into the exponent above a fraction of 1.75
  const int e = (int)(b >> 23) - (e5m2 ? 15 : 8);        // a subnormal amax is below 2^-126 * largest as it is
  return amax == 0.0f ? 127u : (uint32_t)max(e, 1);
}

__device__ __forceinline__ float power(uint32_t biased) { return __uint_as_float(biased << 23); }
// 2^-e: 2^127 (e = -127) does not occur, 2^-126 does.
__device__ __forceinline__ float inverse_power(uint32_t biased) { return __uint_as_float((254u - biased) << 23); }

// The 8-bit value of a non-finite x; sign kept.
__device__ __forceinline__ uint32_t non_finite(float x, bool e5m2) {
  const uint32_t b = __float_as_uint(x);
  return (e5m2 && (b & 0x7fffffffu) == 0x7f800000u ? 0x7cu : 0x7fu) | (b >> 24 & 0x80u);
}

// Two values to 8 bits, x0 in the low byte.  AWKWARD: they may be non-finite.
template <bool AWKWARD>
__device__ __forceinline__ uint32_t pair_to_fp8(float x0, float x1, float inv0, float inv1, bool e5m2) {
  uint32_t r = to_fp8x2(x0 * inv0, x1 * inv1, e5m2);
  if (AWKWARD) {
    if (!(fabsf(x0) <= 3.402823466e38f)) r = (r & 0xff00u) | non_finite(x0, e5m2);
    if (!(fabsf(x1) <= 3.402823466e38f)) r = (r & 0xffu) | non_finite(x1, e5m2) << 8;
  }
  return r;
}

// 8 values in a row, little-endian.
template <typename T, bool AWKWARD>
__device__ __forceinline__ uint2 row_to_fp8(const uint32_t *w, float inv, bool e5m2) {
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = pair_to_fp8<AWKWARD>(element<T>(w, 2 * i), element<T>(w, 2 * i + 1), inv, inv, e5m2);
  return {__byte_perm(h[0], h[1], 0x5410), __byte_perm(h[2], h[3], 0x5410)};
}

// 8 elements from x, of which the first n exist, as words; `wide`: x is 16-byte aligned.
template <typename T>
__device__ __forceinline__ void load8(uint32_t *w, const T *x, int n, bool wide) {
  constexpr int kWords = 8 / Word<T>::kPer;
  if (wide && n >= 8) {
#pragma unroll
    for (int i = 0; i < kWords; i += 4) {
      const uint4 v = __ldg(reinterpret_cast<const uint4 *>(x) + i / 4);
      w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if (sizeof(T) == 4) {
        w[i] = i < n ? __ldg(reinterpret_cast<const uint32_t *>(x) + i) : 0;
      } else {
        const uint32_t lo = 2 * i < n ? __ldg(reinterpret_cast<const uint16_t *>(x) + 2 * i) : 0;
        const uint32_t hi = 2 * i + 1 < n ? __ldg(reinterpret_cast<const uint16_t *>(x) + 2 * i + 1) : 0;
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

// ---------------------------------------------------------------------------
// Rows alone.  The blocks of the whole matrix in row order; half a warp takes
// one, 8 elements a lane, kRowUnroll of them in flight.
constexpr int kRowThreads = 256, kRowUnroll = 4;

template <typename T>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(const T *x, int64_t pitch, uint32_t rows, uint32_t cols, QuantOut q,
                                                           bool wide) {
  constexpr int kWords = 8 / Word<T>::kPer;
  const uint32_t lane = threadIdx.x % 32, side = lane / 16, c8 = lane % 16 * 8;
  const uint32_t across = (cols + kBlock - 1) / kBlock;
  const uint64_t blocks = (uint64_t)across * rows, step = (uint64_t)gridDim.x * (kRowThreads / 32) * (2 * kRowUnroll);
  for (uint64_t b0 = ((uint64_t)blockIdx.x * (kRowThreads / 32) + threadIdx.x / 32) * (2 * kRowUnroll); b0 < blocks; b0 += step) {
    uint32_t w[kRowUnroll][kWords], row[kRowUnroll], bc[kRowUnroll];
    int n[kRowUnroll];
#pragma unroll
    for (int u = 0; u < kRowUnroll; ++u) {
      const uint64_t b = b0 + 2 * u + side;
      row[u] = blocks >> 32 ? (uint32_t)(b / across) : (uint32_t)b / across;
      bc[u] = (uint32_t)b - row[u] * across;
      const uint32_t c = bc[u] * kBlock + c8;
      n[u] = b < blocks && c < cols ? (int)min(8u, cols - c) : 0;
      load8<T>(w[u], x + (int64_t)row[u] * pitch + c, n[u], wide);
    }
#pragma unroll
    for (int u = 0; u < kRowUnroll; ++u) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < kWords; ++i) m = Word<T>::max(m, w[u][i] & Word<T>::kAbs);
      uint32_t top = larger<T>(m);
#pragma unroll
      for (int o = 8; o; o >>= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
      const bool awkward = __any_sync(~0u, top >= inf_bits<T>());
      if (awkward) {
        m = 0;
        for (int i = 0; i < kWords; ++i) m = Word<T>::max(m, finite_abs<T>(w[u][i]));
        top = larger<T>(m);
        for (int o = 8; o; o >>= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
      }
      const uint32_t e = scale_exponent(bits_to_float<T>(top), q.e5m2);
      const float inv = inverse_power(e);
      if (c8 == 0 && n[u]) q.scale[(int64_t)bc[u] * q.scale_pitch + row[u]] = power(e);
      if (n[u])
        store8(q.data + (int64_t)row[u] * q.pitch + bc[u] * kBlock + c8,
               awkward ? row_to_fp8<T, true>(w[u], inv, q.e5m2) : row_to_fp8<T, false>(w[u], inv, q.e5m2), n[u]);
    }
  }
}

// ---------------------------------------------------------------------------
// Tiles of 128 x 128.  Thread (tx, ty) holds rows 8 ty + 0..7 of columns 8 tx +
// 0..7 in registers from one load to both stores.  Row maxima are reduced over the
// 16 lanes of a row, column maxima through shared memory; the transpose goes
// through shared memory in 8-byte pieces, swizzled so that neither side meets a
// bank twice.
constexpr int kTileThreads = 256;

template <typename T, bool AWKWARD>
__device__ __forceinline__ void store_tile(const uint32_t (&w)[8][8 / Word<T>::kPer], const uint32_t (&re)[8], const uint32_t (&ce)[8],
                                           const QuantArgs &a, uint32_t r0, uint32_t c0, uint32_t tx, uint32_t ty, uint2 *turn) {
  const uint32_t r = r0 + 8 * ty, c = c0 + 8 * tx;
  const int nc = c < a.cols ? (int)min(8u, a.cols - c) : 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (r + i < a.rows && nc)
      store8(a.q.data + (int64_t)(r + i) * a.q.pitch + c, row_to_fp8<T, AWKWARD>(w[i], inverse_power(re[i]), a.q.e5m2), nc);
  if (!a.qt.data) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t h[4];
    const float inv = inverse_power(ce[j]);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = pair_to_fp8<AWKWARD>(element<T>(w[2 * i], j), element<T>(w[2 * i + 1], j), inv, inv, a.qt.e5m2);
    turn[(8 * tx + j) * 16 + (ty ^ tx)] = {__byte_perm(h[0], h[1], 0x5410), __byte_perm(h[2], h[3], 0x5410)};
  }
  __syncthreads();
  const uint32_t rr = r0 + 8 * tx;  // now tx counts pieces down a column
  const int nr = rr < a.rows ? (int)min(8u, a.rows - rr) : 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t col = 16 * i + ty;
    if (c0 + col < a.cols && nr)
      store8(a.qt.data + (int64_t)(c0 + col) * a.qt.pitch + rr, turn[col * 16 + (tx ^ col / 8)], nr);
  }
}

template <typename T, bool SQUARE>
__global__ void __launch_bounds__(kTileThreads, sizeof(T) == 4 ? 2 : 3) tile_kernel(const __grid_constant__ QuantArgs a, bool wide) {
  constexpr int kWords = 8 / Word<T>::kPer;  // words of 8 elements
  __shared__ uint2 turn[128 * 16];
  __shared__ __align__(16) uint32_t s_col[8][16 * kWords];
  const uint32_t tx = threadIdx.x % 16, ty = threadIdx.x / 16, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t across = (a.cols + kBlock - 1) / kBlock, down = (a.rows + kBlock - 1) / kBlock;
  for (uint64_t t = blockIdx.x; t < (uint64_t)across * down; t += gridDim.x) {
    const uint32_t tr = (uint32_t)(t / across), tc = (uint32_t)(t % across), r0 = tr * kBlock, c0 = tc * kBlock;
    uint32_t w[8][kWords];
    {
      const uint32_t r = r0 + 8 * ty, c = c0 + 8 * tx;
      const int nc = c < a.cols ? (int)min(8u, a.cols - c) : 0;
      const T *x = static_cast<const T *>(a.x) + (int64_t)r * a.pitch + c;
#pragma unroll
      for (int i = 0; i < 8; ++i) load8<T>(w[i], x + (int64_t)i * a.pitch, r + i < a.rows ? nc : 0, wide);
    }
    uint32_t re[8], ce[8];  // exponents of the scales
    // The maxima of the tile's rows and columns; whether something in it is not finite.
    auto reduce = [&](auto magnitude) {
      uint32_t col[kWords], row[8];
#pragma unroll
      for (int k = 0; k < kWords; ++k) col[k] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < kWords; ++k) {
          const uint32_t v = magnitude(w[i][k]);
          col[k] = Word<T>::max(col[k], v);
          m = Word<T>::max(m, v);
        }
        row[i] = larger<T>(m);
      }
      if (SQUARE) {
        uint32_t m = row[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) m = max(m, row[i]);
        m = __reduce_max_sync(~0u, m);
        if (lane == 0) s_col[0][warp] = m;
        __syncthreads();
        m = s_col[0][lane % 8];
        m = __reduce_max_sync(~0u, m);
        const uint32_t eq = scale_exponent(bits_to_float<T>(m), a.q.e5m2), et = scale_exponent(bits_to_float<T>(m), a.qt.e5m2);
#pragma unroll
        for (int i = 0; i < 8; ++i) re[i] = eq, ce[i] = et;
        return m >= inf_bits<T>();
      }
      // rows: 16-bit maxima travel in pairs
      uint32_t top = 0;
      if (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          uint32_t p = row[i] | row[i + 1] << 16;
#pragma unroll
          for (int o = 8; o; o >>= 1) p = __vmaxu2(p, __shfl_xor_sync(~0u, p, o));
          row[i] = p & 0xffffu, row[i + 1] = p >> 16;
          top = max(top, max(row[i], row[i + 1]));
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
          for (int o = 8; o; o >>= 1) row[i] = max(row[i], __shfl_xor_sync(~0u, row[i], o));
          top = max(top, row[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) re[i] = scale_exponent(bits_to_float<T>(row[i]), a.q.e5m2);
      // columns
#pragma unroll
      for (int k = 0; k < kWords; ++k) col[k] = Word<T>::max(col[k], __shfl_xor_sync(~0u, col[k], 16));
      if (lane < 16) {
#pragma unroll
        for (int k = 0; k < kWords; k += 4)
          *reinterpret_cast<uint4 *>(&s_col[warp][tx * kWords + k]) = make_uint4(col[k], col[k + 1], col[k + 2], col[k + 3]);
      }
      const bool awkward = __syncthreads_or(top >= inf_bits<T>());
#pragma unroll
      for (int v = 0; v < 8; ++v) {
#pragma unroll
        for (int k = 0; k < kWords; k += 4) {
          const uint4 o = *reinterpret_cast<const uint4 *>(&s_col[v][tx * kWords + k]);
          col[k] = Word<T>::max(col[k], o.x), col[k + 1] = Word<T>::max(col[k + 1], o.y);
          col[k + 2] = Word<T>::max(col[k + 2], o.z), col[k + 3] = Word<T>::max(col[k + 3], o.w);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) ce[j] = scale_exponent(bits_to_float<T>(element_bits<T>(col, j)), a.qt.e5m2);
      return awkward;
    };
    const bool awkward = reduce([](uint32_t v) { return v & Word<T>::kAbs; });
    if (awkward) {
      __syncthreads();
      reduce([](uint32_t v) { return finite_abs<T>(v); });
    }
    if (SQUARE) {
      if (threadIdx.x == 0) {
        a.q.scale[(int64_t)tc * a.q.scale_pitch + tr] = power(re[0]);
        if (a.qt.data) a.qt.scale[(int64_t)tr * a.qt.scale_pitch + tc] = power(ce[0]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t r = r0 + 8 * ty + j, c = c0 + 8 * tx + j;
        if (tx == j && r < a.rows) a.q.scale[(int64_t)tc * a.q.scale_pitch + r] = power(re[j]);
        if (ty == j && c < a.cols) a.qt.scale[(int64_t)tr * a.qt.scale_pitch + c] = power(ce[j]);
      }
    }
    if (awkward) store_tile<T, true>(w, re, ce, a, r0, c0, tx, ty, turn);
    else store_tile<T, false>(w, re, ce, a, r0, c0, tx, ty, turn);
    __syncthreads();
  }
}

// Rows alone need no tile unless the blocks are square.
bool rows_alone(const QuantArgs &a) { return !a.square && !a.qt.data; }

}  // namespace

int quantize_per_sm(const QuantArgs &a) { return rows_alone(a) ? 8 : a.dtype == APC_F32 ? 2 : 3; }

int launch_quantize(const QuantArgs &a, unsigned cap, void *stream) {
  return with_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    const bool wide = (uintptr_t)a.x % 16 == 0 && a.pitch * sizeof(T) % 16 == 0;
    const uint32_t across = (a.cols + kBlock - 1) / kBlock, down = (a.rows + kBlock - 1) / kBlock;
    cudaStream_t s = (cudaStream_t)stream;
    if (rows_alone(a)) {
      const uint64_t each = kRowThreads / 32 * 2 * kRowUnroll, want = ((uint64_t)across * a.rows + each - 1) / each;
      rows_kernel<T><<<(unsigned)(want < cap ? want : cap), kRowThreads, 0, s>>>(static_cast<const T *>(a.x), a.pitch, a.rows, a.cols,
                                                                                 a.q, wide);
    } else {
      const uint64_t want = (uint64_t)across * down;
      const unsigned grid = (unsigned)(want < cap ? want : cap);
      if (a.square) tile_kernel<T, true><<<grid, kTileThreads, 0, s>>>(a, wide);
      else tile_kernel<T, false><<<grid, kTileThreads, 0, s>>>(a, wide);
    }
    return (int)cudaGetLastError();
  });
}

}  // namespace apc
