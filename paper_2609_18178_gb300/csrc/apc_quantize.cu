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
#include "apc_tcgen05.cuh"

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
// one, 8 elements a lane, kRowUnroll of them in flight.  Bound by memory and issue
// alike (68% of the slots).  Measured: 8192 x 4096 of bf16 21.6 us (4.7 TB/s), one row of
// 4096 2 us.
constexpr int kRowThreads = 256, kRowUnroll = 2;

template <typename T, bool E5M2>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(const T *x, int64_t pitch, uint32_t rows, uint32_t cols, QuantOut q,
                                                           bool wide) {
  constexpr int kWords = 8 / Word<T>::kPer;
  const uint32_t lane = threadIdx.x % 32, side = lane / 16, c8 = lane % 16 * 8;
  const uint32_t across = (cols + kBlock - 1) / kBlock;
  const uint64_t blocks = (uint64_t)across * rows, step = (uint64_t)gridDim.x * (kRowThreads / 32) * (2 * kRowUnroll);
  for (uint64_t b0 = ((uint64_t)blockIdx.x * (kRowThreads / 32) + threadIdx.x / 32) * (2 * kRowUnroll); b0 < blocks; b0 += step) {
    uint32_t w[kRowUnroll][kWords], row[kRowUnroll], bc[kRowUnroll];
    int n[kRowUnroll];
    uint64_t left = blocks - b0;
    uint32_t r = blocks >> 32 ? (uint32_t)((b0 + side) / across) : (uint32_t)(b0 + side) / across;
    uint32_t b = (uint32_t)(b0 + side - (uint64_t)r * across);
#pragma unroll
    for (int u = 0; u < kRowUnroll; ++u) {
      const uint32_t c = b * kBlock + c8;
      row[u] = r, bc[u] = b;
      n[u] = 2 * u + side < left && c < cols ? (int)min(8u, cols - c) : 0;
      load8<T>(w[u], x + (int64_t)r * pitch + c, n[u], wide);
      b += 2;
      while (b >= across) b -= across, ++r;
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
      if (awkward) {  // something is not finite
        m = 0;
        for (int i = 0; i < kWords; ++i) m = Word<T>::max(m, finite_abs<T>(w[u][i]));
        top = larger<T>(m);
        for (int o = 8; o; o >>= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
      }
      const uint32_t e = scale_exponent<E5M2>(bits_to_float<T>(top));
      const float inv = inverse_power(e);
      if (!n[u]) continue;
      if (c8 == 0) q.scale[(int64_t)bc[u] * q.scale_pitch + row[u]] = power(e);
      uint8_t *at = q.data + (int64_t)row[u] * q.pitch + bc[u] * kBlock + c8;
      if (!awkward) {
        uint64_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pack2(element<T>(w[u], 2 * i), element<T>(w[u], 2 * i + 1));
        store8(at, to_fp8x8<E5M2>(v, pack2(inv, inv)), n[u]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n[u]) at[i] = any_to_fp8<E5M2>(element<T>(w[u], i), inv);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Tiles of 128 x 128.  Thread (tx, ty) holds rows 8 ty + 0..7 of columns 8 tx +
// 0..7 in registers from one load to both stores.  Its maxima of rows and columns go
// to shared memory, where each row and each column is then one thread's: that
// thread stores the scale and leaves its inverse.  The transpose goes through
// shared memory in 8-byte pieces, swizzled so that neither side meets a bank twice.
constexpr int kTileThreads = 256;

struct TileShared {
  uint2 turn[128 * 16];
  uint32_t col[8][128];  // by warp: column maxima
  uint32_t row[128];
  float inv[2][128];     // rows', columns'
  uint32_t all[8];
};

// A tile that holds something not finite, element by element: seldom.
template <typename T, bool SQUARE, bool E5M2>
__device__ __noinline__ void awkward_tile(const QuantArgs &a, uint32_t tr, uint32_t tc, TileShared &sh) {
  const uint32_t r0 = tr * kBlock, c0 = tc * kBlock, t = threadIdx.x % 128, side = threadIdx.x / 128;
  const T *x = static_cast<const T *>(a.x) + (int64_t)r0 * a.pitch + c0;
  const uint32_t nr = min((uint32_t)kBlock, a.rows - r0), nc = min((uint32_t)kBlock, a.cols - c0);
  __syncthreads();
  float top = 0.0f;
  if (t < (side ? nc : nr))
    for (uint32_t i = 0; i < (side ? nr : nc); ++i) {
      const float v = fabsf(to_float(side ? x[(int64_t)i * a.pitch + t] : x[(int64_t)t * a.pitch + i]));
      if (v <= 3.402823466e38f) top = fmaxf(top, v);
    }
  sh.inv[side][t] = top;
  __syncthreads();
  if (SQUARE) {
    for (int i = 0; i < 128; ++i) top = fmaxf(top, sh.inv[0][i]);
    __syncthreads();
  }
  const uint32_t e = scale_exponent<E5M2>(top);
  sh.inv[side][t] = inverse_power(e);
  if (SQUARE ? t == 0 : t < (side ? nc : nr)) {
    if (side == 0) a.q.scale[(int64_t)tc * a.q.scale_pitch + (SQUARE ? tr : r0 + t)] = power(e);
    else if (a.qt.data) a.qt.scale[(int64_t)tr * a.qt.scale_pitch + (SQUARE ? tc : c0 + t)] = power(e);
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < kBlock * kBlock; i += kTileThreads) {
    const uint32_t r = i / kBlock, c = i % kBlock;
    if (r >= nr || c >= nc) continue;
    const float v = to_float(x[(int64_t)r * a.pitch + c]);
    a.q.data[(int64_t)(r0 + r) * a.q.pitch + c0 + c] = any_to_fp8<E5M2>(v, sh.inv[0][r]);
    if (a.qt.data) a.qt.data[(int64_t)(c0 + c) * a.qt.pitch + r0 + r] = any_to_fp8<E5M2>(v, sh.inv[1][c]);
  }
}

// A CTA walks tiles of 128 x 128, 8 x 8 elements a thread in registers.  The row and
// column maxima meet in shared memory, so that both outputs come from one read.
// Bound by memory and by issue (57% of the slots, 3 CTAs on an SM).  Measured: 8192 x
// 4096 of bf16, both ways, 29 us (4.6 TB/s: 13.5 tiles an SM, three at a time);
// 14336 x 4096 in square blocks, both ways, 42 us (5.5 TB/s).
template <typename T, bool SQUARE, bool E5M2>
__global__ void __launch_bounds__(kTileThreads, sizeof(T) == 4 ? 2 : 3) tile_kernel(const __grid_constant__ QuantArgs a, bool wide) {
  constexpr int kWords = 8 / Word<T>::kPer;  // words of 8 elements
  __shared__ __align__(16) TileShared sh;
  const uint32_t tx = threadIdx.x % 16, ty = threadIdx.x / 16, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t across = (a.cols + kBlock - 1) / kBlock, down = (a.rows + kBlock - 1) / kBlock;
  for (uint64_t t = blockIdx.x; t < (uint64_t)across * down; t += gridDim.x) {
    const uint32_t tr = (uint32_t)(t / across), tc = (uint32_t)(t % across), r0 = tr * kBlock, c0 = tc * kBlock;
    const uint32_t r = r0 + 8 * ty, c = c0 + 8 * tx;
    const int nc = c < a.cols ? (int)min(8u, a.cols - c) : 0;
    uint32_t w[8][kWords];
    {
      const T *x = static_cast<const T *>(a.x) + (int64_t)r * a.pitch + c;
#pragma unroll
      for (int i = 0; i < 8; ++i, x += a.pitch) load8<T>(w[i], x, r + i < a.rows ? nc : 0, wide);
    }
    uint32_t col[kWords], row[8], any = 0;
#pragma unroll
    for (int k = 0; k < kWords; ++k) col[k] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t m = 0;
#pragma unroll
      for (int k = 0; k < kWords; ++k) {
        const uint32_t v = w[i][k] & Word<T>::kAbs;
        col[k] = Word<T>::max(col[k], v);
        m = Word<T>::max(m, v);
      }
      row[i] = larger<T>(m);
      any = max(any, row[i]);
    }
    if (SQUARE) {
      any = __reduce_max_sync(~0u, any);
      if (lane == 0) sh.all[warp] = any;
    } else {
      // rows: each step halves the rows that a lane still holds and the lanes that hold them
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t keep = lane & 8 ? row[i + 4] : row[i], give = lane & 8 ? row[i] : row[i + 4];
        row[i] = max(keep, __shfl_xor_sync(~0u, give, 8));
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t keep = lane & 4 ? row[i + 2] : row[i], give = lane & 4 ? row[i] : row[i + 2];
        row[i] = max(keep, __shfl_xor_sync(~0u, give, 4));
      }
      const uint32_t keep = lane & 2 ? row[1] : row[0], give = lane & 2 ? row[0] : row[1];
      row[0] = max(keep, __shfl_xor_sync(~0u, give, 2));
      row[0] = max(row[0], __shfl_xor_sync(~0u, row[0], 1));
      if (!(lane & 1)) sh.row[8 * ty + (lane & 8 ? 4 : 0) + (lane & 4 ? 2 : 0) + (lane & 2 ? 1 : 0)] = row[0];
      // columns: two rows of threads a warp
#pragma unroll
      for (int k = 0; k < kWords; ++k) col[k] = Word<T>::max(col[k], __shfl_xor_sync(~0u, col[k], 16));
      if (lane < 16) {
#pragma unroll
        for (int k = 0; k < kWords; k += 4)
          *reinterpret_cast<uint4 *>(&sh.col[warp][tx * kWords + k]) = make_uint4(col[k], col[k + 1], col[k + 2], col[k + 3]);
      }
    }
    if (__syncthreads_or(any >= inf_bits<T>())) {
      awkward_tile<T, SQUARE, E5M2>(a, tr, tc, sh);
      __syncthreads();
      continue;
    }
    float inv = 0.0f;  // of a square block
    if (SQUARE) {
      uint32_t m = sh.all[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) m = max(m, sh.all[i]);
      const uint32_t e = scale_exponent<E5M2>(bits_to_float<T>(m));
      if (threadIdx.x == 0) {
        a.q.scale[(int64_t)tc * a.q.scale_pitch + tr] = power(e);
        if (a.qt.data) a.qt.scale[(int64_t)tr * a.qt.scale_pitch + tc] = power(e);
      }
      inv = inverse_power(e);
    } else {
      const uint32_t k = threadIdx.x % 128, side = threadIdx.x / 128;
      uint32_t m = 0;
      if (side) {
#pragma unroll
        for (int v = 0; v < 8; ++v) m = Word<T>::max(m, sh.col[v][k / Word<T>::kPer]);
        if (sizeof(T) == 2) m = k % 2 ? m >> 16 : m & 0xffffu;
      } else {
        m = sh.row[k];
      }
      const uint32_t e = scale_exponent<E5M2>(bits_to_float<T>(m));
      sh.inv[side][k] = inverse_power(e);
      if (side) {
        if (c0 + k < a.cols) a.qt.scale[(int64_t)tr * a.qt.scale_pitch + c0 + k] = power(e);
      } else {
        if (r0 + k < a.rows) a.q.scale[(int64_t)tc * a.q.scale_pitch + r0 + k] = power(e);
      }
      __syncthreads();
    }
    uint8_t *to = a.q.data + (int64_t)r * a.q.pitch + c;
#pragma unroll
    for (int i = 0; i < 8; ++i, to += a.q.pitch) {
      uint64_t v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = pack2(element<T>(w[i], 2 * j), element<T>(w[i], 2 * j + 1));
      const float scale = SQUARE ? inv : sh.inv[0][8 * ty + i];
      const uint2 y = to_fp8x8<E5M2>(v, pack2(scale, scale));
      if (r + i < a.rows && nc) store8(to, y, nc);
    }
    if (a.qt.data) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint64_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pack2(element<T>(w[2 * i], j), element<T>(w[2 * i + 1], j));
        const float scale = SQUARE ? inv : sh.inv[1][8 * tx + j];
        sh.turn[(8 * tx + j) * 16 + (ty ^ tx)] = to_fp8x8<E5M2>(v, pack2(scale, scale));
      }
      __syncthreads();
      const uint32_t rr = r0 + 8 * tx;  // now tx counts pieces down a column
      const int nr = rr < a.rows ? (int)min(8u, a.rows - rr) : 0;
      to = a.qt.data + (int64_t)(c0 + ty) * a.qt.pitch + rr;
#pragma unroll
      for (int i = 0; i < 8; ++i, to += 16 * a.qt.pitch) {
        const uint32_t k = 16 * i + ty;
        if (c0 + k < a.cols && nr) store8(to, sh.turn[k * 16 + (tx ^ k / 8)], nr);
      }
    }
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
    const auto rows = a.q.e5m2 ? rows_kernel<T, true> : rows_kernel<T, false>;
    const auto tiles = a.square ? a.q.e5m2 ? tile_kernel<T, true, true> : tile_kernel<T, true, false>
                                : a.q.e5m2 ? tile_kernel<T, false, true> : tile_kernel<T, false, false>;
    if (rows_alone(a)) {
      const uint64_t each = kRowThreads / 32 * 2 * kRowUnroll, want = ((uint64_t)across * a.rows + each - 1) / each;
      rows<<<(unsigned)(want < cap ? want : cap), kRowThreads, 0, s>>>(static_cast<const T *>(a.x), a.pitch, a.rows, a.cols, a.q, wide);
    } else {
      const uint64_t want = (uint64_t)across * down;
      tiles<<<(unsigned)(want < cap ? want : cap), kTileThreads, 0, s>>>(a, wide);
    }
    return (int)cudaGetLastError();
  });
}

}  // namespace apc
