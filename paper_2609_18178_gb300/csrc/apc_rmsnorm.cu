// The root-mean-square norm with the residual's addition (apc_rms_norm,
// apc_rms_norm_fp8) and its gradient (apc_rms_norm_grad).
//
//   h    = x + residual, rounded to x's type          (the residual stream)
//   rstd = 1 / sqrt(mean of h^2 + eps)
//   y    = (h * rstd) * weight, in fp32, then rounded or quantized
//
//   z  = h * rstd, g = dout * weight
//   dx = (g - z * mean of g*z) * rstd + dresidual,  dweight = sum over rows of dout * z
//
// One read of each input and one write of each output, a few operations for each
// element: bound by memory.
//
// A row is spread over the threads of a group, 8 elements each in one or two
// places, and stays in registers between its statistics and its output.
#include <cuda_runtime.h>

#include "apc_fp8.cuh"

namespace apc {

namespace {

// ---------------------------------------------------------------------------
// Eight elements of a row.  WIDE: neighbours, in 16-byte accesses.  Otherwise (rows
// at any boundary) every 32nd element, so that a warp's accesses stay dense.  n: how
// many of them exist, the first ones.

template <bool WIDE>
__device__ __forceinline__ uint32_t first_of(uint32_t group, uint32_t lane) { return group * 256 + (WIDE ? lane * 8 : lane); }

template <bool WIDE>
__device__ __forceinline__ int count_of(uint32_t first, uint32_t cols) {
  if (first >= cols) return 0;
  return (int)min(8u, WIDE ? cols - first : (cols - first + 31) / 32);
}

template <typename T, bool WIDE>
__device__ __forceinline__ void load(uint32_t (&w)[8 / Word<T>::kPer], const T *x, int n) {
  if (WIDE) {
    load8<T>(w, x, n, true);
  } else if (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = i < n ? reinterpret_cast<const uint32_t *>(x)[32 * i] : 0;
  } else {
    const uint16_t *h = reinterpret_cast<const uint16_t *>(x);
#pragma unroll
    for (int i = 0; i < 8 / Word<T>::kPer; ++i) {
      const uint32_t lo = 2 * i < n ? h[64 * i] : 0, hi = 2 * i + 1 < n ? h[64 * i + 32] : 0;
      w[i] = hi << 16 | lo;
    }
  }
}

template <typename T, bool WIDE>
__device__ __forceinline__ void store(T *x, const uint32_t (&w)[8 / Word<T>::kPer], int n) {
  if (WIDE && n == 8) {
#pragma unroll
    for (int i = 0; i < 8 / Word<T>::kPer; i += 4)
      *(reinterpret_cast<uint4 *>(x) + i / 4) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= n) continue;
      if (sizeof(T) == 4) reinterpret_cast<uint32_t *>(x)[WIDE ? i : 32 * i] = w[i];
      else reinterpret_cast<uint16_t *>(x)[WIDE ? i : 32 * i] = (uint16_t)element_bits<T>(w, i);
    }
  }
}

// Two values rounded to T, as they lie in its words.
template <typename T>
__device__ __forceinline__ void round_pair(uint32_t *w, int pair, float lo, float hi) {
  if (sizeof(T) == 4) {
    w[2 * pair] = __float_as_uint(lo);
    w[2 * pair + 1] = __float_as_uint(hi);
  } else {
    const T a = from_float<T>(lo), b = from_float<T>(hi);
    w[pair] = (uint32_t)*reinterpret_cast<const uint16_t *>(&b) << 16 | *reinterpret_cast<const uint16_t *>(&a);
  }
}
template <>
__device__ __forceinline__ void round_pair<__nv_bfloat16>(uint32_t *w, int pair, float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  w[pair] = *reinterpret_cast<const uint32_t *>(&v);
}
template <>
__device__ __forceinline__ void round_pair<__half>(uint32_t *w, int pair, float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  w[pair] = *reinterpret_cast<const uint32_t *>(&v);
}

// The weights of eight columns, of any type.
template <bool WIDE>
__device__ __forceinline__ void weights(uint64_t (&v)[4], const void *weight, uint32_t dtype, bool aligned, uint32_t first, int n) {
  float f[8];
  if (dtype == APC_F32) {
    const float *p = static_cast<const float *>(weight) + first;
    if (WIDE && aligned && n == 8) {
      const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
      f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = i < n ? __ldg(p + (WIDE ? i : 32 * i)) : 0.0f;
    }
  } else {
    const uint16_t *p = static_cast<const uint16_t *>(weight) + first;
    uint32_t w[4];
    if (WIDE && aligned && n == 8) {
      const uint4 a = __ldg(reinterpret_cast<const uint4 *>(p));
      w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = 2 * i < n ? __ldg(p + (WIDE ? 2 * i : 64 * i)) : 0;
        const uint32_t hi = 2 * i + 1 < n ? __ldg(p + (WIDE ? 2 * i + 1 : 64 * i + 32)) : 0;
        w[i] = hi << 16 | lo;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = dtype == APC_BF16 ? element<__nv_bfloat16>(w, i) : element<__half>(w, i);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack2(f[2 * i], f[2 * i + 1]);
}

// ---------------------------------------------------------------------------
// A row's sum of squares and its rstd.  Blocks are quantized by their largest value,
// so a last bit of rstd can turn a scale: it is rounded once from a sum that does not
// depend on how the row lies over the threads, up to the threads' own sums of 8 or 16
// squares.  Those are added as integers: of 26 bits under the largest of a warp, warps'
// sums with 20 bits more.  Integer additions across a warp are one instruction where
// five shuffles and additions of pairs of floats took 35.

struct Stat {
  uint32_t sum, e;  // sum * 2^(e - 152)
};
constexpr uint32_t kLeast = 32;  // least e: 2^-120 of the sum, far below eps

__device__ __forceinline__ Stat warp_stat(float p) {
  const uint32_t top = __reduce_max_sync(~0u, __float_as_uint(p) & 0x7fffffffu);
  const uint32_t e = max(top >> 23, kLeast);
  const uint32_t i = e == 255 ? 0 : __float2uint_rn(p * __uint_as_float((279 - e) << 23));
  return {__reduce_add_sync(~0u, i), e};
}

struct NormConst {
  float inv_hi, inv_lo, eps_hi, eps_lo;  // 1/cols and eps in two parts
};

// 1 / sqrt((hi + lo) * 2^k / cols + eps), rounded to nearest but for one in some 2^20.
__device__ __forceinline__ float rstd_of(float hi, float lo, int k, const NormConst &c, bool with_eps) {
  const float two_k = __uint_as_float((uint32_t)(k + 127) << 23);
  float m = hi * c.inv_hi, rest = __fmaf_rn(hi, c.inv_hi, -m);
  rest += hi * c.inv_lo + lo * c.inv_hi;
  m *= two_k, rest *= two_k;
  if (with_eps) {
    const float s = m + c.eps_hi, b = s - m;
    rest += ((m - (s - b)) + (c.eps_hi - b)) + c.eps_lo;
    m = s;
  }
  const float move = m > 0x1p60f ? 0x1p-80f : m < 0x1p-60f ? 0x1p80f : 1.0f;
  const float back = m > 0x1p60f ? 0x1p-40f : m < 0x1p-60f ? 0x1p40f : 1.0f;
  m *= move, rest *= move;
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(m));
  // a Newton step whose remainder 1 - (m + rest) y^2 is taken with y^2 in two parts
  const float a = y * y, low = __fmaf_rn(y, y, -a);
  const float r = __fmaf_rn(-m, a, 1.0f) - __fmaf_rn(m, low, rest * a);
  return __fmaf_rn(0.5f * y, r, y) * back;
}

__device__ __forceinline__ void split_sum(uint32_t s, float &hi, float &lo) {
  hi = (float)s;
  lo = (float)(int32_t)(s - __float2uint_rz(hi));
}

__device__ __forceinline__ void group_sync(uint32_t id, uint32_t threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// A group of threads that share a row.
struct Group {
  uint32_t warps, id, warp, lane;

  __device__ void sync() const {
    if (warps > 1) group_sync(id, warps * 32);
  }
};

// rstd of a row whose threads' sums of squares are p; false: a sum is not finite.
__device__ __forceinline__ bool row_rstd(float p, const Group &g, Stat *room, const NormConst &c, bool with_eps, float *rstd) {
  Stat s = warp_stat(p);
  float hi, lo;
  if (g.warps == 1) {
    if (s.e == 255) return false;
    split_sum(s.sum, hi, lo);
    *rstd = rstd_of(hi, lo, (int)s.e - 152, c, with_eps);
    return true;
  }
  if (g.lane == 0) room[g.warp] = s;
  g.sync();
  s = g.lane < g.warps ? room[g.lane] : Stat{0, kLeast};
  const uint32_t e = __reduce_max_sync(~0u, s.e);
  if (e == 255) return false;
  const uint32_t down = e - s.e;
  const uint64_t v = down < 64 ? ((uint64_t)s.sum << 20) >> down : 0;
  const uint32_t high = __reduce_add_sync(~0u, (uint32_t)(v >> 26)), low = __reduce_add_sync(~0u, (uint32_t)v & 0x3ffffffu);
  split_sum(high, hi, lo);
  lo += (float)low * 0x1p-26f;
  *rstd = rstd_of(hi, lo, (int)e - 146, c, with_eps);
  return true;
}

// The largest magnitude's bits over a group.
__device__ __forceinline__ uint32_t group_max(uint32_t m, const Group &g, Stat *room) {
  m = __reduce_max_sync(~0u, m);
  if (g.warps == 1) return m;
  g.sync();
  if (g.lane == 0) room[g.warp].sum = m;
  g.sync();
  m = __reduce_max_sync(~0u, g.lane < g.warps ? room[g.lane].sum : 0u);
  g.sync();
  return m;
}

template <typename T>
__device__ __forceinline__ float squares(const uint32_t (&w)[8 / Word<T>::kPer], float scale) {
  uint64_t acc[2] = {0, 0};
  const uint64_t both = pack2(scale, scale);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint64_t v = mul2(pack2(element<T>(w, 2 * i), element<T>(w, 2 * i + 1)), both);
    acc[i % 2] = fma2(v, v, acc[i % 2]);
  }
  const float2 a = unpack2(acc[0]), b = unpack2(acc[1]);
  return (a.x + a.y) + (b.x + b.y);
}

template <typename T>
__device__ __forceinline__ uint32_t largest(const uint32_t (&w)[8 / Word<T>::kPer]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(element<T>(w, i)) & 0x7fffffffu);
  return m;
}

// ---------------------------------------------------------------------------
// Forward.

constexpr int kSame = 0, kE4M3 = 1, kE5M2 = 2;  // what y becomes

struct ForwardArgs {
  const void *x, *residual, *weight;
  void *sum, *out;
  QuantOut q;
  float *rstd;
  int64_t pitch, residual_pitch, sum_pitch, out_pitch;
  uint32_t rows, cols, wdtype;
  uint32_t weight_aligned;
  NormConst c;
};

// Eight values of y to 8 bits; bits: their largest magnitude over the block of 128.
template <bool E5M2, bool WIDE>
__device__ __forceinline__ void quantize8(const ForwardArgs &a, uint32_t row, uint32_t first, int n, const uint64_t (&y)[4],
                                          uint32_t lane) {
  uint8_t *at = a.q.data + (int64_t)row * a.q.pitch + first;
  uint32_t m[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = unpack2(y[i]);
    m[2 * i] = __float_as_uint(v.x) & 0x7fffffffu, m[2 * i + 1] = __float_as_uint(v.y) & 0x7fffffffu;
  }
#pragma unroll
  for (int part = 0; part < (WIDE ? 1 : 2); ++part) {  // blocks: half a warp's 8 values each, or 4 of a whole warp's
    const int from = WIDE ? 0 : 4 * part, to = WIDE ? 8 : from + 4;
    uint32_t top = 0;
#pragma unroll
    for (int i = from; i < to; ++i) top = max(top, m[i]);
    const auto over_block = [&](uint32_t v) {
      if (!WIDE) return __reduce_max_sync(~0u, v);
#pragma unroll
      for (int o = 8; o; o >>= 1) v = max(v, __shfl_xor_sync(~0u, v, o));
      return v;
    };
    top = over_block(top);
    const bool awkward = __any_sync(~0u, top >= 0x7f800000u);
    if (awkward) {  // something is not finite
      top = 0;
#pragma unroll
      for (int i = from; i < to; ++i) top = max(top, m[i] < 0x7f800000u ? m[i] : 0u);
      top = over_block(top);
    }
    const uint32_t e = scale_exponent<E5M2>(__uint_as_float(top));
    const float inv = inverse_power(e);
    const int here = WIDE ? n : min(max(n - from, 0), 4);
    const uint32_t c = first + (WIDE ? 0 : 32 * from);
    if (c % kBlock == 0 && here > 0) a.q.scale[(int64_t)(c / kBlock) * a.q.scale_pitch + row] = power(e);
    if (WIDE && !awkward) {
      if (n) store8(at, to_fp8x8<E5M2>(y, pack2(inv, inv)), n);
    } else {
#pragma unroll
      for (int i = from; i < to; ++i) {
        const float2 v = unpack2(y[i / 2]);
        if (i < n) at[WIDE ? i : 32 * i] = any_to_fp8<E5M2>(i % 2 ? v.y : v.x, inv);
      }
    }
  }
}

// Threads (g, r): group r of the CTA takes a row, thread g of it V times 8 elements.
// LONG: a row has more than the group holds, and is read again for the output.
template <typename T, int OUT, int V, bool WIDE, bool LONG>
__global__ void __launch_bounds__(1024, 1) forward_kernel(const __grid_constant__ ForwardArgs a) {
  constexpr int kWords = 8 / Word<T>::kPer;
  extern __shared__ Stat s_room[];  // [2][groups][warps]
  const Group g{blockDim.x / 32, 1 + threadIdx.y, threadIdx.x / 32, threadIdx.x % 32};
  const uint32_t groups = (LONG ? (a.cols + 255) / 256 : V * g.warps);  // runs of 256 columns
  uint32_t turn = 0;
  for (uint64_t row = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y; row < a.rows; row += (uint64_t)gridDim.x * blockDim.y) {
    const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.pitch;
    const T *res = static_cast<const T *>(a.residual) + (int64_t)row * a.residual_pitch;
    T *sum = static_cast<T *>(a.sum) + (int64_t)row * a.sum_pitch;
    Stat *room = s_room + (turn ^= 1) * blockDim.y * g.warps + threadIdx.y * g.warps;
    uint32_t w[V][kWords];
    // the sum's elements of V runs from `run` on, as they are stored
    const auto fetch = [&](uint32_t run, bool again) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const uint32_t c = first_of<WIDE>(run + v * g.warps, g.lane);
        const int n = count_of<WIDE>(c, a.cols);
        if (again && a.residual) {
          load<T, WIDE>(w[v], const_cast<const T *>(sum) + c, 0);
          if (n) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              if (i >= n) continue;
              const uint32_t at = c + (WIDE ? i : 32 * i);
              if (sizeof(T) == 4) w[v][i] = reinterpret_cast<volatile uint32_t *>(sum)[at];
              else w[v][i / 2] |= (uint32_t)reinterpret_cast<volatile uint16_t *>(sum)[at] << (i % 2 * 16);
            }
          }
          continue;
        }
        load<T, WIDE>(w[v], x + c, n);
        if (a.residual) {
          uint32_t o[kWords];
          load<T, WIDE>(o, res + c, n);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            round_pair<T>(w[v], i, element<T>(w[v], 2 * i) + element<T>(o, 2 * i), element<T>(w[v], 2 * i + 1) + element<T>(o, 2 * i + 1));
          store<T, WIDE>(sum + c, w[v], n);
        }
      }
    };
    const auto over_row = [&](bool again, auto f) {  // f() for each part that the registers hold
      if (!LONG) return f(0u);
      for (uint32_t run = 0; run < groups; run += V * g.warps) {
        fetch(run + g.warp, again);
        f(run);
      }
    };
    if (!LONG) fetch(g.warp, false);
    float p = 0.0f, rstd;
    over_row(false, [&](uint32_t) {
#pragma unroll
      for (int v = 0; v < V; ++v) p += squares<T>(w[v], 1.0f);
    });
    if (!row_rstd(p, g, room, a.c, true, &rstd)) {
      uint32_t m = 0;
      over_row(true, [&](uint32_t) {
#pragma unroll
        for (int v = 0; v < V; ++v) m = max(m, largest<T>(w[v]));
      });
      m = group_max(m, g, room);
      if (m >= 0x7f800000u) {
        rstd = m > 0x7f800000u ? __uint_as_float(0x7fffffffu) : 0.0f;
      } else {  // squares beyond the largest number: eps is nothing beside them
        const float scale = __uint_as_float(max(254u - (m >> 23), 1u) << 23);
        p = 0.0f;
        over_row(true, [&](uint32_t) {
#pragma unroll
          for (int v = 0; v < V; ++v) p += squares<T>(w[v], scale);
        });
        row_rstd(p, g, room, a.c, false, &rstd);
        rstd *= scale;
        g.sync();
      }
    }
    if (threadIdx.x == 0) a.rstd[row] = rstd;
    over_row(true, [&](uint32_t run) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const uint32_t c = first_of<WIDE>(run + g.warp + v * g.warps, g.lane);
        const int n = count_of<WIDE>(c, a.cols);
        uint64_t wt[4], y[4];
        weights<WIDE>(wt, a.weight, a.wdtype, a.weight_aligned, c, n);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = mul2(mul2(pack2(element<T>(w[v], 2 * i), element<T>(w[v], 2 * i + 1)), pack2(rstd, rstd)), wt[i]);
        if (OUT == kSame) {
          uint32_t o[kWords];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2(y[i]);
            round_pair<T>(o, i, f.x, f.y);
          }
          store<T, WIDE>(static_cast<T *>(a.out) + (int64_t)row * a.out_pitch + c, o, n);
        } else {
          if (n < 8)
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // what is not there: no NaN of 0 times an infinity
              const float2 f = unpack2(y[i]);
              y[i] = pack2(2 * i < n ? f.x : 0.0f, 2 * i + 1 < n ? f.y : 0.0f);
            }
          quantize8<OUT == kE5M2, WIDE>(a, (uint32_t)row, c, n, y, g.lane);
        }
      }
    });
  }
}

// The transpose in 8 bits, from the sum and rstd that the forward kernel left.  A CTA walks
// tiles of 128 x 128, as the quantization's tile kernel does: thread (tx, ty) holds rows 8
// ty + 0..7 of columns 8 tx + 0..7.
struct TurnArgs {
  const void *h, *weight;
  const float *rstd;
  QuantOut qt;
  int64_t pitch;
  uint32_t rows, cols, wdtype, weight_aligned, wide;
};

struct TurnShared {
  uint2 turn[128 * 16];
  uint32_t col[8][128];
  float inv[128], rstd[128];
};

template <typename T, bool E5M2>
__global__ void __launch_bounds__(256, 2) turn_kernel(const __grid_constant__ TurnArgs a) {
  constexpr int kWords = 8 / Word<T>::kPer;
  __shared__ __align__(16) TurnShared sh;
  const uint32_t tx = threadIdx.x % 16, ty = threadIdx.x / 16, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t across = (a.cols + kBlock - 1) / kBlock, down = (a.rows + kBlock - 1) / kBlock;
  for (uint64_t t = blockIdx.x; t < (uint64_t)across * down; t += gridDim.x) {
    const uint32_t tr = (uint32_t)(t / across), tc = (uint32_t)(t % across), r0 = tr * kBlock, c0 = tc * kBlock;
    const uint32_t r = r0 + 8 * ty, c = c0 + 8 * tx;
    const int nc = c < a.cols ? (int)min(8u, a.cols - c) : 0;
    uint32_t w[8][kWords];
    {
      const T *h = static_cast<const T *>(a.h) + (int64_t)r * a.pitch + c;
#pragma unroll
      for (int i = 0; i < 8; ++i, h += a.pitch) load8<T>(w[i], h, r + i < a.rows ? nc : 0, a.wide);
    }
    uint64_t wt[4];
    weights<true>(wt, a.weight, a.wdtype, a.weight_aligned, c, nc);
    if (threadIdx.x < 128) sh.rstd[threadIdx.x] = r0 + threadIdx.x < a.rows ? __ldg(a.rstd + r0 + threadIdx.x) : 0.0f;
    __syncthreads();
    const auto value = [&](int i, int j) {  // columns 2j and 2j + 1 of row i
      const float s = sh.rstd[8 * ty + i];
      return mul2(mul2(pack2(element<T>(w[i], 2 * j), element<T>(w[i], 2 * j + 1)), pack2(s, s)), wt[j]);
    };
    uint32_t col[8], any = 0;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t lo = 0, hi = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (r + i >= a.rows) continue;
          const uint64_t y = value(i, j);
          uint32_t u = (uint32_t)y & 0x7fffffffu, v = (uint32_t)(y >> 32) & 0x7fffffffu;
          if (pass) u = u < 0x7f800000u ? u : 0, v = v < 0x7f800000u ? v : 0;
          lo = max(lo, u), hi = max(hi, v);
        }
        col[2 * j] = lo, col[2 * j + 1] = hi;
      }
      if (pass == 0) {
        any = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) any = max(any, j < nc ? col[j] : 0u);
        any = __syncthreads_or(any >= 0x7f800000u);
        if (!any) break;
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) col[j] = max(col[j], __shfl_xor_sync(~0u, col[j], 16));
    if (lane < 16) {
      *reinterpret_cast<uint4 *>(&sh.col[warp][tx * 8]) = make_uint4(col[0], col[1], col[2], col[3]);
      *reinterpret_cast<uint4 *>(&sh.col[warp][tx * 8 + 4]) = make_uint4(col[4], col[5], col[6], col[7]);
    }
    __syncthreads();
    if (threadIdx.x < 128) {
      uint32_t m = 0;
#pragma unroll
      for (int v = 0; v < 8; ++v) m = max(m, sh.col[v][threadIdx.x]);
      const uint32_t e = scale_exponent<E5M2>(__uint_as_float(m));
      sh.inv[threadIdx.x] = inverse_power(e);
      if (c0 + threadIdx.x < a.cols) a.qt.scale[(int64_t)tr * a.qt.scale_pitch + c0 + threadIdx.x] = power(e);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint64_t lo[4], hi[4];  // pairs of rows, of columns 2j and 2j + 1
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 p = unpack2(value(2 * i, j)), q = unpack2(value(2 * i + 1, j));
        lo[i] = pack2(p.x, q.x), hi[i] = pack2(p.y, q.y);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint64_t(&v)[4] = k ? hi : lo;
        const float inv = sh.inv[8 * tx + 2 * j + k];
        uint2 o;
        if (!any) {
          o = to_fp8x8<E5M2>(v, pack2(inv, inv));
        } else {
          uint32_t b[2] = {0, 0};
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float2 f = unpack2(v[i / 2]);
            b[i / 4] |= (uint32_t)any_to_fp8<E5M2>(i % 2 ? f.y : f.x, inv) << (i % 4 * 8);
          }
          o = make_uint2(b[0], b[1]);
        }
        sh.turn[(8 * tx + 2 * j + k) * 16 + (ty ^ tx)] = o;
      }
    }
    __syncthreads();
    const uint32_t rr = r0 + 8 * tx;  // now tx counts pieces down a column
    const int nr = rr < a.rows ? (int)min(8u, a.rows - rr) : 0;
    uint8_t *to = a.qt.data + (int64_t)(c0 + ty) * a.qt.pitch + rr;
#pragma unroll
    for (int i = 0; i < 8; ++i, to += 16 * a.qt.pitch) {
      const uint32_t k = 16 * i + ty;
      if (c0 + k < a.cols && nr) store8(to, sh.turn[k * 16 + (tx ^ k / 8)], nr);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Gradient.  The rows are cut into `parts` runs whose number follows the sizes alone
// (rms_norm_parts); a group walks a run and keeps its columns' sums of dout * z in
// registers, which go to the workspace, from where a second kernel adds them in order.

struct GradArgs {
  const void *dout, *x, *weight, *dresidual;
  const float *rstd;
  void *dx;
  float *partial;  // [parts][cols]; null: no dweight
  int64_t dout_pitch, pitch, dresidual_pitch, dx_pitch;
  uint32_t rows, cols, parts, wdtype, weight_aligned;
  float inv_cols;
};

__device__ __forceinline__ uint32_t part_begin(uint32_t rows, uint32_t parts, uint32_t p) {
  return (uint32_t)((uint64_t)rows * p / parts);
}

// The sum of p over a group, in an order of its own, in every thread.
__device__ __forceinline__ float group_sum(float p, const Group &g, float *room) {
#pragma unroll
  for (int o = 16; o; o >>= 1) p += __shfl_xor_sync(~0u, p, o);
  if (g.warps == 1) return p;
  if (g.lane == 0) room[g.warp] = p;
  g.sync();
  p = g.lane < g.warps ? room[g.lane] : 0.0f;
#pragma unroll
  for (int o = 16; o; o >>= 1) p += __shfl_xor_sync(~0u, p, o);
  return p;
}

// One run of 8 columns a thread: z and g = dout * weight of a row.
template <typename T>
__device__ __forceinline__ void z_and_g(const uint32_t (&x)[8 / Word<T>::kPer], const uint32_t (&d)[8 / Word<T>::kPer], float rstd,
                                        const uint64_t (&wt)[4], int i, uint64_t *z, uint64_t *g, uint64_t *dd) {
  *dd = pack2(element<T>(d, 2 * i), element<T>(d, 2 * i + 1));
  *z = mul2(pack2(element<T>(x, 2 * i), element<T>(x, 2 * i + 1)), pack2(rstd, rstd));
  *g = mul2(*dd, wt[i]);
}

template <typename T, int V, bool WIDE>
__global__ void __launch_bounds__(1024, 1) grad_kernel(const __grid_constant__ GradArgs a) {
  constexpr int kWords = 8 / Word<T>::kPer;
  extern __shared__ float s_sums[];  // [2][groups][warps]
  const Group g{blockDim.x / 32, 1 + threadIdx.y, threadIdx.x / 32, threadIdx.x % 32};
  uint32_t turn = 0;
  uint32_t c[V];
  int n[V];
  uint64_t wt[V][4];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    c[v] = first_of<WIDE>(g.warp + v * g.warps, g.lane);
    n[v] = count_of<WIDE>(c[v], a.cols);
    weights<WIDE>(wt[v], a.weight, a.wdtype, a.weight_aligned, c[v], n[v]);
  }
  for (uint32_t part = blockIdx.x * blockDim.y + threadIdx.y; part < a.parts; part += gridDim.x * blockDim.y) {
    uint64_t acc[V][4] = {};
    const uint32_t end = part_begin(a.rows, a.parts, part + 1);
    for (uint32_t row = part_begin(a.rows, a.parts, part); row < end; ++row) {
      float *room = s_sums + (turn ^= 1) * blockDim.y * g.warps + threadIdx.y * g.warps;
      const float rstd = __ldg(a.rstd + row);
      uint32_t x[V][kWords], d[V][kWords], r[V][kWords];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        load<T, WIDE>(x[v], static_cast<const T *>(a.x) + (int64_t)row * a.pitch + c[v], n[v]);
        load<T, WIDE>(d[v], static_cast<const T *>(a.dout) + (int64_t)row * a.dout_pitch + c[v], n[v]);
        if (a.dresidual) load<T, WIDE>(r[v], static_cast<const T *>(a.dresidual) + (int64_t)row * a.dresidual_pitch + c[v], n[v]);
      }
      uint64_t dot = 0;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint64_t z, gg, dd;
          z_and_g<T>(x[v], d[v], rstd, wt[v], i, &z, &gg, &dd);
          dot = fma2(gg, z, dot);
          acc[v][i] = fma2(dd, z, acc[v][i]);
        }
      const float2 both = unpack2(dot);
      const float mean = group_sum(both.x + both.y, g, room) * a.inv_cols;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        uint32_t o[kWords];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint64_t z, gg, dd;
          z_and_g<T>(x[v], d[v], rstd, wt[v], i, &z, &gg, &dd);
          uint64_t y = mul2(fma2(z, pack2(-mean, -mean), gg), pack2(rstd, rstd));
          float2 f = unpack2(y);
          if (a.dresidual) f.x += element<T>(r[v], 2 * i), f.y += element<T>(r[v], 2 * i + 1);
          round_pair<T>(o, i, f.x, f.y);
        }
        store<T, WIDE>(static_cast<T *>(a.dx) + (int64_t)row * a.dx_pitch + c[v], o, n[v]);
      }
    }
    if (!a.partial) continue;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float *to = a.partial + (uint64_t)part * a.cols + c[v];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 f = unpack2(acc[v][i / 2]);
        if (i < n[v]) to[WIDE ? i : 32 * i] = i % 2 ? f.y : f.x;
      }
    }
  }
}

// Rows that a group does not hold: twice over each, element by element.
template <typename T>
__global__ void __launch_bounds__(1024, 1) grad_long_kernel(const __grid_constant__ GradArgs a) {
  __shared__ float room[2][32];
  const Group g{32, 0, threadIdx.x / 32, threadIdx.x % 32};
  uint32_t turn = 0;
  const auto weight = [&](uint32_t c) {
    return a.wdtype == APC_F32    ? __ldg(static_cast<const float *>(a.weight) + c)
           : a.wdtype == APC_BF16 ? to_float(static_cast<const __nv_bfloat16 *>(a.weight)[c])
                                  : to_float(static_cast<const __half *>(a.weight)[c]);
  };
  for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.pitch, *d = static_cast<const T *>(a.dout) + (int64_t)row * a.dout_pitch;
    const T *r = static_cast<const T *>(a.dresidual) + (int64_t)row * a.dresidual_pitch;
    T *dx = static_cast<T *>(a.dx) + (int64_t)row * a.dx_pitch;
    const float rstd = __ldg(a.rstd + row);
    float dot = 0.0f;
    for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) dot = __fmaf_rn(to_float(d[c]) * weight(c), to_float(x[c]) * rstd, dot);
    const float mean = group_sum(dot, g, room[turn ^= 1]) * a.inv_cols;
    for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) {
      float y = __fmaf_rn(to_float(x[c]) * rstd, -mean, to_float(d[c]) * weight(c)) * rstd;
      if (a.dresidual) y += to_float(r[c]);
      dx[c] = from_float<T>(y);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) grad_long_parts_kernel(const __grid_constant__ GradArgs a) {
  const uint64_t per = (a.cols + 255) / 256;
  for (uint64_t t = blockIdx.x; t < per * a.parts; t += gridDim.x) {
    const uint32_t part = (uint32_t)(t / per), c = (uint32_t)(t % per) * 256 + threadIdx.x, end = part_begin(a.rows, a.parts, part + 1);
    if (c >= a.cols) continue;
    float acc = 0.0f;
    for (uint32_t row = part_begin(a.rows, a.parts, part); row < end; ++row)
      acc = __fmaf_rn(to_float(static_cast<const T *>(a.dout)[(int64_t)row * a.dout_pitch + c]),
                      to_float(static_cast<const T *>(a.x)[(int64_t)row * a.pitch + c]) * __ldg(a.rstd + row), acc);
    a.partial[(uint64_t)part * a.cols + c] = acc;
  }
}

// dweight: the parts' sums, warp k of a CTA those of parts k, k + 8, ..., then the warps'.
__global__ void __launch_bounds__(256) parts_kernel(const float *partial, uint32_t parts, uint32_t cols, void *dweight, uint32_t dtype) {
  __shared__ float sums[8][32];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint32_t runs = (cols + 31) / 32;
  for (uint32_t run = blockIdx.x; run < runs; run += gridDim.x) {
    const uint32_t c = run * 32 + lane;
    float s = 0.0f;
    if (c < cols)
      for (uint32_t p = warp; p < parts; p += 8) s += __ldcg(partial + (uint64_t)p * cols + c);
    __syncthreads();
    sums[warp][lane] = s;
    __syncthreads();
    if (warp || c >= cols) continue;
    const float y = ((sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane])) +
                    ((sums[4][lane] + sums[5][lane]) + (sums[6][lane] + sums[7][lane]));
    if (dtype == APC_F32) static_cast<float *>(dweight)[c] = y;
    else if (dtype == APC_BF16) static_cast<__nv_bfloat16 *>(dweight)[c] = from_float<__nv_bfloat16>(y);
    else static_cast<__half *>(dweight)[c] = from_float<__half>(y);
  }
}

// ---------------------------------------------------------------------------
// How a row lies over threads.

struct Shape {
  uint32_t threads, groups;  // threads of a group, groups of a CTA
  int v;                     // times 8 elements a thread
  bool fits;                 // a group holds the row
};

Shape shape_of(uint32_t cols, bool few) {
  Shape s;
  s.v = few && cols <= 8192 ? 1 : 2;
  const uint32_t per = 256 * s.v, warps = (cols + per - 1) / per;
  s.fits = warps <= 32;
  s.threads = 32 * (s.fits ? warps : 32);
  s.groups = s.threads >= 256 ? 1 : 256 / s.threads;
  return s;
}

// CTAs for so much work, `per_sm` of them on an SM.
unsigned grid_of(uint64_t want, uint32_t per_sm) {
  unsigned cap = 1;
  op_grid((int)per_sm, &cap);
  return (unsigned)(want < cap ? want : cap);
}

bool aligned(const void *p, int64_t pitch_bytes) { return (uintptr_t)p % 16 == 0 && pitch_bytes % 16 == 0; }

template <typename T, int OUT, int V, bool WIDE, bool LONG>
int forward_launch(const ForwardArgs &a, const Shape &s, void *stream) {
  const uint32_t per = s.threads * s.groups;
  const unsigned grid = grid_of((a.rows + s.groups - 1) / s.groups, 2048 / per);
  const size_t room = sizeof(Stat) * 2 * per / 32;
  forward_kernel<T, OUT, V, WIDE, LONG><<<grid, dim3(s.threads, s.groups), room, (cudaStream_t)stream>>>(a);
  return (int)cudaGetLastError();
}

template <typename T, int OUT>
int forward(const ForwardArgs &a, const Shape &s, bool wide, void *stream) {
  if (!s.fits) return wide ? forward_launch<T, OUT, 2, true, true>(a, s, stream) : forward_launch<T, OUT, 2, false, true>(a, s, stream);
  if (s.v == 1) return wide ? forward_launch<T, OUT, 1, true, false>(a, s, stream) : forward_launch<T, OUT, 1, false, false>(a, s, stream);
  return wide ? forward_launch<T, OUT, 2, true, false>(a, s, stream) : forward_launch<T, OUT, 2, false, false>(a, s, stream);
}

void two_parts(double v, float *hi, float *lo) {
  *hi = (float)v;
  *lo = (float)(v - (double)*hi);
}

}  // namespace

int launch_rms_norm(const NormArgs &n, unsigned sms, void *stream) {
  ForwardArgs a = {};
  a.x = n.x, a.residual = n.residual, a.weight = n.weight, a.sum = n.sum, a.out = n.out;
  a.q = n.q;
  a.rstd = n.rstd;
  a.pitch = n.pitch, a.residual_pitch = n.residual_pitch, a.sum_pitch = n.sum_pitch, a.out_pitch = n.out_pitch;
  a.rows = n.rows, a.cols = n.cols, a.wdtype = n.wdtype;
  a.weight_aligned = (uintptr_t)n.weight % 16 == 0;
  two_parts(1.0 / n.cols, &a.c.inv_hi, &a.c.inv_lo);
  two_parts(n.eps, &a.c.eps_hi, &a.c.eps_lo);
  const Shape s = shape_of(n.cols, n.rows <= sms);
  return with_dtype(n.dtype, [&](auto t) {
    using T = decltype(t);
    const auto at = [](const void *p, int64_t pitch) { return aligned(p, pitch * (int64_t)sizeof(T)); };
    const bool wide = at(n.x, n.pitch) && at(n.residual, n.residual_pitch) && at(n.sum, n.sum_pitch) && at(n.out, n.out_pitch);
    int e;
    if (n.out) e = forward<T, kSame>(a, s, wide, stream);
    else e = n.q.e5m2 ? forward<T, kE5M2>(a, s, wide, stream) : forward<T, kE4M3>(a, s, wide, stream);
    if (e || !n.qt.data) return e;
    TurnArgs r = {};
    r.h = n.residual ? n.sum : n.x, r.weight = n.weight, r.rstd = n.rstd;
    r.qt = n.qt;
    r.pitch = n.residual ? n.sum_pitch : n.pitch;
    r.rows = n.rows, r.cols = n.cols, r.wdtype = n.wdtype;
    r.weight_aligned = a.weight_aligned;
    r.wide = at(r.h, r.pitch);
    const unsigned grid = grid_of((uint64_t)((n.cols + kBlock - 1) / kBlock) * ((n.rows + kBlock - 1) / kBlock), 2);
    if (n.qt.e5m2) turn_kernel<T, true><<<grid, 256, 0, (cudaStream_t)stream>>>(r);
    else turn_kernel<T, false><<<grid, 256, 0, (cudaStream_t)stream>>>(r);
    return (int)cudaGetLastError();
  });
}

// Enough runs for every SM, more of them where a group is small.
uint32_t rms_norm_parts(uint32_t rows, uint32_t cols) {
  const uint32_t parts = 304 * (cols <= 512 ? 8 : cols <= 1024 ? 4 : cols <= 2048 ? 2 : 1);
  return rows < parts ? rows : parts;
}

int launch_rms_norm_grad(const NormGradArgs &n, void *stream) {
  GradArgs a = {};
  a.dout = n.dout, a.x = n.x, a.weight = n.weight, a.dresidual = n.dresidual, a.rstd = n.rstd, a.dx = n.dx;
  a.partial = n.dweight ? n.work : nullptr;
  a.dout_pitch = n.dout_pitch, a.pitch = n.pitch, a.dresidual_pitch = n.dresidual_pitch, a.dx_pitch = n.dx_pitch;
  a.rows = n.rows, a.cols = n.cols, a.wdtype = n.wdtype;
  a.parts = rms_norm_parts(n.rows, n.cols);
  a.weight_aligned = (uintptr_t)n.weight % 16 == 0;
  a.inv_cols = (float)(1.0 / n.cols);
  cudaStream_t s = (cudaStream_t)stream;
  const Shape sh = shape_of(n.cols, false);
  const int e = !n.rows ? 0 : with_dtype(n.dtype, [&](auto t) {
    using T = decltype(t);
    const auto at = [](const void *p, int64_t pitch) { return aligned(p, pitch * (int64_t)sizeof(T)); };
    if (!sh.fits) {
      grad_long_kernel<T><<<grid_of(n.rows, 1), 1024, 0, s>>>(a);
      if (a.partial) grad_long_parts_kernel<T><<<grid_of((uint64_t)((n.cols + 255) / 256) * a.parts, 8), 256, 0, s>>>(a);
      return (int)cudaGetLastError();
    }
    const bool wide = at(n.x, n.pitch) && at(n.dout, n.dout_pitch) && at(n.dresidual, n.dresidual_pitch) && at(n.dx, n.dx_pitch);
    const uint32_t per = sh.threads * sh.groups;
    const unsigned grid = grid_of((a.parts + sh.groups - 1) / sh.groups, 1024 / per);
    const size_t room = sizeof(float) * 2 * per / 32;
    if (wide) grad_kernel<T, 2, true><<<grid, dim3(sh.threads, sh.groups), room, s>>>(a);
    else grad_kernel<T, 2, false><<<grid, dim3(sh.threads, sh.groups), room, s>>>(a);
    return (int)cudaGetLastError();
  });
  if (e || !n.dweight) return e;
  parts_kernel<<<grid_of((n.cols + 31) / 32, 8), 256, 0, s>>>(n.work, a.parts, n.cols, n.dweight, n.dwdtype);
  return (int)cudaGetLastError();
}

}  // namespace apc
