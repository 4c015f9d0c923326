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

#include "apc_cluster.cuh"
#include "apc_fp8.cuh"

namespace apc {

namespace {

// A call's second kernel may start while its first one drains (launch_after), and waits
// for it to have completed before it does anything.
__device__ __forceinline__ void start_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_first() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... P, typename... A>
int launch_after(void (*kernel)(P...), unsigned grid, unsigned threads, uint32_t bytes, void *stream, const A &...args) {
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return (int)cudaLaunchKernelEx(&cfg, kernel, args...);
}

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

// w + x, rounded to T.  The packed 16-bit addition rounds once, and so does one in fp32
// that is rounded again: a sum that 24 bits do not hold has a term below half a last place
// of the other.
template <typename T>
__device__ __forceinline__ void add_rounded(uint32_t (&w)[8 / Word<T>::kPer], const uint32_t (&x)[8 / Word<T>::kPer]) {
#pragma unroll
  for (int i = 0; i < 8 / Word<T>::kPer; ++i) {
    if (sizeof(T) == 4) {
      w[i] = __float_as_uint(__uint_as_float(w[i]) + __uint_as_float(x[i]));
    } else if (inf_bits<T>() == 0x7f80u) {
      asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(w[i]) : "r"(x[i]));
    } else {
      asm("add.rn.f16x2 %0, %0, %1;" : "+r"(w[i]) : "r"(x[i]));
    }
  }
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

// The squares of eight elements, each times `scale`.
template <typename T, bool SCALED = false>
__device__ __forceinline__ float squares(const uint32_t (&w)[8 / Word<T>::kPer], float scale = 1.0f) {
  uint64_t acc[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint64_t v = pack2(element<T>(w, 2 * i), element<T>(w, 2 * i + 1));
    if (SCALED) v = mul2(v, pack2(scale, scale));
    acc[i % 2] = i < 2 ? mul2(v, v) : fma2(v, v, acc[i % 2]);
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

// rstd of a row some of whose threads' sums are not finite: infinities and NaNs, or
// squares beyond the largest number, which are taken scaled (eps is nothing beside them).
template <typename T, int V>
__device__ __forceinline__ float wild_rstd(const uint32_t (&w)[V][8 / Word<T>::kPer], const Group &g, Stat *room, const NormConst &c) {
  uint32_t m = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) m = max(m, largest<T>(w[v]));
  m = group_max(m, g, room);
  if (m >= 0x7f800000u) return m > 0x7f800000u ? __uint_as_float(0x7fffffffu) : 0.0f;
  const float scale = __uint_as_float(max(254u - (m >> 23), 1u) << 23);
  float p = 0.0f, rstd;
#pragma unroll
  for (int v = 0; v < V; ++v) p += squares<T, true>(w[v], scale);
  row_rstd(p, g, room, c, false, &rstd);
  g.sync();
  return rstd * scale;
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
  uint32_t then;  // the transpose's kernel follows
  NormConst c;
};

// The largest magnitude of three values, a NaN's bits above all.
__device__ __forceinline__ float max_abs(float a, float b, float c) {
  float y;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// Eight values of y to 8 bits; bits: their largest magnitude over the block of 128.
template <bool E5M2, bool WIDE>
__device__ __forceinline__ void quantize8(const ForwardArgs &a, uint32_t row, uint32_t first, int n, const uint64_t (&y)[4],
                                          uint32_t lane) {
  uint8_t *at = a.q.data + (int64_t)row * a.q.pitch + first;
  const auto value = [&](int i) {
    const float2 v = unpack2(y[i / 2]);
    return i % 2 ? v.y : v.x;
  };
#pragma unroll
  for (int part = 0; part < (WIDE ? 1 : 2); ++part) {  // blocks: half a warp's 8 values each, or 4 of a whole warp's
    const int from = WIDE ? 0 : 4 * part, to = WIDE ? 8 : from + 4;
    float high = 0.0f;
#pragma unroll
    for (int i = from; i < to; i += 2) high = max_abs(high, value(i), value(i + 1));
    uint32_t top = __float_as_uint(high);
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
      for (int i = from; i < to; ++i) {
        const uint32_t m = __float_as_uint(value(i)) & 0x7fffffffu;
        top = max(top, m < 0x7f800000u ? m : 0u);
      }
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
        if (i < n) at[WIDE ? i : 32 * i] = any_to_fp8<E5M2>(value(i), inv);
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
  if (a.then) start_next();
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
          add_rounded<T>(w[v], o);
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
      for (int v = 0; v < V; ++v) p += squares<T>(w[v]);
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
          for (int v = 0; v < V; ++v) p += squares<T, true>(w[v], scale);
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

// Many rows that a warp holds: U rows at a time, so that one's latencies lie beside the others'
// (16384 x 128: 10.4 us a row at a time).
template <typename T, int OUT, int V, int U, bool WIDE>
__global__ void __launch_bounds__(256) narrow_kernel(const __grid_constant__ ForwardArgs a) {
  constexpr int kWords = 8 / Word<T>::kPer;
  const Group g{1, 0, 0, threadIdx.x % 32};
  const uint64_t step = (uint64_t)gridDim.x * (blockDim.x / 32) * U;
  if (a.then) start_next();
  uint32_t c[V];
  int n[V];
  uint64_t wt[V][4];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    c[v] = first_of<WIDE>(v, g.lane);
    n[v] = count_of<WIDE>(c[v], a.cols);
    weights<WIDE>(wt[v], a.weight, a.wdtype, a.weight_aligned, c[v], n[v]);
  }
  for (uint64_t first = ((uint64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32) * U; first < a.rows; first += step) {
    uint32_t w[U][V][kWords];
    float rstd[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool there = first + u < a.rows;
#pragma unroll
      for (int v = 0; v < V; ++v)
        load<T, WIDE>(w[u][v], static_cast<const T *>(a.x) + (int64_t)(first + u) * a.pitch + c[v], there ? n[v] : 0);
    }
    if (a.residual) {
      uint32_t o[U][V][kWords];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool there = first + u < a.rows;
#pragma unroll
        for (int v = 0; v < V; ++v)
          load<T, WIDE>(o[u][v], static_cast<const T *>(a.residual) + (int64_t)(first + u) * a.residual_pitch + c[v], there ? n[v] : 0);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool there = first + u < a.rows;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          add_rounded<T>(w[u][v], o[u][v]);
          store<T, WIDE>(static_cast<T *>(a.sum) + (int64_t)(first + u) * a.sum_pitch + c[v], w[u][v], there ? n[v] : 0);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float p = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) p += squares<T>(w[u][v]);
      if (!row_rstd(p, g, nullptr, a.c, true, &rstd[u])) rstd[u] = wild_rstd<T, V>(w[u], g, nullptr, a.c);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (first + u >= a.rows) break;
      const uint32_t row = (uint32_t)first + u;
      if (g.lane == 0) a.rstd[row] = rstd[u];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        uint64_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          y[i] = mul2(mul2(pack2(element<T>(w[u][v], 2 * i), element<T>(w[u][v], 2 * i + 1)), pack2(rstd[u], rstd[u])), wt[v][i]);
        if (OUT == kSame) {
          uint32_t o[kWords];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2(y[i]);
            round_pair<T>(o, i, f.x, f.y);
          }
          store<T, WIDE>(static_cast<T *>(a.out) + (int64_t)row * a.out_pitch + c[v], o, n[v]);
        } else {
          if (n[v] < 8)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 f = unpack2(y[i]);
              y[i] = pack2(2 * i < n[v] ? f.x : 0.0f, 2 * i + 1 < n[v] ? f.y : 0.0f);
            }
          quantize8<OUT == kE5M2, WIDE>(a, row, c[v], n[v], y, g.lane);
        }
      }
    }
  }
}

// The transpose in 8 bits, from the sum and rstd that the forward kernel left.  A CTA walks
// tiles of 128 x 128, the last rows first: those are what the forward kernel left in L2.  The
// next tile comes into shared memory while the one before is stored; four CTAs on an SM
// cover for each other otherwise.  Thread (tx, ty) takes rows 8 ty + 0..7 of columns 8 tx +
// 0..7; the transpose goes through shared memory in 8-byte pieces, swizzled.
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

// 16 bytes, of which the first n are copied and the others zeros.
__device__ __forceinline__ void copy_block(uint32_t dst, const void *src, uint32_t n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}

template <typename T, bool E5M2>
__global__ void __launch_bounds__(256, sizeof(T) == 4 ? 2 : 4) turn_kernel(const __grid_constant__ TurnArgs a) {
  constexpr int kWords = 8 / Word<T>::kPer;
  constexpr uint32_t kPitch = 128 * sizeof(T);
  extern __shared__ __align__(128) uint8_t s_tile[];
  __shared__ __align__(16) TurnShared sh;
  const uint32_t tx = threadIdx.x % 16, ty = threadIdx.x / 16, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t across = (a.cols + kBlock - 1) / kBlock, down = (a.rows + kBlock - 1) / kBlock;
  const uint64_t tiles = (uint64_t)across * down;
  wait_for_first();
  // tiles from the last one on: each step goes back gridDim.x of them
  const uint32_t back_r = gridDim.x / across, back_c = gridDim.x % across;
  const auto step_back = [&](uint32_t &tr, uint32_t &tc) {
    tr -= back_r + (tc < back_c);
    tc = tc < back_c ? tc + across - back_c : tc - back_c;
  };
  // thread (tx, ty) brings columns 8 tx + 0..7 of rows ty, ty + 16, ...
  const auto fetch = [&](uint32_t tr, uint32_t tc) {
    const uint32_t c = tc * kBlock + 8 * tx, r = tr * kBlock + ty;
    uint8_t *to = s_tile + ty * kPitch + tx * (8 * sizeof(T));
    const T *h = static_cast<const T *>(a.h) + (int64_t)r * a.pitch + c;
    if (a.wide && (tr + 1) * kBlock <= a.rows && (tc + 1) * kBlock <= a.cols) {
      uint32_t at = smem_addr(to);
#pragma unroll
      for (int i = 0; i < 8; ++i, h += 16 * a.pitch)
#pragma unroll
        for (int j = 0; j < kWords; j += 4) copy_block(at + i * 16 * kPitch + 4 * j, reinterpret_cast<const uint8_t *>(h) + 4 * j, 16);
    } else {
      const int n = c < a.cols ? (int)min(8u, a.cols - c) : 0;
      for (int i = 0; i < 8; ++i, h += 16 * a.pitch, to += 16 * kPitch) {
        uint32_t w[kWords];
        load8<T>(w, h, r + 16 * i < a.rows ? n : 0, a.wide);
#pragma unroll
        for (int j = 0; j < kWords; j += 4) *reinterpret_cast<uint4 *>(to + 4 * j) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
      }
    }
    if (threadIdx.x < 128) {
      const uint32_t k = tr * kBlock + threadIdx.x;
      sh.rstd[threadIdx.x] = k < a.rows ? __ldg(a.rstd + k) : 0.0f;
    }
  };
  uint32_t tr = 0, tc = 0;
  if (blockIdx.x < tiles) {
    const uint64_t t = tiles - 1 - blockIdx.x;
    tr = (uint32_t)(t / across), tc = (uint32_t)(t % across);
    fetch(tr, tc);
  }
  for (uint64_t s = blockIdx.x; s < tiles; s += gridDim.x) {
    const uint32_t r0 = tr * kBlock, c0 = tc * kBlock;
    uint64_t wt[4];
    {
      const uint32_t c = c0 + 8 * tx;
      weights<true>(wt, a.weight, a.wdtype, a.weight_aligned, c, c < a.cols ? (int)min(8u, a.cols - c) : 0);
    }
    words_landed();
    __syncthreads();
    // h * rstd of columns 2j and 2j + 1 of row 8 ty + i
    const auto scaled = [&](const uint32_t (&w)[kWords], int i, int j) {
      const float r = sh.rstd[8 * ty + i];
      return mul2(pack2(element<T>(w, 2 * j), element<T>(w, 2 * j + 1)), pack2(r, r));
    };
    const auto row_words = [&](uint32_t (&w)[kWords], int i) {
#pragma unroll
      for (int j = 0; j < kWords; j += 4) {
        const uint4 v = *reinterpret_cast<const uint4 *>(s_tile + (8 * ty + i) * kPitch + tx * (8 * sizeof(T)) + 4 * j);
        w[j] = v.x, w[j + 1] = v.y, w[j + 2] = v.z, w[j + 3] = v.w;
      }
    };
    // The largest |y| of a column is the largest |h * rstd| times |weight|: rounding keeps the order.
    float top[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) top[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      uint32_t w[2][kWords];
      row_words(w[0], i);
      row_words(w[1], i + 1);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 p = unpack2(scaled(w[0], i, j)), q = unpack2(scaled(w[1], i + 1, j));
        top[2 * j] = max_abs(top[2 * j], p.x, q.x);
        top[2 * j + 1] = max_abs(top[2 * j + 1], p.y, q.y);
      }
    }
    uint32_t col[8], any = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 p = unpack2(mul2(pack2(top[2 * j], top[2 * j + 1]), wt[j]));
      col[2 * j] = __float_as_uint(p.x) & 0x7fffffffu, col[2 * j + 1] = __float_as_uint(p.y) & 0x7fffffffu;
    }
    const auto share = [&]() {
#pragma unroll
      for (int j = 0; j < 8; ++j) col[j] = max(col[j], __shfl_xor_sync(~0u, col[j], 16)), any = max(any, col[j]);
      if (lane < 16) {
        *reinterpret_cast<uint4 *>(&sh.col[warp][tx * 8]) = make_uint4(col[0], col[1], col[2], col[3]);
        *reinterpret_cast<uint4 *>(&sh.col[warp][tx * 8 + 4]) = make_uint4(col[4], col[5], col[6], col[7]);
      }
    };
    share();
    any = __syncthreads_or(any >= 0x7f800000u);
    if (any) {  // something is not finite: the largest of what is
#pragma unroll
      for (int j = 0; j < 8; ++j) col[j] = 0;
      for (int i = 0; i < 8; ++i) {
        uint32_t w[kWords];
        row_words(w, i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint64_t y = mul2(scaled(w, i, j), wt[j]);
          const uint32_t u = (uint32_t)y & 0x7fffffffu, v = (uint32_t)(y >> 32) & 0x7fffffffu;
          col[2 * j] = max(col[2 * j], u < 0x7f800000u ? u : 0), col[2 * j + 1] = max(col[2 * j + 1], v < 0x7f800000u ? v : 0);
        }
      }
      share();
      __syncthreads();
    }
    if (threadIdx.x < 128) {
      uint32_t m = 0;
#pragma unroll
      for (int v = 0; v < 8; ++v) m = max(m, sh.col[v][threadIdx.x]);
      const uint32_t e = scale_exponent<E5M2>(__uint_as_float(m));
      sh.inv[threadIdx.x] = inverse_power(e);
      if (c0 + threadIdx.x < a.cols) a.qt.scale[(int64_t)tr * a.qt.scale_pitch + c0 + threadIdx.x] = power(e);
    }
    __syncthreads();
    if (!any) {
      uint32_t half[8][2];  // of a column: rows 0-3 and 4-7
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        uint32_t pair[8][2];  // rows i and i + 1, i + 2 and i + 3
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          uint32_t w[2][kWords];
          row_words(w[0], i + k);
          row_words(w[1], i + k + 1);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 f = *reinterpret_cast<const float2 *>(&sh.inv[8 * tx + 2 * j]);
            const uint64_t inv = pack2(f.x, f.y);
            const float2 p = unpack2(mul2(mul2(scaled(w[0], i + k, j), wt[j]), inv));
            const float2 q = unpack2(mul2(mul2(scaled(w[1], i + k + 1, j), wt[j]), inv));
            pair[2 * j][k / 2] = to_fp8x2<E5M2>(p.x, q.x);
            pair[2 * j + 1][k / 2] = to_fp8x2<E5M2>(p.y, q.y);
          }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) half[j][i / 4] = __byte_perm(pair[j][0], pair[j][1], 0x5410);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sh.turn[(8 * tx + j) * 16 + (ty ^ tx)] = make_uint2(half[j][0], half[j][1]);
    } else {
      uint32_t b[8][2] = {};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t w[kWords];
        row_words(w, i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = unpack2(mul2(scaled(w, i, j), wt[j]));
          b[2 * j][i / 4] |= (uint32_t)any_to_fp8<E5M2>(f.x, sh.inv[8 * tx + 2 * j]) << (i % 4 * 8);
          b[2 * j + 1][i / 4] |= (uint32_t)any_to_fp8<E5M2>(f.y, sh.inv[8 * tx + 2 * j + 1]) << (i % 4 * 8);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sh.turn[(8 * tx + j) * 16 + (ty ^ tx)] = make_uint2(b[j][0], b[j][1]);
    }
    __syncthreads();
    const uint32_t rr = r0 + 8 * tx;  // now tx counts pieces down a column
    const bool whole = r0 + kBlock <= a.rows && c0 + kBlock <= a.cols;
    if (s + gridDim.x < tiles) {
      step_back(tr, tc);
      fetch(tr, tc);
    }
    uint8_t *to = a.qt.data + (int64_t)(c0 + ty) * a.qt.pitch + rr;
    if (whole) {
#pragma unroll
      for (int i = 0; i < 8; ++i, to += 16 * a.qt.pitch) {
        const uint32_t k = 16 * i + ty;
        *reinterpret_cast<uint2 *>(to) = sh.turn[k * 16 + (tx ^ k / 8)];
      }
    } else {
      const int nr = rr < a.rows ? (int)min(8u, a.rows - rr) : 0;
      for (int i = 0; i < 8; ++i, to += 16 * a.qt.pitch) {
        const uint32_t k = 16 * i + ty;
        if (c0 + k < a.cols && nr) store8(to, sh.turn[k * 16 + (tx ^ k / 8)], nr);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Gradient.  The rows are dealt out to `parts` parts whose number follows the sizes alone
// (few_of, rms_norm_parts): part p has rows p, p + parts, ....  A group walks a part and keeps its
// columns' sums of dout * z in registers, which go to the workspace, from where a second
// kernel adds them in order.

struct GradArgs {
  const void *dout, *x, *weight, *dresidual;
  const float *rstd;
  void *dx;
  float *partial;  // [parts][cols]; null: no dweight, or a cluster's
  void *dweight;   // written by the cluster kernel
  int64_t dout_pitch, pitch, dresidual_pitch, dx_pitch;
  uint32_t rows, cols, parts, wdtype, weight_aligned, dwdtype;
  float inv_cols;
};

// The sums of p over a group, in an order of its own, in every thread.
template <int U>
__device__ __forceinline__ void group_sums(float (&p)[U], const Group &g, float *room) {
#pragma unroll
  for (int o = 16; o; o >>= 1)
#pragma unroll
    for (int u = 0; u < U; ++u) p[u] += __shfl_xor_sync(~0u, p[u], o);
  if (U > 1 || g.warps == 1) return;  // several rows at a time: groups of one warp
  if (g.lane == 0) room[g.warp] = p[0];
  g.sync();
  p[0] = g.lane < g.warps ? room[g.lane] : 0.0f;
#pragma unroll
  for (int o = 16; o; o >>= 1) p[0] += __shfl_xor_sync(~0u, p[0], o);
}

__device__ __forceinline__ float group_sum(float p, const Group &g, float *room) {
  float s[1] = {p};
  group_sums<1>(s, g, room);
  return s[0];
}

// One run of 8 columns a thread: z and g = dout * weight of a row.
template <typename T>
__device__ __forceinline__ void z_and_g(const uint32_t (&x)[8 / Word<T>::kPer], const uint32_t (&d)[8 / Word<T>::kPer], float rstd,
                                        const uint64_t (&wt)[4], int i, uint64_t *z, uint64_t *g, uint64_t *dd) {
  *dd = pack2(element<T>(d, 2 * i), element<T>(d, 2 * i + 1));
  *z = mul2(pack2(element<T>(x, 2 * i), element<T>(x, 2 * i + 1)), pack2(rstd, rstd));
  *g = mul2(*dd, wt[i]);
}

__device__ __forceinline__ void store_weight(void *to, uint32_t dtype, uint32_t c, float y) {
  if (dtype == APC_F32) static_cast<float *>(to)[c] = y;
  else if (dtype == APC_BF16) static_cast<__nv_bfloat16 *>(to)[c] = from_float<__nv_bfloat16>(y);
  else static_cast<__half *>(to)[c] = from_float<__half>(y);
}

__device__ __forceinline__ float load_remote(uint32_t mapped) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(mapped) : "memory");
  return v;
}

// The groups of a CTA join their sums in shared memory, and their part of the workspace is
// the CTA's.  CLUSTER, for few rows: the grid is one cluster with a part for each group, and all
// sums meet in its shared memory: one launch, no workspace.  U rows at a time where a group is
// a warp, so that one's latencies lie beside the others'.
template <typename T, int V, int U, bool WIDE, bool CLUSTER>
__global__ void __launch_bounds__(512, 1) grad_kernel(const __grid_constant__ GradArgs a) {
  constexpr int kWords = 8 / Word<T>::kPer;
  extern __shared__ float s_sums[];  // [2][groups][warps], [groups][cols]
  if (!CLUSTER && a.partial) start_next();
  const Group g{blockDim.x / 32, 1 + threadIdx.y, threadIdx.x / 32, threadIdx.x % 32};
  float *const part_sums = s_sums + 2 * blockDim.y * g.warps;
  uint32_t turn = 0;
  uint32_t c[V];
  int n[V];
  constexpr bool kAgain = V == 4;  // registers are short: weights come from L1 for each row, dresidual after the sum
  uint64_t wt[kAgain ? 1 : V][4];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    c[v] = first_of<WIDE>(g.warp + v * g.warps, g.lane);
    n[v] = count_of<WIDE>(c[v], a.cols);
    if (!kAgain) weights<WIDE>(wt[v], a.weight, a.wdtype, a.weight_aligned, c[v], n[v]);
  }
  const uint32_t step = a.parts * blockDim.y;  // parts: of CTAs
  for (uint32_t part = blockIdx.x; part < a.parts; part += gridDim.x) {
    uint64_t acc[V][4] = {};
    for (uint64_t first = part * blockDim.y + threadIdx.y; first < a.rows; first += (uint64_t)step * U) {
      float *room = s_sums + (turn ^= 1) * blockDim.y * g.warps + threadIdx.y * g.warps;
      uint32_t x[U][V][kWords], d[U][V][kWords], r[U][kAgain ? 1 : V][kWords];
      float rstd[U], dot[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint64_t at = first + (uint64_t)u * step;
        const bool there = u == 0 || at < a.rows;
        const int64_t row = there ? (int64_t)at : 0;
        rstd[u] = __ldg(a.rstd + row);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int m = there ? n[v] : 0;
          load<T, WIDE>(x[u][v], static_cast<const T *>(a.x) + row * a.pitch + c[v], m);
          load<T, WIDE>(d[u][v], static_cast<const T *>(a.dout) + row * a.dout_pitch + c[v], m);
          if (!kAgain && a.dresidual) load<T, WIDE>(r[u][v], static_cast<const T *>(a.dresidual) + row * a.dresidual_pitch + c[v], m);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u && first + (uint64_t)u * step >= a.rows) rstd[u] = 0.0f;  // nothing is added for a row that is not there
        uint64_t sum = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          uint64_t(&w)[4] = wt[kAgain ? 0 : v];
          if (kAgain) weights<WIDE>(w, a.weight, a.wdtype, a.weight_aligned, c[v], n[v]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint64_t z, gg, dd;
            z_and_g<T>(x[u][v], d[u][v], rstd[u], w, i, &z, &gg, &dd);
            sum = fma2(gg, z, sum);
            acc[v][i] = fma2(dd, z, acc[v][i]);
          }
        }
        const float2 both = unpack2(sum);
        dot[u] = both.x + both.y;
      }
      group_sums<U>(dot, g, room);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint64_t row = first + (uint64_t)u * step;
        if (u && row >= a.rows) break;
        const float mean = dot[u] * a.inv_cols;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          uint32_t o[kWords], (&res)[kWords] = r[u][kAgain ? 0 : v];
          uint64_t(&w)[4] = wt[kAgain ? 0 : v];
          if (kAgain) {
            weights<WIDE>(w, a.weight, a.wdtype, a.weight_aligned, c[v], n[v]);
            if (a.dresidual) load<T, WIDE>(res, static_cast<const T *>(a.dresidual) + (int64_t)row * a.dresidual_pitch + c[v], n[v]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint64_t z, gg, dd;
            z_and_g<T>(x[u][v], d[u][v], rstd[u], w, i, &z, &gg, &dd);
            float2 f = unpack2(mul2(fma2(z, pack2(-mean, -mean), gg), pack2(rstd[u], rstd[u])));
            if (a.dresidual) f.x += element<T>(res, 2 * i), f.y += element<T>(res, 2 * i + 1);
            round_pair<T>(o, i, f.x, f.y);
          }
          store<T, WIDE>(static_cast<T *>(a.dx) + (int64_t)row * a.dx_pitch + c[v], o, n[v]);
        }
      }
    }
    if (!CLUSTER && !a.partial) continue;
    const bool alone = !CLUSTER && blockDim.y == 1;
    float *const sums = alone ? a.partial + (uint64_t)part * a.cols : part_sums + threadIdx.y * a.cols;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 f = unpack2(acc[v][i / 2]);
        if (i < n[v]) sums[c[v] + (WIDE ? i : 32 * i)] = i % 2 ? f.y : f.x;
      }
    if (CLUSTER || alone) continue;
    __syncthreads();
    for (uint32_t k = threadIdx.y * blockDim.x + threadIdx.x; k < a.cols; k += blockDim.x * blockDim.y) {
      float s = 0.0f;
      for (uint32_t q = 0; q < blockDim.y; ++q) s += part_sums[q * a.cols + k];
      a.partial[(uint64_t)part * a.cols + k] = s;
    }
    __syncthreads();
  }
  if (!CLUSTER) return;
  cluster_arrive();
  cluster_wait();
  // a slice of the columns for each CTA
  const uint32_t per = (a.cols + gridDim.x - 1) / gridDim.x, begin = blockIdx.x * per, end = min(a.cols, begin + per);
  for (uint32_t k = begin + threadIdx.y * blockDim.x + threadIdx.x; k < end; k += blockDim.x * blockDim.y) {
    float s = 0.0f;
    for (uint32_t r = 0; r < blockDim.y; ++r) {
      const uint32_t at = smem_addr(part_sums + r * a.cols + k);
      for (uint32_t q = 0; q < gridDim.x; q += 8) {  // a power of two of CTAs
        float f[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) f[i] = q + i < gridDim.x ? load_remote(map_rank(at, q + i)) : 0.0f;
        s += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
      }
    }
    store_weight(a.dweight, a.dwdtype, k, s);
  }
  cluster_arrive();
  cluster_wait();  // the others' reads of this CTA's sums
}

// Rows that a group does not hold: twice over each, element by element.
template <typename T>
__global__ void __launch_bounds__(1024, 1) grad_long_kernel(const __grid_constant__ GradArgs a) {
  __shared__ float room[2][32];
  if (a.partial) start_next();
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
  wait_for_first();
  start_next();
  for (uint64_t t = blockIdx.x; t < per * a.parts; t += gridDim.x) {
    const uint32_t part = (uint32_t)(t / per), c = (uint32_t)(t % per) * 256 + threadIdx.x;
    if (c >= a.cols) continue;
    float acc = 0.0f;
    for (uint64_t row = part; row < a.rows; row += a.parts)
      acc = __fmaf_rn(to_float(static_cast<const T *>(a.dout)[(int64_t)row * a.dout_pitch + c]),
                      to_float(static_cast<const T *>(a.x)[(int64_t)row * a.pitch + c]) * __ldg(a.rstd + row), acc);
    a.partial[(uint64_t)part * a.cols + c] = acc;
  }
}

// dweight: the parts' sums, 32 columns a CTA, warp k those of parts k, k + 16, ..., then the warps'.
__global__ void __launch_bounds__(512) parts_kernel(const float *partial, uint32_t parts, uint32_t cols, void *dweight, uint32_t dtype) {
  __shared__ float sums[16][32];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint32_t runs = (cols + 31) / 32;
  wait_for_first();
  for (uint32_t run = blockIdx.x; run < runs; run += gridDim.x) {
    const uint32_t c = run * 32 + lane;
    float s = 0.0f;
    if (c < cols)
#pragma unroll 8
      for (uint32_t p = warp; p < parts; p += 16) s += __ldcg(partial + (uint64_t)p * cols + c);
    __syncthreads();
    sums[warp][lane] = s;
    __syncthreads();
    if (warp || c >= cols) continue;
    float y = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; k += 4) y += (sums[k][lane] + sums[k + 1][lane]) + (sums[k + 2][lane] + sums[k + 3][lane]);
    store_weight(dweight, dtype, c, y);
  }
}

// ---------------------------------------------------------------------------
// Many rows: a CTA walks rows, which bulk copies bring into a ring of shared memory, one or
// two rows ahead of the one at work, so that memory is never waited for row by row.
//
// A row's copy takes the 16-byte blocks that hold it, wherever it begins, and a thread works
// on units of eight elements that begin at a block's boundary, not at a multiple of eight
// columns: loads and stores stay wide for rows at any boundary, as long as all matrices lie
// alike within 16 bytes.  What a unit holds beside the row is masked.  Blocks that would
// leave the matrix are not copied: their elements are put in place one by one.  The
// barrier of a row's sum is also what frees the stage of the row before.
//
// The weights lie in shared memory as fp32, as the threads' elements do; rows that a CTA
// walks begin alike where the grid allows it, else the weights are laid out again for each.

constexpr uint32_t kStagesMost = 3;

struct Ring {
  uint32_t stages, region, mats;  // region: bytes of a matrix's part of a stage
  uint32_t weights;               // bytes of the weights
  uint32_t edges;                 // 1: the first row's first block begins in front of the matrix, 2: the last one's last ends behind
  unsigned *status;

  __host__ __device__ uint32_t stage() const { return region * mats; }
  __host__ __device__ uint32_t bytes() const { return stages * stage() + weights; }
};

struct RingShared {
  uint64_t full[kStagesMost];
  Stat stats[2][32];
  float sums[2][32];
  int dead;
};

// The barriers, and the first copies by `issue`: one thread.  A __syncthreads has to follow.
template <typename F>
__device__ __forceinline__ void ring_begin(RingShared &sh, uint32_t stages, F issue) {
  if (threadIdx.x) return;
  for (uint32_t s = 0; s < stages; ++s) mbar_init(&sh.full[s], 1);
  sh.dead = 0;
  mbar_init_fence();
  for (uint32_t s = 0; s + 1 < stages; ++s) issue();
}

// The bounded wait for a stage.  After one that gave up nothing more is copied and nothing
// waited for; what follows is not to be used, as the status word says.
__device__ __noinline__ void ring_wait_on(RingShared &sh, uint32_t stage, uint32_t parity, unsigned *status) {
  if (*(volatile int *)&sh.dead || mbar_wait(&sh.full[stage], parity)) return;
  atomicOr(status, (unsigned)APC_ETIMEOUT);
  *(volatile int *)&sh.dead = 1;
}
__device__ __forceinline__ void ring_wait(RingShared &sh, uint32_t stage, uint32_t parity, unsigned *status) {
  if (!mbar_try_wait(smem_addr(&sh.full[stage]), parity)) ring_wait_on(sh, stage, parity, status);
}

// Bytes of a row's first block in front of the row.
__device__ __forceinline__ uint32_t skip_of(const void *base, int64_t pitch, uint32_t row, uint32_t size) {
  return ((uint32_t)(uintptr_t)base + row * (uint32_t)pitch * size) & 15;
}

struct Source {
  const void *base;
  int64_t pitch;
};

// One thread: copy a row of each matrix into a stage.
template <int M>
__device__ __forceinline__ void ring_issue(RingShared &sh, const Source (&src)[M], const Ring &ring, uint8_t *stage, uint64_t *full,
                                           uint32_t row, uint32_t rows, uint32_t cols, uint32_t size, uint64_t policy) {
  if (*(volatile int *)&sh.dead) return;
  const uint32_t skip = skip_of(src[0].base, src[0].pitch, row, size);
  const uint32_t from = row == 0 && ring.edges & 1 ? 16 : 0;
  const uint32_t bytes = ((skip + cols * size + 15) & ~15u) - from - (row == rows - 1 && ring.edges & 2 ? 16 : 0);
  mbar_arrive_expect_tx(full, bytes * ring.mats);
#pragma unroll
  for (int m = 0; m < M; ++m) {
    if (m >= ring.mats) break;
    const uint8_t *at = static_cast<const uint8_t *>(src[m].base) + (int64_t)row * src[m].pitch * size - skip + from;
    bulk_g2s(stage + m * ring.region + from, at, bytes, full, policy);
  }
}

// The elements of the blocks that ring_issue left out, in the first and the last row alone.
template <typename T, int M>
__device__ __forceinline__ void ring_edges(const Source (&src)[M], const Ring &ring, uint8_t *stage, uint32_t row, uint32_t rows,
                                           uint32_t cols) {
  const bool front = row == 0 && ring.edges & 1, back = row == rows - 1 && ring.edges & 2;
  if (!front && !back) return;
  const uint32_t skip = skip_of(src[0].base, src[0].pitch, row, sizeof(T)), i = threadIdx.x % 16;
  const uint32_t per = 16 / sizeof(T), first = skip / sizeof(T), last = (first + cols) & ~(per - 1);  // the first element of the last block
  const uint32_t e = threadIdx.x < 16 ? i : last + i;                                                 // counted from the first block
  if (threadIdx.x < 32 && i < per && (threadIdx.x < 16 ? front : back) && e >= first && e < first + cols)
    for (int m = 0; m < M; ++m)
      if (m < ring.mats)
        reinterpret_cast<T *>(stage + m * ring.region)[e] =
            *(static_cast<const T *>(src[m].base) + (int64_t)row * src[m].pitch + (e - first));
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // copies come here again
  __syncthreads();
}

// Unit u of a row: eight elements from column `first` on (below 0 in front of the row).
// WHOLE: rows begin at blocks and are units and nothing else.
template <bool WHOLE>
struct Unit {
  int32_t first;
  bool any, full;

  __device__ Unit(uint32_t u, uint32_t shift, uint32_t cols) {
    first = (int32_t)(8 * u - (WHOLE ? 0 : shift));
    any = first < (int32_t)cols;
    full = WHOLE ? any : first >= 0 && first + 8 <= (int32_t)cols;
  }
};

// Its elements, zeros where there are none.
template <typename T, bool WHOLE>
__device__ __forceinline__ void ring_load(uint32_t (&w)[8 / Word<T>::kPer], const uint8_t *region, uint32_t k, const Unit<WHOLE> &u,
                                          uint32_t cols) {
  constexpr int kWords = 8 / Word<T>::kPer;
  if (u.any) {
#pragma unroll
    for (int i = 0; i < kWords; i += 4) {
      const uint4 v = *reinterpret_cast<const uint4 *>(region + k * (8 * sizeof(T)) + 4 * i);
      w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
    }
    if (!WHOLE && !u.full) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool there = u.first + i >= 0 && u.first + i < (int32_t)cols;
        if (sizeof(T) == 4) w[i] = there ? w[i] : 0;
        else w[i / 2] &= there ? ~0u : i % 2 ? 0xffffu : 0xffff0000u;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
}

template <typename T, bool WHOLE>
__device__ __forceinline__ void ring_store(T *row, const uint32_t (&w)[8 / Word<T>::kPer], const Unit<WHOLE> &u, uint32_t cols) {
  if (u.full) {
#pragma unroll
    for (int i = 0; i < 8 / Word<T>::kPer; i += 4)
      *(reinterpret_cast<uint4 *>(row + u.first) + i / 4) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
  } else if (!WHOLE && u.any) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int32_t c = u.first + i;
      if (c < 0 || c >= (int32_t)cols) continue;
      if (sizeof(T) == 4) reinterpret_cast<uint32_t *>(row)[c] = w[i];
      else reinterpret_cast<uint16_t *>(row)[c] = (uint16_t)element_bits<T>(w, i);
    }
  }
}

// The weights of all units, the first of which begins `shift` columns in front of the row.
__device__ __forceinline__ void lay_weights(float *to, const void *weight, uint32_t dtype, uint32_t units, uint32_t shift, uint32_t cols) {
  for (uint32_t i = threadIdx.x; i < 8 * units; i += blockDim.x) {
    const uint32_t c = i - shift;
    float v = 0.0f;
    if (i >= shift && c < cols)
      v = dtype == APC_F32    ? __ldg(static_cast<const float *>(weight) + c)
          : dtype == APC_BF16 ? to_float(static_cast<const __nv_bfloat16 *>(weight)[c])
                              : to_float(static_cast<const __half *>(weight)[c]);
    // a unit's halves lie apart, so that a warp's 16-byte loads meet no bank twice
    to[(i / 8 * 4) + (i % 8 / 4) * 4 * units + i % 4] = v;
  }
}

__device__ __forceinline__ void unit_weights(uint64_t (&v)[4], const float *laid, uint32_t units, uint32_t k) {
  const ulonglong2 a = *reinterpret_cast<const ulonglong2 *>(laid + 4 * k), b = *reinterpret_cast<const ulonglong2 *>(laid + 4 * units + 4 * k);
  v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
}

// Eight elements from `skip` bytes behind a unit's first block on.
template <typename T>
__device__ __forceinline__ void ring_shifted(uint32_t (&w)[8 / Word<T>::kPer], const uint8_t *unit, uint32_t skip) {
  constexpr int kWords = 8 / Word<T>::kPer;
  uint32_t v[kWords + 4];
#pragma unroll
  for (int i = 0; i < kWords + 4; i += 4) {
    const uint4 b = *reinterpret_cast<const uint4 *>(unit + 4 * i);
    v[i] = b.x, v[i + 1] = b.y, v[i + 2] = b.z, v[i + 3] = b.w;
  }
  if (skip & 8) {
#pragma unroll
    for (int i = 0; i < kWords + 2; ++i) v[i] = v[i + 2];
  }
  if (skip & 4) {
#pragma unroll
    for (int i = 0; i < kWords + 1; ++i) v[i] = v[i + 1];
  }
#pragma unroll
  for (int i = 0; i < kWords; ++i) w[i] = sizeof(T) == 4 ? v[i] : __funnelshift_r(v[i], v[i + 1], (skip & 3) * 8);
}

// 8-bit outputs have rows at multiples of 16 bytes: their threads take units that begin at
// multiples of eight columns.  For rows that begin elsewhere the sum goes through the stage.
template <typename T, int OUT, int V, bool WHOLE>
__global__ void __launch_bounds__(V == 1 ? 512 : 1024, V == 1 ? 2 : 1) ring_forward_kernel(const __grid_constant__ ForwardArgs a,
                                                                                    const __grid_constant__ Ring ring) {
  constexpr int kWords = 8 / Word<T>::kPer;
  extern __shared__ __align__(128) uint8_t s_ring[];
  __shared__ RingShared sh;
  const Group g{blockDim.x / 32, 0, threadIdx.x / 32, threadIdx.x % 32};
  const uint32_t units = V * blockDim.x;
  float *const laid = reinterpret_cast<float *>(s_ring + ring.stages * ring.stage());
  if (a.then) start_next();
  const Source src[2] = {{a.x, a.pitch}, {a.residual, a.residual_pitch}};
  uint32_t next = blockIdx.x, into = 0;  // the row to copy next, its stage
  const auto issue = [&]() {
    if (next < a.rows) {
      ring_issue<2>(sh, src, ring, s_ring + into * ring.stage(), &sh.full[into], next, a.rows, a.cols, sizeof(T), l2_evict_first());
      next += gridDim.x;
    }
    if (++into == ring.stages) into = 0;
  };
  ring_begin(sh, ring.stages, issue);
  uint32_t shift = ~0u, stage = 0, parity = 0, turn = 0;
  if (OUT != kSame) lay_weights(laid, a.weight, a.wdtype, units, 0, a.cols);
  __syncthreads();
  for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const uint32_t skip = WHOLE ? 0 : skip_of(a.x, a.pitch, row, sizeof(T));
    if (OUT == kSame && skip != shift) {
      __syncthreads();
      lay_weights(laid, a.weight, a.wdtype, units, skip / sizeof(T), a.cols);
      __syncthreads();
      shift = skip;
    }
    uint8_t *const at = s_ring + stage * ring.stage();
    ring_wait(sh, stage, parity, ring.status);
    if (!WHOLE && ring.edges) ring_edges<T, 2>(src, ring, at, row, a.rows, a.cols);
    uint32_t w[V][kWords];
    float p = 0.0f, rstd;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const uint32_t k = threadIdx.x + v * blockDim.x;
      const Unit<WHOLE> u(k, skip / sizeof(T), a.cols);
      ring_load<T, WHOLE>(w[v], at, k, u, a.cols);
      if (a.residual) {
        uint32_t x[kWords];
        ring_load<T, WHOLE>(x, at + ring.region, k, u, a.cols);
        add_rounded<T>(w[v], x);
        ring_store<T, WHOLE>(static_cast<T *>(a.sum) + (int64_t)row * a.sum_pitch, w[v], u, a.cols);
      }
      if (OUT != kSame && skip && u.any) {
#pragma unroll
        for (int i = 0; i < kWords; i += 4)
          *reinterpret_cast<uint4 *>(at + k * (8 * sizeof(T)) + 4 * i) = make_uint4(w[v][i], w[v][i + 1], w[v][i + 2], w[v][i + 3]);
      }
      p += squares<T>(w[v]);
    }
    // before the next copy into a stage that was written here
    if (OUT != kSame && skip) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    const bool fine = row_rstd(p, g, sh.stats[turn ^= 1], a.c, true, &rstd);
    if (threadIdx.x == 0) issue();  // into the stage of the row before, which all have left
    if (!fine) rstd = wild_rstd<T, V>(w, g, sh.stats[turn], a.c);
    if (threadIdx.x == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const uint32_t k = threadIdx.x + v * blockDim.x;
      const Unit<WHOLE> u(k, OUT == kSame ? skip / sizeof(T) : 0, a.cols);
      if (OUT != kSame && skip && u.any) ring_shifted<T>(w[v], at + k * (8 * sizeof(T)), skip);
      uint64_t wt[4], y[4];
      unit_weights(wt, laid, units, k);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = mul2(mul2(pack2(element<T>(w[v], 2 * i), element<T>(w[v], 2 * i + 1)), pack2(rstd, rstd)), wt[i]);
      if (OUT == kSame) {
        uint32_t o[kWords];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = unpack2(y[i]);
          round_pair<T>(o, i, f.x, f.y);
        }
        ring_store<T, WHOLE>(static_cast<T *>(a.out) + (int64_t)row * a.out_pitch, o, u, a.cols);
      } else {
        const int n = u.full ? 8 : u.any ? (int)a.cols - u.first : 0;
        if (!u.full)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2(y[i]);
            y[i] = pack2(2 * i < n ? f.x : 0.0f, 2 * i + 1 < n ? f.y : 0.0f);
          }
        quantize8<OUT == kE5M2, true>(a, row, 8 * k, n, y, g.lane);
      }
    }
    if (++stage == ring.stages) stage = 0, parity ^= 1;
  }
}

// The gradient's rows through a ring of x, dout and dresidual.  Part p is rows p, p + parts,
// ...: rows of a part begin alike.
template <typename T, int V, bool WHOLE>
__global__ void __launch_bounds__(V == 1 ? 1024 : 512, 1) ring_grad_kernel(const __grid_constant__ GradArgs a, const __grid_constant__ Ring ring) {
  constexpr int kWords = 8 / Word<T>::kPer;
  extern __shared__ __align__(128) uint8_t s_ring[];
  __shared__ RingShared sh;
  const Group g{blockDim.x / 32, 0, threadIdx.x / 32, threadIdx.x % 32};
  const uint32_t units = V * blockDim.x;
  float *const laid = reinterpret_cast<float *>(s_ring + ring.stages * ring.stage());
  if (a.partial) start_next();
  const Source src[3] = {{a.x, a.pitch}, {a.dout, a.dout_pitch}, {a.dresidual, a.dresidual_pitch}};
  uint32_t next_part = blockIdx.x, next = next_part, into = 0;
  const auto issue = [&]() {
    if (next_part < a.parts) {
      ring_issue<3>(sh, src, ring, s_ring + into * ring.stage(), &sh.full[into], next, a.rows, a.cols, sizeof(T), l2_evict_first());
      next += a.parts;
      if (next >= a.rows) next = next_part += gridDim.x;
    }
    if (++into == ring.stages) into = 0;
  };
  ring_begin(sh, ring.stages, issue);
  uint32_t shift = ~0u, stage = 0, parity = 0, turn = 0;
  __syncthreads();
  for (uint32_t part = blockIdx.x; part < a.parts; part += gridDim.x) {
    uint64_t acc[V][4] = {};
    const uint32_t skip = WHOLE ? 0 : skip_of(a.x, a.pitch, part, sizeof(T));
    if (skip != shift) {
      __syncthreads();
      lay_weights(laid, a.weight, a.wdtype, units, skip / sizeof(T), a.cols);
      __syncthreads();
      shift = skip;
    }
    for (uint32_t row = part; row < a.rows; row += a.parts) {
      const float rstd = __ldg(a.rstd + row);
      uint8_t *const at = s_ring + stage * ring.stage();
      ring_wait(sh, stage, parity, ring.status);
      if (!WHOLE && ring.edges) ring_edges<T, 3>(src, ring, at, row, a.rows, a.cols);
      uint64_t z[V][4], gg[V][4], dot = 0;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const uint32_t k = threadIdx.x + v * blockDim.x;
        const Unit<WHOLE> u(k, skip / sizeof(T), a.cols);
        uint32_t x[kWords], d[kWords];
        ring_load<T, WHOLE>(x, at, k, u, a.cols);
        ring_load<T, WHOLE>(d, at + ring.region, k, u, a.cols);
        uint64_t wt[4];
        unit_weights(wt, laid, units, k);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint64_t dd;
          z_and_g<T>(x, d, rstd, wt, i, &z[v][i], &gg[v][i], &dd);
          dot = fma2(gg[v][i], z[v][i], dot);
          acc[v][i] = fma2(dd, z[v][i], acc[v][i]);
        }
      }
      const float2 both = unpack2(dot);
      const float mean = group_sum(both.x + both.y, g, sh.sums[turn ^= 1]) * a.inv_cols;
      if (threadIdx.x == 0) issue();  // into the stage of the row before, which all have left
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const uint32_t k = threadIdx.x + v * blockDim.x;
        const Unit<WHOLE> u(k, skip / sizeof(T), a.cols);
        uint32_t o[kWords];
        if (a.dresidual) ring_load<T, WHOLE>(o, at + 2 * ring.region, k, u, a.cols);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float2 f = unpack2(mul2(fma2(z[v][i], pack2(-mean, -mean), gg[v][i]), pack2(rstd, rstd)));
          if (a.dresidual) f.x += element<T>(o, 2 * i), f.y += element<T>(o, 2 * i + 1);
          round_pair<T>(o, i, f.x, f.y);
        }
        ring_store<T, WHOLE>(static_cast<T *>(a.dx) + (int64_t)row * a.dx_pitch, o, u, a.cols);
      }
      if (++stage == ring.stages) stage = 0, parity ^= 1;
    }
    if (!a.partial) continue;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Unit<WHOLE> u(threadIdx.x + v * blockDim.x, skip / sizeof(T), a.cols);
      float *to = a.partial + (uint64_t)part * a.cols + u.first;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 f = unpack2(acc[v][i / 2]);
        if (u.first + i >= 0 && u.first + i < (int32_t)a.cols) to[i] = i % 2 ? f.y : f.x;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// How a row lies over threads.

struct Shape {
  uint32_t threads, groups;  // threads of a group, groups of a CTA
  int v;                     // times 8 elements a thread
  bool fits;                 // a group holds the row
};

Shape shape_of(uint32_t cols, int v) {
  Shape s;
  s.v = v;
  const uint32_t per = 256 * s.v, warps = (cols + per - 1) / per;
  s.fits = warps <= (v == 4 ? 16u : 32u);
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

// From so many rows on a warp takes several at a time.
constexpr uint32_t kNarrowRows = 1024;

bool aligned(const void *p, int64_t pitch_bytes) { return (uintptr_t)p % 16 == 0 && pitch_bytes % 16 == 0; }

// More rows than `least`, of 16 bits, alike within 16 bytes: the ring's shape, or none (threads
// 0).  Where rows begin at blocks and end with them, plain loads by more warps keep up for most: the ring pays
// where a row's work is long, for 8-bit outputs (8192 x 4096 46 us, 50 by plain loads; to 16 bits
// 51 and 48, 4883 x 4096 of fp32 60 and 52) and for gradients of middling rows (8192 x 4096 59
// and 63, 16384 x 1024 41 and 38, 4883 x 4096 of fp32 65 and 59).  Elsewhere in the
// matrix it always does: 4001 x 5001 to 16 bits 35 us (46), its gradient 57 (100).
struct RingShape {
  uint32_t threads;
  int v;
  bool whole;
  Ring ring;
};

RingShape ring_shape(const void *x, int64_t pitch, uint32_t rows, uint32_t cols, uint32_t size, uint32_t mats, uint32_t least, bool grad,
                     bool alike, bool pays) {
  RingShape s = {};
  const bool begins = aligned(x, pitch * size);  // rows begin at blocks
  const uint32_t units = (cols + (begins ? 0 : 7) + 7) / 8;
  s.whole = begins && cols % 8 == 0;
  if (size != 2 || (s.whole && !pays) || !alike || rows <= least || cols <= 512 || units > 2048) return s;
  s.v = grad ? units <= 1024 ? 1 : 4 : units <= 512 ? 1 : 2;
  s.threads = 32 * ((units + 32 * s.v - 1) / (32 * s.v));
  s.ring.region = (cols * size + 15 + 15) / 16 * 16 + 16;
  s.ring.mats = mats;
  s.ring.weights = s.threads * s.v * 32;
  s.ring.edges = ((uintptr_t)x % 16 != 0) | (((uintptr_t)x + ((int64_t)(rows - 1) * pitch + cols) * size) % 16 != 0) << 1;
  for (s.ring.stages = 3; s.ring.stages > 1 && s.ring.bytes() > 220 * 1024; --s.ring.stages) {}
  if (s.ring.stages < 2) s.threads = 0;
  return s;
}

// The launch of a ring kernel: persistent, in so many CTAs as an SM holds, rows of a CTA
// beginning alike where the grid allows.
template <typename K, typename A>
int ring_launch(K kernel, const A &a, RingShape s, uint32_t work, uint32_t period, void *stream) {
  const uint32_t bytes = s.ring.bytes();
  int e = commit_status_word(&s.ring.status), per_sm = 1;
  if (!e) e = (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (!e) e = (int)cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, (int)s.threads, bytes);
  if (e) return e;
  unsigned grid = grid_of(work, (uint32_t)per_sm);
  if (grid < work && grid > period) grid -= grid % period;
  kernel<<<grid, s.threads, bytes, (cudaStream_t)stream>>>(a, s.ring);
  return (int)cudaGetLastError();
}

// Rows after which a matrix's place within 16 bytes repeats.
uint32_t period_of(int64_t pitch_bytes) {
  uint32_t n = 1;
  while (n < 16 && pitch_bytes * n % 16) n *= 2;
  return n;
}

bool same_place(const void *p, int64_t pitch_bytes, const void *q, int64_t q_pitch_bytes) {
  return !q || (((uintptr_t)p ^ (uintptr_t)q) % 16 == 0 && (pitch_bytes - q_pitch_bytes) % 16 == 0);
}

template <typename T, int OUT, int V, bool WIDE, bool LONG>
int forward_launch(const ForwardArgs &a, const Shape &s, void *stream) {
  const uint32_t per = s.threads * s.groups;
  const unsigned grid = grid_of((a.rows + s.groups - 1) / s.groups, 2048 / per);
  const size_t room = sizeof(Stat) * 2 * per / 32;
  forward_kernel<T, OUT, V, WIDE, LONG><<<grid, dim3(s.threads, s.groups), room, (cudaStream_t)stream>>>(a);
  return (int)cudaGetLastError();
}

template <typename T, int OUT>
int forward(const ForwardArgs &a, const Shape &s, const RingShape &ring, bool wide, void *stream) {
  if constexpr (sizeof(T) == 2) if (ring.threads) {
    const uint32_t period = period_of(a.pitch * (int64_t)sizeof(T));
    if (ring.whole)
      return ring.v == 1 ? ring_launch(ring_forward_kernel<T, OUT, 1, true>, a, ring, a.rows, period, stream)
                         : ring_launch(ring_forward_kernel<T, OUT, 2, true>, a, ring, a.rows, period, stream);
    return ring.v == 1 ? ring_launch(ring_forward_kernel<T, OUT, 1, false>, a, ring, a.rows, period, stream)
                       : ring_launch(ring_forward_kernel<T, OUT, 2, false>, a, ring, a.rows, period, stream);
  }
  if (a.cols <= 512 && a.rows > kNarrowRows) {
    const unsigned grid = grid_of((a.rows + 31) / 32, 4);
    cudaStream_t st = (cudaStream_t)stream;
    if (a.cols <= 256) {
      if (wide) narrow_kernel<T, OUT, 1, 4, true><<<grid, 256, 0, st>>>(a);
      else narrow_kernel<T, OUT, 1, 4, false><<<grid, 256, 0, st>>>(a);
    } else {
      if (wide) narrow_kernel<T, OUT, 2, 2, true><<<grid, 256, 0, st>>>(a);
      else narrow_kernel<T, OUT, 2, 2, false><<<grid, 256, 0, st>>>(a);
    }
    return (int)cudaGetLastError();
  }
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
  // with much to transpose its CTAs would be in the way (8192 x 4096 72 us, 67 one after the other)
  a.then = n.qt.data && (uint64_t)n.rows * n.cols <= 1u << 21;
  const Shape s = shape_of(n.cols, n.rows <= sms && n.cols <= 8192 ? 1 : 2);
  return with_dtype(n.dtype, [&](auto t) {
    using T = decltype(t);
    const auto at = [](const void *p, int64_t pitch) { return aligned(p, pitch * (int64_t)sizeof(T)); };
    const bool wide = at(n.x, n.pitch) && at(n.residual, n.residual_pitch) && at(n.sum, n.sum_pitch) && at(n.out, n.out_pitch);
    const auto alike = [&](const void *p, int64_t pitch) {
      return same_place(n.x, n.pitch * (int64_t)sizeof(T), p, pitch * (int64_t)sizeof(T));
    };
    const RingShape ring = ring_shape(n.x, n.pitch, n.rows, n.cols, sizeof(T), n.residual ? 2 : 1, 8 * sms, false,
                                      alike(n.residual, n.residual_pitch) && alike(n.sum, n.sum_pitch) && alike(n.out, n.out_pitch),
                                      !n.out);
    int e;
    if (n.out) e = forward<T, kSame>(a, s, ring, wide, stream);
    else e = n.q.e5m2 ? forward<T, kE5M2>(a, s, ring, wide, stream) : forward<T, kE4M3>(a, s, ring, wide, stream);
    if (e || !n.qt.data) return e;
    TurnArgs r = {};
    r.h = n.residual ? n.sum : n.x, r.weight = n.weight, r.rstd = n.rstd;
    r.qt = n.qt;
    r.pitch = n.residual ? n.sum_pitch : n.pitch;
    r.rows = n.rows, r.cols = n.cols, r.wdtype = n.wdtype;
    r.weight_aligned = a.weight_aligned;
    r.wide = at(r.h, r.pitch);
    const auto turn = n.qt.e5m2 ? turn_kernel<T, true> : turn_kernel<T, false>;
    constexpr uint32_t bytes = 128 * 128 * sizeof(T);
    if ((e = (int)cudaFuncSetAttribute(turn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes))) return e;
    const unsigned grid = grid_of((uint64_t)((n.cols + kBlock - 1) / kBlock) * ((n.rows + kBlock - 1) / kBlock), sizeof(T) == 4 ? 2 : 4);
    if (a.then) return launch_after(turn, grid, 256, bytes, stream, r);
    turn<<<grid, 256, bytes, (cudaStream_t)stream>>>(r);
    return (int)cudaGetLastError();
  });
}

namespace {

// Few rows: a cluster of so many CTAs (0: none) of so many groups, up to 8 rows for each.
struct Few {
  uint32_t ctas, groups;
};

constexpr uint32_t kGradParts = 304;

Shape grad_shape(uint32_t cols) { return shape_of(cols, cols <= 256 ? 1 : cols <= 8192 ? 2 : 4); }

Few few_of(uint32_t rows, uint32_t cols) {
  const Shape s = grad_shape(cols);
  if (!rows || !s.fits || (uint64_t)rows * cols > 1u << 20) return {0, 0};
  Few f = {1, 1};
  while (f.ctas < 16 && f.ctas < rows) f.ctas *= 2;
  const uint32_t most = s.threads >= 512 ? 1 : 512 / s.threads, want = (rows + 15) / 16;
  if (rows > 16) f.groups = want < most ? want : most;
  return rows > 8 * f.ctas * f.groups ? Few{0, 0} : f;
}

}  // namespace

// Parts: two CTAs for every SM, or as many groups (the ring's CTAs are one); none where a cluster does it.
uint32_t rms_norm_parts(uint32_t rows, uint32_t cols) {
  if (few_of(rows, cols).ctas) return 0;
  const uint32_t parts = kGradParts * grad_shape(cols).groups;
  return rows < parts ? rows : parts;
}

namespace {

template <typename K>
int grad_few(K kernel, const GradArgs &a, const Shape &s, const Few &few, cudaStream_t stream) {
  const uint32_t bytes = (2 * few.groups * (s.threads / 32) + few.groups * a.cols) * sizeof(float);
  int e = (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (!e && few.ctas > 8) e = (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e) return e;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim = {few.ctas, 1, 1};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(few.ctas);
  cfg.blockDim = dim3(s.threads, few.groups);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return (int)cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace

int launch_rms_norm_grad(const NormGradArgs &n, unsigned sms, void *stream) {
  GradArgs a = {};
  a.dout = n.dout, a.x = n.x, a.weight = n.weight, a.dresidual = n.dresidual, a.rstd = n.rstd, a.dx = n.dx;
  a.partial = n.dweight ? n.work : nullptr;
  a.dout_pitch = n.dout_pitch, a.pitch = n.pitch, a.dresidual_pitch = n.dresidual_pitch, a.dx_pitch = n.dx_pitch;
  a.rows = n.rows, a.cols = n.cols, a.wdtype = n.wdtype;
  const Few few = n.dweight ? few_of(n.rows, n.cols) : Few{0, 0};
  a.parts = few.ctas ? few.ctas : n.rows < kGradParts ? n.rows : kGradParts;
  if (few.ctas) a.partial = nullptr, a.dweight = n.dweight, a.dwdtype = n.dwdtype;
  a.weight_aligned = (uintptr_t)n.weight % 16 == 0;
  a.inv_cols = (float)(1.0 / n.cols);
  cudaStream_t s = (cudaStream_t)stream;
  const Shape sh = grad_shape(n.cols);
  const int e = !n.rows ? 0 : with_dtype(n.dtype, [&](auto t) {
    using T = decltype(t);
    const auto at = [](const void *p, int64_t pitch) { return aligned(p, pitch * (int64_t)sizeof(T)); };
    if (!sh.fits) {
      grad_long_kernel<T><<<grid_of(n.rows, 1), 1024, 0, s>>>(a);
      const int e = (int)cudaGetLastError();
      if (e || !a.partial) return e;
      return launch_after(grad_long_parts_kernel<T>, grid_of((uint64_t)((n.cols + 255) / 256) * a.parts, 8), 256, 0, s, a);
    }
    const auto alike = [&](const void *p, int64_t pitch) {
      return same_place(n.x, n.pitch * (int64_t)sizeof(T), p, pitch * (int64_t)sizeof(T));
    };
    const RingShape ring = ring_shape(n.x, n.pitch, n.rows, n.cols, sizeof(T), n.dresidual ? 3 : 2, 2 * sms, true,
                                      alike(n.dout, n.dout_pitch) && alike(n.dresidual, n.dresidual_pitch) && alike(n.dx, n.dx_pitch),
                                      n.cols >= 2048 && n.cols <= 8192);
    if constexpr (sizeof(T) == 2) if (ring.threads && !few.ctas) {
      a.parts = n.dweight ? rms_norm_parts(n.rows, n.cols) : n.rows;
      const uint32_t period = period_of(n.pitch * (int64_t)sizeof(T));
      if (ring.whole)
        return ring.v == 1 ? ring_launch(ring_grad_kernel<T, 1, true>, a, ring, a.parts, period, stream)
                           : ring_launch(ring_grad_kernel<T, 4, true>, a, ring, a.parts, period, stream);
      return ring.v == 1 ? ring_launch(ring_grad_kernel<T, 1, false>, a, ring, a.parts, period, stream)
                         : ring_launch(ring_grad_kernel<T, 4, false>, a, ring, a.parts, period, stream);
    }
    const bool wide = at(n.x, n.pitch) && at(n.dout, n.dout_pitch) && at(n.dresidual, n.dresidual_pitch) && at(n.dx, n.dx_pitch);
    const auto with_shape = [&](auto f) {
      if (sh.v == 1) return wide ? f(grad_kernel<T, 1, 4, true, false>, grad_kernel<T, 1, 4, true, true>)
                                 : f(grad_kernel<T, 1, 4, false, false>, grad_kernel<T, 1, 4, false, true>);
      if (sh.threads == 32) return wide ? f(grad_kernel<T, 2, 2, true, false>, grad_kernel<T, 2, 2, true, true>)
                                        : f(grad_kernel<T, 2, 2, false, false>, grad_kernel<T, 2, 2, false, true>);
      if (sh.v == 2) return wide ? f(grad_kernel<T, 2, 1, true, false>, grad_kernel<T, 2, 1, true, true>)
                                 : f(grad_kernel<T, 2, 1, false, false>, grad_kernel<T, 2, 1, false, true>);
      return wide ? f(grad_kernel<T, 4, 1, true, false>, grad_kernel<T, 4, 1, true, true>)
                  : f(grad_kernel<T, 4, 1, false, false>, grad_kernel<T, 4, 1, false, true>);
    };
    if (few.ctas) return with_shape([&](auto, auto kernel) { return grad_few(kernel, a, sh, few, s); });
    const uint32_t room = (2 * sh.groups * (sh.threads / 32) + (sh.groups > 1 ? sh.groups * n.cols : 0)) * sizeof(float);
    return with_shape([&](auto kernel, auto) {
      kernel<<<grid_of(a.parts, 2), dim3(sh.threads, sh.groups), room, s>>>(a);
      return (int)cudaGetLastError();
    });
  });
  if (e || !n.dweight || few.ctas) return e;
  const unsigned grid = grid_of((n.cols + 31) / 32, 4);
  const float *work = n.work;
  if (n.rows) return launch_after(parts_kernel, grid, 512, 0, s, work, a.parts, n.cols, n.dweight, n.dwdtype);
  parts_kernel<<<grid, 512, 0, s>>>(work, a.parts, n.cols, n.dweight, n.dwdtype);
  return (int)cudaGetLastError();
}

}  // namespace apc
