// The root-mean-square norm with the residual's addition (apc_rms_norm,
// apc_rms_norm_fp8).
//
//   h    = x + residual, rounded to x's type          (the residual stream)
//   rstd = 1 / sqrt(mean of h^2 + eps)
//   y    = (h * rstd) * weight, in fp32, then rounded or quantized
//
// One read of each input and one write of each output, a few operations for each
// element: bound by memory.  A row is spread over the threads of a group, 8 elements
// each in one or two places, and stays in registers between its statistics and its
// output.
#include "apc_rmsnorm.cuh"

namespace apc {

namespace {

// ---------------------------------------------------------------------------
// A row's sum of squares and its rstd.  Blocks are quantized by their largest value,
// so a last bit of rstd can turn a scale, and the roundings of a whole row with it: rstd is
// rounded once, from a sum that is within 2^-38 of itself, however the row lies over the threads.
// Layouts then differ only in rows at a rounding's border: in none of 12 million, aligned rows
// against rows at odd places and few against many.  The 2^-38 are the worst that 32 threads'
// roundings to the warp's integers can do.  A thread adds its squares in pairs of floats, the
// second of which holds what the first one's additions lost (D. Knuth's sum, The Art of
// Computer Programming 2, 4.2.2): 30 instructions for 8 squares, 7 without.  Threads' sums
// are added as integers, of 26 bits under the largest of a warp and 20 behind: integer
// additions across a warp are one instruction where five shuffles and additions of such
// pairs took 50.

constexpr uint32_t kLeast = 32;  // least e: 2^-120 of the sum, far below eps

struct Two {
  float hi, lo;
};

__device__ __forceinline__ Two operator+(Two a, Two b) {
  const float s = __fadd_rn(a.hi, b.hi), t = __fsub_rn(s, a.hi);
  return {s, __fadd_rn(__fadd_rn(a.lo, b.lo), __fadd_rn(__fsub_rn(a.hi, __fsub_rn(s, t)), __fsub_rn(b.hi, t)))};
}

__device__ __forceinline__ uint64_t sub2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// a + b rounded; err: what that lost.
__device__ __forceinline__ float two_sum(float a, float b, float *err) {
  const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
  *err = __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t));
  return s;
}

// A thread's sum over the many parts of a long row.  The second float of a pair that is only
// added to grows with every addition: where the values are alike it passed what warp_stat's
// integers hold, from 600,000 columns on.  So it goes back into the first after each addition,
// and what the second one's additions lose is kept too: a sum of 2^17 parts (2^31 columns) is
// then off by 2^-39 of itself at most, and by 2^-46 of 2^10 parts of one value.
struct LongSum {
  float hi = 0.0f, lo = 0.0f, rest = 0.0f;

  __device__ __forceinline__ void add(Two b) {
    float e[3];
    const float s = two_sum(hi, b.hi, &e[0]);
    const float l = two_sum(two_sum(lo, e[0], &e[1]), b.lo, &e[2]);
    rest = __fadd_rn(rest, __fadd_rn(e[1], e[2]));
    hi = __fadd_rn(s, l);
    lo = __fsub_rn(l, __fsub_rn(hi, s));
  }
  __device__ __forceinline__ Two sum() const { return {hi, __fadd_rn(lo, rest)}; }
};

// The sum of two pairs, lane by lane; err: what it lost.
__device__ __forceinline__ uint64_t two_sum2(uint64_t a, uint64_t b, uint64_t *err) {
  const uint64_t s = add2(a, b), t = sub2(s, a);
  *err = add2(sub2(a, sub2(s, t)), sub2(b, t));
  return s;
}

// The squares of eight elements, each times `scale`.
template <typename T, bool SCALED = false>
__device__ __forceinline__ Two squares(const uint32_t (&w)[8 / Word<T>::kPer], float scale = 1.0f) {
  uint64_t p[4], lost = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint64_t v = pack2(element<T>(w, 2 * i), element<T>(w, 2 * i + 1));
    if (SCALED) v = mul2(v, pack2(scale, scale));
    p[i] = mul2(v, v);  // exact for 16 bits
    if (sizeof(T) == 4) lost = add2(lost, fma2(v, v, p[i] ^ 0x8000000080000000ull));
  }
  uint64_t e[3];
  const uint64_t s = two_sum2(two_sum2(p[0], p[1], &e[0]), two_sum2(p[2], p[3], &e[1]), &e[2]);
  lost = add2(add2(e[0], e[1]), sizeof(T) == 4 ? add2(e[2], lost) : e[2]);
  const float2 a = unpack2(s), b = unpack2(lost);
  return Two{a.x, b.x} + Two{a.y, b.y};
}

// A warp's sum of its threads' sums.
__device__ __forceinline__ Stat warp_stat(Two p) {
  const uint32_t top = __reduce_max_sync(~0u, __float_as_uint(p.hi) & 0x7fffffffu);
  const uint32_t e = max(top >> 23, kLeast);
  if (e == 255) return {0, 255, 0};
  const float f = __uint_as_float((279 - e) << 23), t = p.hi * f;  // below 2^26
  const uint32_t i = __float2uint_rn(t);
  const int32_t low = __float2int_rn((__fsub_rn(t, (float)i) + p.lo * f) * 0x1p20f);
  return {__reduce_add_sync(~0u, i), e, (int32_t)__reduce_add_sync(~0u, (uint32_t)low)};
}

struct NormConst {
  float inv_hi, inv_lo, eps_hi, eps_lo;  // 1/cols and eps in two parts

  // for rows whose elements are taken times `scale`, a power of two
  __device__ __forceinline__ NormConst scaled(float scale) const {
    return {inv_hi, inv_lo, eps_hi * scale * scale, eps_lo * scale * scale};
  }
};

// 1 / sqrt((hi + lo) * 2^k / cols + eps), rounded to nearest but for one in some 2^20.
__device__ __forceinline__ float rstd_of(float hi, float lo, int k, const NormConst &c) {
  const float two_k = __uint_as_float((uint32_t)(k + 127) << 23);
  float m = hi * c.inv_hi, rest = __fmaf_rn(hi, c.inv_hi, -m);
  rest += hi * c.inv_lo + lo * c.inv_hi;
  m *= two_k, rest *= two_k;
  const float top = fmaxf(m, c.eps_hi);  // mean and eps may be large enough for their sum to overflow
  const float move = top > 0x1p60f ? 0x1p-80f : top < 0x1p-60f ? 0x1p80f : 1.0f;
  const float back = top > 0x1p60f ? 0x1p-40f : top < 0x1p-60f ? 0x1p40f : 1.0f;
  m *= move, rest *= move;
  const float eps = c.eps_hi * move, s = m + eps, b = s - m;
  rest += ((m - (s - b)) + (eps - b)) + c.eps_lo * move;
  m = s;
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

// rstd of a row whose threads' sums of squares are p; false: a sum is not finite.
__device__ __forceinline__ bool row_rstd(Two p, const Group &g, Stat *room, const NormConst &c, float *rstd) {
  Stat s = warp_stat(p);
  float hi, lo;
  if (g.warps == 1) {
    if (s.e == 255) return false;
    split_sum(s.sum, hi, lo);
    lo += (float)s.low * 0x1p-20f;
    *rstd = rstd_of(hi, lo, (int)s.e - 152, c);
    return true;
  }
  if (g.lane == 0) room[g.warp] = s;
  if (g.warp == 0) {  // the others wait for one warp's work instead of doing it too
    g.sync();
    s = g.lane < g.warps ? room[g.lane] : Stat{0, kLeast, 0};
    const uint32_t e = __reduce_max_sync(~0u, s.e);
    const int64_t v = (((int64_t)s.sum << 20) + s.low) >> min(e - s.e, 63u);
    const uint32_t high = __reduce_add_sync(~0u, (uint32_t)(v >> 26)), low = __reduce_add_sync(~0u, (uint32_t)v & 0x3ffffffu);
    split_sum(high, hi, lo);
    lo += (float)low * 0x1p-26f;
    const float r = rstd_of(hi, lo, (int)min(e, 254u) - 146, c);
    if (g.lane == 0) room[g.warps] = {__float_as_uint(r), e, 0};
  } else {
    g.arrive();
  }
  g.sync_again();
  s = room[g.warps];
  *rstd = __uint_as_float(s.sum);
  return s.e != 255;
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
__device__ __forceinline__ uint32_t largest(const uint32_t (&w)[8 / Word<T>::kPer]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(element<T>(w, i)) & 0x7fffffffu);
  return m;
}

// rstd of a row some of whose threads' sums are not finite: infinities and NaNs, or
// squares beyond the largest number, which are taken scaled, and eps too.
template <typename T, int V>
__device__ __forceinline__ float wild_rstd(const uint32_t (&w)[V][8 / Word<T>::kPer], const Group &g, Stat *room, const NormConst &c) {
  uint32_t m = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) m = max(m, largest<T>(w[v]));
  m = group_max(m, g, room);
  if (m >= 0x7f800000u) return m > 0x7f800000u ? __uint_as_float(0x7fffffffu) : 0.0f;
  const float scale = __uint_as_float(max(254u - (m >> 23), 1u) << 23);
  Two p = {0.0f, 0.0f};
  float rstd;
#pragma unroll
  for (int v = 0; v < V; ++v) p = p + squares<T, true>(w[v], scale);
  row_rstd(p, g, room, c.scaled(scale), &rstd);
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
  uint32_t then;  // the transpose's kernel follows, and may start: 1 at once, 2 as CTAs end
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
      if constexpr (WIDE) {
#pragma unroll
        for (int o = 8; o; o >>= 1) v = max(v, __shfl_xor_sync(~0u, v, o));
        return v;
      } else {
        return __reduce_max_sync(~0u, v);
      }
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
      if (n == 8) __stcs(reinterpret_cast<uint2 *>(at), to_fp8x8<E5M2>(y, pack2(inv, inv)));
      else if (n) store8(at, to_fp8x8<E5M2>(y, pack2(inv, inv)), n);
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
  extern __shared__ Stat s_room[];  // [2][groups][warps + 1]
  const Group g{blockDim.x / 32, 1 + threadIdx.y, threadIdx.x / 32, threadIdx.x % 32};
  if (a.then == 1) start_next();
  const uint32_t groups = (LONG ? (a.cols + 255) / 256 : V * g.warps);  // runs of 256 columns
  uint32_t turn = 0;
  for (uint64_t row = (uint64_t)blockIdx.x * blockDim.y + threadIdx.y; row < a.rows; row += (uint64_t)gridDim.x * blockDim.y) {
    const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.pitch;
    const T *res = static_cast<const T *>(a.residual) + (int64_t)row * a.residual_pitch;
    T *sum = static_cast<T *>(a.sum) + (int64_t)row * a.sum_pitch;
    Stat *room = s_room + ((turn ^= 1) * blockDim.y + threadIdx.y) * (g.warps + 1);
    uint32_t w[V][kWords];
    // the sum's elements of V runs from `run` on, as they are stored.  All loads stand in front
    // of the stores, which they might not pass (1200 x 16384 bf16 32.4 us, 36.9 in turns), but for
    // aligned fp32 rows to fp32, which do as well or better with fewer under way: 8192 x 4096 82.3 us
    // (92.7), though 2441 x 8192 56.5 (52.7).
    constexpr bool kTurns = sizeof(T) == 4 && OUT == kSame && WIDE && !LONG;
    const auto fetch = [&](uint32_t run, bool again) {
      const bool adds = !again && a.residual;
      uint32_t c[V], o[V][kWords];
      int n[V];
      const auto add = [&](int v) {
        add_rounded<T>(w[v], o[v]);
        store<T, WIDE>(sum + c[v], w[v], n[v]);
      };
#pragma unroll
      for (int v = 0; v < V; ++v) {
        c[v] = first_of<WIDE>(run + v * g.warps, g.lane);
        n[v] = count_of<WIDE>(c[v], a.cols);
        load<T, WIDE>(w[v], (again && a.residual ? sum : x) + c[v], n[v]);
        if (!kTurns || !adds) continue;
        load<T, WIDE>(o[v], res + c[v], n[v]);
        add(v);
      }
      if (kTurns || !adds) return;
#pragma unroll
      for (int v = 0; v < V; ++v) load<T, WIDE>(o[v], res + c[v], n[v]);
#pragma unroll
      for (int v = 0; v < V; ++v) add(v);
    };
    const auto over_row = [&](bool again, auto f) {  // f() for each part that the registers hold
      if constexpr (LONG) {
        for (uint32_t run = 0; run < groups; run += V * g.warps) {
          fetch(run + g.warp, again);
          f(run);
        }
      } else {
        f(0u);
      }
    };
    if (!LONG) fetch(g.warp, false);
    // the sum of squares over the row
    const auto sum_of = [&](bool again, auto square) {
      LongSum all;
      Two p;
      over_row(again, [&](uint32_t) {
#pragma unroll
        for (int v = 0; v < V; ++v) p = v ? p + square(w[v]) : square(w[v]);
        if (LONG) all.add(p);
      });
      return LONG ? all.sum() : p;
    };
    float rstd;
    if (!row_rstd(sum_of(false, [](const auto &x) { return squares<T>(x); }), g, room, a.c, &rstd)) {
      uint32_t m = 0;
      over_row(true, [&](uint32_t) {
#pragma unroll
        for (int v = 0; v < V; ++v) m = max(m, largest<T>(w[v]));
      });
      m = group_max(m, g, room);
      if (m >= 0x7f800000u) {
        rstd = m > 0x7f800000u ? __uint_as_float(0x7fffffffu) : 0.0f;
      } else {  // squares beyond the largest number
        const float scale = __uint_as_float(max(254u - (m >> 23), 1u) << 23);
        row_rstd(sum_of(true, [&](const auto &x) { return squares<T, true>(x, scale); }), g, room, a.c.scaled(scale), &rstd);
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
  if (a.then == 1) start_next();
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
      Two p;
#pragma unroll
      for (int v = 0; v < V; ++v) p = v ? p + squares<T>(w[u][v]) : squares<T>(w[u][v]);
      if (!row_rstd(p, g, nullptr, a.c, &rstd[u])) rstd[u] = wild_rstd<T, V>(w[u], g, nullptr, a.c);
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

// The transpose in 8 bits, from the sum and rstd that the forward kernel left: that one may still
// run when this one starts, so they are read from L2 (cp.async.cg, ld.cg), behind the wait.  A CTA walks
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
    } else if (a.wide) {  // zeros where there is nothing
      const int n = c < a.cols ? (int)min(8u, a.cols - c) * (int)sizeof(T) : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i, h += 16 * a.pitch)
#pragma unroll
        for (int j = 0; j < kWords; j += 4) {
          const int bytes = r + 16 * i < a.rows ? min(max(n - 4 * j, 0), 16) : 0;
          copy_block(smem_addr(to) + i * 16 * kPitch + 4 * j, bytes ? reinterpret_cast<const uint8_t *>(h) + 4 * j : a.h, bytes);
        }
    } else {
      const int n = c < a.cols ? (int)min(8u, a.cols - c) : 0;
#pragma unroll 4
      for (int i = 0; i < 8; ++i, h += 16 * a.pitch, to += 16 * kPitch) {
        uint32_t w[kWords];
        load8<T, Read::kL2>(w, h, r + 16 * i < a.rows ? n : 0, false);
#pragma unroll
        for (int j = 0; j < kWords; j += 4) *reinterpret_cast<uint4 *>(to + 4 * j) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
      }
    }
    if (threadIdx.x < 128) {
      const uint32_t k = tr * kBlock + threadIdx.x;
      sh.rstd[threadIdx.x] = k < a.rows ? __ldcg(a.rstd + k) : 0.0f;
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
        __stcs(reinterpret_cast<uint2 *>(to), sh.turn[k * 16 + (tx ^ k / 8)]);
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
  if (a.then == 1) start_next();
  const Source src[2] = {{a.x, a.pitch}, {a.residual, a.residual_pitch}};
  uint32_t next = blockIdx.x, into = 0, issued = 0;  // the row to copy next, its stage; rows so far
  const auto issue = [&]() {
    if (next < a.rows) {
      issued += ring_issue<2>(sh, src, ring, s_ring + into * ring.stage(), &sh.full[into], next, a.rows, a.cols, sizeof(T), l2_evict_first());
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
    Two p;
    float rstd;
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
      p = v ? p + squares<T>(w[v]) : squares<T>(w[v]);
    }
    // before the next copy into a stage that was written here
    if (OUT != kSame && skip) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    const bool fine = row_rstd(p, g, sh.stats[turn ^= 1], a.c, &rstd);
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
  ring_end(sh, ring.stages, issued);
  if (a.then == 2) start_next();
}

// From so many rows on a warp takes several at a time.
constexpr uint32_t kNarrowRows = 1024;

template <typename T, int OUT, int V, bool WIDE, bool LONG>
int forward_launch(const ForwardArgs &a, const Shape &s, void *stream) {
  const uint32_t per = s.threads * s.groups;
  const unsigned grid = grid_of((a.rows + s.groups - 1) / s.groups, 2048 / per);
  const size_t room = sizeof(Stat) * 2 * (per / 32 + s.groups);
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
  // with much to transpose CTAs that wait would be in the way (8192 x 4096: 72 us, 64 so)
  a.then = !n.qt.data ? 0 : (uint64_t)n.rows * n.cols <= 1u << 21 ? 1 : 2;
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
                                      true);
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


}  // namespace apc
