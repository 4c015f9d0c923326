// Distillation from a teacher's largest logits: loss and gradient
// (apc_distill_loss, apc_distill_grad, apc_distill_loss_grad).
//
// With m the row's largest logit,
//   S = sum of exp((z - m)/tau),  log q_i = (z_i - m)/tau - log S
//   dz = c0/S exp((z - m)/tau) + (the same at tau = 1 for the labels) - p
// The difference comes before the scaling: it is exact near m, where the sums
// are made, and logits at their type's lowest value do not overflow.  Elements
// go through in pairs, two fp32 lanes an instruction.
//
// A row belongs to one CTA or, where rows are few or long, to a cluster whose
// CTAs exchange maxima and sums.  Its logits are read once: they stay in
// registers between the normaliser and the gradient where they fit (kVectors of
// 16 bytes a thread), else the second sweep reads them again.  One extra warp
// works on the teacher's few entries, a row ahead.
#include <cuda_runtime.h>

#include "apc_ops.cuh"
#include "apc_tcgen05.cuh"

namespace apc {

namespace {

#ifndef APC_DISTILL_WORKERS
#define APC_DISTILL_WORKERS 256
#endif
#ifndef APC_DISTILL_KEEP
#define APC_DISTILL_KEEP 16
#endif
#ifndef APC_DISTILL_STREAM
#define APC_DISTILL_STREAM 8
#endif
#ifndef APC_DISTILL_STREAM_CTAS
#define APC_DISTILL_STREAM_CTAS 4
#endif
constexpr int kWorkers = APC_DISTILL_WORKERS, kThreads = kWorkers + 32, kWarps = kWorkers / 32;
// Vectors of 16 bytes that a thread holds, and CTAs on an SM: the rows that stay
// in registers, and the forms that pass over the logits once.
constexpr int kKeep = APC_DISTILL_KEEP, kStream = APC_DISTILL_STREAM;
constexpr int residents(int form) { return form == 3 ? 2 : APC_DISTILL_STREAM_CTAS; }
constexpr int kSlots = 2048;  // of the table that finds equal ids
constexpr int kMaxSplit = 8;
constexpr float kInf = __builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The largest logit m and the sums of exp((z - m)/tau) and exp(z - m).
struct Sum {
  float m, s, s1;
};

// What z's difference is taken to: m, or 0 where every logit is -infinity.
__device__ __forceinline__ float reference(float m) { return m == -kInf ? 0.0f : m; }

// A sum about `from` as one about `to`, the larger.
__device__ __forceinline__ float moved(float s, float from, float to, float scale) {
  return s * exp2_approx((from - reference(to)) * scale);
}

template <bool TWO>
__device__ __forceinline__ void join(Sum &a, const Sum &b, float scale) {
  const float t = fmaxf(a.m, b.m);
  a.s = moved(a.s, a.m, t, scale) + moved(b.s, b.m, t, scale);
  if (TWO) a.s1 = moved(a.s1, a.m, t, kLog2e) + moved(b.s1, b.m, t, kLog2e);
  a.m = t;
}

// Over the lanes of a warp (or the first `lanes` of them), the same in each.
template <bool TWO>
__device__ __forceinline__ Sum joined(Sum a, float scale, int lanes = 32) {
  float t = a.m;
  for (int o = lanes / 2; o; o >>= 1) t = fmaxf(t, __shfl_xor_sync(~0u, t, o));
  a.s = moved(a.s, a.m, t, scale);
  if (TWO) a.s1 = moved(a.s1, a.m, t, kLog2e);
  for (int o = lanes / 2; o; o >>= 1) {
    a.s += __shfl_xor_sync(~0u, a.s, o);
    if (TWO) a.s1 += __shfl_xor_sync(~0u, a.s1, o);
  }
  a.m = t;
  return a;
}

// What the teacher's warp leaves of a row's entries; the label is entry k.
struct Entries {
  int32_t id[APC_DISTILL_MAX_K + 1];  // -1: does not count
  float p[APC_DISTILL_MAX_K + 1];     // the probability; the label's is 1
  float z[APC_DISTILL_MAX_K + 1];     // the student's logit there
  float p_sum, entropy;               // sum of p and of p log p
  int32_t same;                       // some place occurs twice
};

struct Shared {
  Entries e[2];
  __align__(16) int32_t slot[kSlots];
  Sum part[2][kWarps];
  Sum peer[2][kMaxSplit];
};

__device__ __forceinline__ int64_t index_at(const void *p, bool wide, int64_t i) {
  return wide ? static_cast<const int64_t *>(p)[i] : static_cast<const int32_t *>(p)[i];
}

__device__ __forceinline__ float number_at(const void *p, uint32_t dtype, int64_t i) {
  return dtype == APC_F32 ? static_cast<const float *>(p)[i]
         : dtype == APC_BF16 ? to_float(static_cast<const __nv_bfloat16 *>(p)[i])
                             : to_float(static_cast<const __half *>(p)[i]);
}

// One warp: the entries of a row.  Equal ids are looked for with a table of the
// ids by hash.
template <typename T>
__device__ void teacher_entries(const DistillArgs &a, uint32_t row, Entries &e, int32_t *slot, uint32_t lane) {
  const T *z = static_cast<const T *>(a.logits) + (int64_t)row * a.pitch;
  float top = -kInf;
  for (uint32_t i = lane; i < a.k; i += 32) {
    const int64_t id = index_at(a.ids, a.ids64, (int64_t)row * a.ids_pitch + i);
    const float u = number_at(a.teacher, a.teacher_dtype, (int64_t)row * a.teacher_pitch + i);
    const bool counts = id >= 0 && id < (int64_t)a.vocab && u != -kInf;
    e.id[i] = counts ? (int32_t)id : -1;
    e.p[i] = counts ? u : -kInf;
    e.z[i] = counts ? to_float(z[id]) : 0.0f;
    if (counts) top = fmaxf(top, u);
  }
  if (lane == 0) {
    int64_t y = a.labels ? index_at(a.labels, a.labels64, row) : -1;
    if (y >= (int64_t)a.vocab || y < 0) y = -1;
    e.id[a.k] = (int32_t)y;
    e.p[a.k] = 1.0f;
    e.z[a.k] = y >= 0 ? to_float(z[y]) : 0.0f;
  }
  for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
  float norm = 0.0f;
  if (a.teacher_lse) {
    top = 0.0f;
    norm = a.teacher_lse[row];
  } else {
    if (top == -kInf) top = 0.0f;
    float s = 0.0f;
    for (uint32_t i = lane; i < a.k; i += 32) s += exp2f((e.p[i] - top) * a.scale2);
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    norm = logf(s);
  }
  float p_sum = 0.0f, entropy = 0.0f;
  for (uint32_t i = lane; i < a.k; i += 32) {
    const float lp = e.id[i] >= 0 ? __fmaf_rn(e.p[i] - top, a.inv_tau, -norm) : -kInf, p = expf(lp);
    e.p[i] = p;
    p_sum += p;
    if (p != 0.0f) entropy = __fmaf_rn(p, lp, entropy);
  }
  for (int o = 16; o; o >>= 1) {
    p_sum += __shfl_xor_sync(~0u, p_sum, o);
    entropy += __shfl_xor_sync(~0u, entropy, o);
  }
  if (lane == 0) e.p_sum = p_sum, e.entropy = entropy;
  if (!a.dlogits) return;
  for (uint32_t i = lane; i < kSlots / 4; i += 32) reinterpret_cast<int4 *>(slot)[i] = make_int4(-1, -1, -1, -1);
  __syncwarp();
  bool same = false;
  for (uint32_t i = lane; i <= a.k; i += 32) {
    const int32_t id = e.id[i];
    if (id < 0) continue;
    for (uint32_t h = (uint32_t)id * 2654435761u >> 21;; h = (h + 1) % kSlots) {  // at most half full
      const int32_t was = atomicCAS(&slot[h], -1, id);
      same |= was == id;
      if (was == -1 || was == id) break;
    }
  }
  same = __any_sync(~0u, same);
  if (lane == 0) e.same = same;
}

// Words of T: a pair of 16 bits or one of 32.
template <typename T>
__device__ __forceinline__ float2 widen(uint32_t w);
template <>
__device__ __forceinline__ float2 widen<__nv_bfloat16>(uint32_t w) {
  return {__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
}
template <>
__device__ __forceinline__ float2 widen<__half>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}

template <typename T>
__device__ __forceinline__ uint32_t narrow(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t narrow<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
template <>
__device__ __forceinline__ uint32_t narrow<__half>(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}

// Pair i of a vector, as two fp32 lanes.
template <typename T>
__device__ __forceinline__ uint64_t pair(const uint4 &v, int i) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if constexpr (sizeof(T) == 4) {
    return pack2(w[2 * i], w[2 * i + 1]);
  } else {
    const float2 x = widen<T>(w[i]);
    return pack2(x.x, x.y);
  }
}

// 2^x of both lanes.
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x) {
  const float2 v = unpack2(x);
  return pack2(exp2_approx(v.x), exp2_approx(v.y));
}

// The vector of f's results on the pairs.
template <typename T, typename F>
__device__ __forceinline__ uint4 map(const uint4 &v, F f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 8 / (int)sizeof(T); ++i) {
    const float2 y = unpack2(f(pair<T>(v, i)));
    if constexpr (sizeof(T) == 4) w[2 * i] = __float_as_uint(y.x), w[2 * i + 1] = __float_as_uint(y.y);
    else w[i] = narrow<T>(y.x, y.y);
  }
  return {w[0], w[1], w[2], w[3]};
}

// The largest element of a vector and m.
template <typename T>
__device__ __forceinline__ uint32_t word_max(uint32_t a, uint32_t b);
template <>
__device__ __forceinline__ uint32_t word_max<__nv_bfloat16>(uint32_t a, uint32_t b) {
  const __nv_bfloat162 v = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
  return *reinterpret_cast<const uint32_t *>(&v);
}
template <>
__device__ __forceinline__ uint32_t word_max<__half>(uint32_t a, uint32_t b) {
  const __half2 v = __hmax2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
  return *reinterpret_cast<const uint32_t *>(&v);
}
template <>
__device__ __forceinline__ uint32_t word_max<float>(uint32_t a, uint32_t b) {
  return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
}

template <typename T, int N>
__device__ __forceinline__ float largest(const uint4 (&x)[N]) {
  uint4 m = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) {
    m.x = word_max<T>(m.x, x[i].x), m.y = word_max<T>(m.y, x[i].y);
    m.z = word_max<T>(m.z, x[i].z), m.w = word_max<T>(m.w, x[i].w);
  }
  const uint32_t w = word_max<T>(word_max<T>(m.x, m.y), word_max<T>(m.z, m.w));
  if constexpr (sizeof(T) == 4) {
    return __uint_as_float(w);
  } else {
    const float2 y = widen<T>(w);
    return fmaxf(y.x, y.y);
  }
}

// Nothing known of the words beyond this point: they are widened anew, not kept wide.
template <int N>
__device__ __forceinline__ void forget(uint4 (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(x[i].x), "+r"(x[i].y), "+r"(x[i].z), "+r"(x[i].w));
}

// A vector of elements that leave every maximum and sum alone.
template <typename T>
__device__ __forceinline__ uint4 nothing() {
  const uint32_t w = sizeof(T) == 4 ? 0xff800000u : sizeof(T) == 2 && __is_same(T, __half) ? 0xfc00fc00u : 0xff80ff80u;
  return {w, w, w, w};
}

// FORM: 1 loss, 2 gradient, 3 both.  TWO: the labels need the sums at tau = 1
// beside those at tau.
template <typename T, int FORM, bool TWO>
__global__ void __launch_bounds__(kThreads, FORM == 3 ? 2 : APC_DISTILL_STREAM_CTAS)
    distill_kernel(const __grid_constant__ DistillArgs a, const uint32_t split, const bool alike) {
  extern __shared__ __align__(16) uint8_t raw[];
  Shared &sh = *reinterpret_cast<Shared *>(raw);
  constexpr int kPer = 16 / sizeof(T);
  constexpr bool kLoss = FORM & 1, kGrad = FORM & 2;
  constexpr int kVectors = FORM == 3 ? kKeep : kStream;
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const uint32_t rank = split > 1 ? blockIdx.x % split : 0, first = blockIdx.x / split, step = gridDim.x / split;
  const bool together = kLoss && split > 1;  // the CTAs of a row are a cluster
  const bool worker = warp < kWarps;
  if (!worker && first < a.rows) teacher_entries<T>(a, first, sh.e[0], sh.slot, lane);
  uint32_t turn = 0;
  for (uint32_t row = first; row < a.rows; row += step, turn ^= 1) {
    const T *z = static_cast<const T *>(a.logits) + (int64_t)row * a.pitch;
    // vectors [v0, v1) of the 16-byte aligned body are this CTA's; the elements
    // outside the body are the first CTA's, one a thread
    const uint32_t head = min(a.vocab, (uint32_t)((16 - (uintptr_t)z % 16) % 16 / sizeof(T)));
    const uint32_t body = (a.vocab - head) / kPer, odd = a.vocab - body * kPer;
    const uint32_t v0 = (uint32_t)((uint64_t)body * rank / split), v1 = (uint32_t)((uint64_t)body * (rank + 1) / split);
    const uint4 *zv = reinterpret_cast<const uint4 *>(z + head);
    const bool has_odd = worker && rank == 0 && tid < odd;
    const uint32_t odd_at = tid < head ? tid : body * kPer + tid;
    const bool keeps = v1 - v0 <= kWorkers * kVectors;  // the row stays in registers
    uint4 x[kVectors];
    float x_odd = -kInf;
    auto load = [&](uint32_t at) {
#pragma unroll
      for (int i = 0; i < kVectors; ++i) {
        const uint32_t v = at + i * kWorkers + tid;
        x[i] = v < v1 ? __ldcs(zv + v) : nothing<T>();
      }
    };
    if (worker) {
      load(v0);
      if (has_odd) x_odd = to_float(z[odd_at]);
    }
    Sum sum = {-kInf, 0.0f, 0.0f};
    if (kLoss) {
      if (worker) {
        sum.m = x_odd;
        for (uint32_t at = v0;;) {
          const float m = fmaxf(sum.m, largest<T>(x));
          if (at != v0) {
            sum.s = moved(sum.s, sum.m, m, a.scale2);
            if (TWO) sum.s1 = moved(sum.s1, sum.m, m, kLog2e);
          }
          sum.m = m;
          const float from = reference(m);
          const uint64_t minus = pack2(-from, -from), scale = pack2(a.scale2, a.scale2), scale1 = pack2(kLog2e, kLog2e);
          if (at == v0 && has_odd) {
            sum.s += exp2_approx((x_odd - from) * a.scale2);
            if (TWO) sum.s1 += exp2_approx((x_odd - from) * kLog2e);
          }
          uint64_t part = 0, part1 = 0;
#pragma unroll
          for (int i = 0; i < kVectors; ++i) {
#pragma unroll
            for (int j = 0; j < 8 / (int)sizeof(T); ++j) {
              const uint64_t y = add2(pair<T>(x[i], j), minus);
              part = add2(part, exp2_pair(mul2(y, scale)));
              if (TWO) part1 = add2(part1, exp2_pair(mul2(y, scale1)));
            }
          }
          const float2 u = unpack2(part), u1 = unpack2(part1);
          sum.s += u.x + u.y;
          if (TWO) sum.s1 += u1.x + u1.y;
          at += kWorkers * kVectors;
          if (at >= v1) break;
          load(at);
        }
        sum = joined<TWO>(sum, a.scale2);
        if (lane == 0) sh.part[turn][warp] = sum;
      }
      __syncthreads();
      sum = joined<TWO>(sh.part[turn][lane % kWarps], a.scale2, kWarps);
      if (together) {
        if (tid < split) {
          const uint32_t at = map_rank(smem_addr(&sh.peer[turn][rank]), tid);
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(sum.m) : "memory");
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 4), "f"(sum.s) : "memory");
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 8), "f"(sum.s1) : "memory");
        }
        cluster_arrive(), cluster_wait();
        sum = sh.peer[turn][0];
        for (uint32_t k = 1; k < split; ++k) join<TWO>(sum, sh.peer[turn][k], a.scale2);
      }
    } else {
      __syncthreads();
    }
    const Entries &en = sh.e[turn];
    const float from = reference(sum.m);
    const float log_s = kLoss ? log2f(sum.s) : 0.0f, log_s1 = kLoss ? (TWO ? log2f(sum.s1) : log_s) : 0.0f;
    if (!worker) {
      // the row's loss, then the next row's entries
      if (kLoss && rank == 0) {
        const bool some = sum.m != -kInf || sum.s != 0.0f;
        float cross = 0.0f;
        for (uint32_t i = lane; i < a.k; i += 32)
          if (en.p[i] != 0.0f) cross = __fmaf_rn(en.p[i], (en.z[i] - from) * a.scale2 - log_s, cross);
        for (int o = 16; o; o >>= 1) cross += __shfl_xor_sync(~0u, cross, o);
        if (lane == 0) {
          float loss = a.loss_kd * __fmaf_rn(-kLn2, cross, en.entropy);
          if (en.id[a.k] >= 0 && a.loss_label != 0.0f) loss -= a.loss_label * kLn2 * ((en.z[a.k] - from) * kLog2e - log_s1);
          a.loss[row] = some ? loss : 0.0f;
          a.lse[row] = some ? __fmaf_rn(from, a.inv_tau, log_s * kLn2) : -kInf;
          if (a.labels) a.lse[(int64_t)a.rows + row] = some ? __fmaf_rn(log_s1, kLn2, from) : -kInf;
        }
      }
      if (row + step < a.rows) teacher_entries<T>(a, row + step, sh.e[turn ^ 1], sh.slot, lane);
      continue;
    }
    if (!kGrad) continue;
    const float g = a.grad_loss[row];
    const bool label = en.id[a.k] >= 0;
    float c0 = g * a.grad_kd * en.p_sum, c1 = label ? g * a.loss_label : 0.0f, l = 0.0f, l1 = 0.0f;
    bool live = g != 0.0f;
    if (kLoss) {
      live = live && (sum.m != -kInf || sum.s != 0.0f);
      c0 /= sum.s, c1 /= TWO ? sum.s1 : sum.s;
    } else {
      l = a.lse[row];
      if (a.labels) l1 = a.lse[(int64_t)a.rows + row];
      live = live && l != -kInf;
    }
    if (!TWO) c0 += c1;  // one temperature for both
    // Both temperatures' parts, without the entries': c 2^((z times + plus) scale),
    // from the row's own maximum and sums or from the given logarithms.
    const float times = kLoss ? 1.0f : a.inv_tau, plus = kLoss ? -from : -l, plus1 = kLoss ? -from : -l1;
    const float scale = kLoss ? a.scale2 : kLog2e;
    const uint64_t times2 = pack2(times, times), plus2 = pack2(plus, plus), plus12 = pack2(plus1, plus1);
    const uint64_t scale2 = pack2(scale, scale), scale12 = pack2(kLog2e, kLog2e), c02 = pack2(c0, c0), c12 = pack2(c1, c1);
    auto whole2 = [&](uint64_t y) {
      const uint64_t t = kLoss ? add2(y, plus2) : fma2(y, times2, plus2);
      const uint64_t q = mul2(c02, exp2_pair(mul2(t, scale2)));
      return TWO ? fma2(c12, exp2_pair(mul2(kLoss ? t : add2(y, plus12), scale12)), q) : q;
    };
    auto whole = [&](float y) { return unpack2(whole2(pack2(y, y))).x; };
    T *d = static_cast<T *>(a.dlogits) + (int64_t)row * a.dpitch;
    auto put = [&](uint32_t at, uint32_t i, uint4 v) {
      const uint32_t k = at + i * kWorkers + tid;
      if (k >= v1) return;
      if (alike) {
        __stcs(reinterpret_cast<uint4 *>(d + head) + k, v);
      } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        for (int j = 0; j < kPer; ++j) {
          if constexpr (sizeof(T) == 4) d[head + k * kPer + j] = __uint_as_float(w[j]);
          else reinterpret_cast<uint16_t *>(d)[head + k * kPer + j] = (uint16_t)(w[j / 2] >> (j % 2 * 16));
        }
      }
    };
    if (!live) {
      for (uint32_t at = v0; at < v1; at += kWorkers * kVectors)
        for (int i = 0; i < kVectors; ++i) put(at, i, make_uint4(0, 0, 0, 0));
      if (has_odd) d[odd_at] = from_float<T>(0.0f);
    } else {
      if (kLoss && !keeps) load(v0);
      if (kLoss) forget(x);
      for (uint32_t at = v0;;) {
#pragma unroll
        for (int i = 0; i < kVectors; ++i) put(at, i, map<T>(x[i], whole2));
        at += kWorkers * kVectors;
        if (at >= v1) break;
        load(at);
      }
      if (has_odd) d[odd_at] = from_float<T>(whole(x_odd));
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kWorkers) : "memory");  // the row is written but for its entries
    if (!live) continue;
    for (uint32_t i = tid; i <= a.k; i += kWorkers) {
      const int32_t id = en.id[i];
      if (id < 0) continue;
      // whoever wrote the place writes it again
      const uint32_t v = ((uint32_t)id - head) / kPer;
      const bool mine = (uint32_t)id < head || v >= body ? rank == 0 : v >= v0 && v < v1;
      if (!mine) continue;
      float take = i == a.k ? a.loss_label : a.grad_kd * en.p[i];
      bool first_one = true;
      if (en.same) {
        take = 0.0f;
        for (uint32_t j = 0; j <= a.k; ++j)
          if (en.id[j] == id) {
            first_one = first_one && j >= i;
            take += j == a.k ? a.loss_label : a.grad_kd * en.p[j];
          }
      }
      if (first_one) d[id] = from_float<T>(__fmaf_rn(-g, take, whole(en.z[i])));
    }
  }
  if (together) cluster_arrive(), cluster_wait();  // nobody writes to a CTA that has left
}

}  // namespace

int distill_per_sm(const DistillArgs &a) { return residents((a.loss ? 1 : 0) | (a.dlogits ? 2 : 0)); }

int launch_distill(const DistillArgs &a, unsigned cap, unsigned sms, void *stream) {
  return with_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    const uint32_t size = sizeof(T), body = a.vocab / (16 / size);
    // a row over more CTAs while they would not fill the GPU, or while its parts do
    // not fit the registers, but not into parts of less than two vectors a thread
    uint32_t split = 1;
    while (split < (uint32_t)kMaxSplit && body / (2 * split) >= 2 * kWorkers &&
           ((uint64_t)a.rows * split <= sms || (a.loss && a.dlogits && body > split * kWorkers * kKeep)))
      split *= 2;
    const uint64_t most = cap >= split ? cap / split : 1;
    const unsigned grid = (unsigned)(a.rows < most ? a.rows : most) * split;
    const bool alike = a.dlogits && ((uintptr_t)a.dlogits - (uintptr_t)a.logits) % 16 == 0 && (a.dpitch - a.pitch) * size % 16 == 0;
    const bool two = a.labels && a.inv_tau != 1.0f;
    auto go = [&](auto kernel, bool cluster) {
      int e = (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared));
      if (e) return e;
      cudaLaunchAttribute attr = {};
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim = {split, 1, 1};
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(grid);
      cfg.blockDim = dim3(kThreads);
      cfg.dynamicSmemBytes = sizeof(Shared);
      cfg.stream = (cudaStream_t)stream;
      cfg.attrs = &attr;
      cfg.numAttrs = cluster && split > 1 ? 1 : 0;
      return (int)cudaLaunchKernelEx(&cfg, kernel, a, split, alike);
    };
    if (!a.dlogits) return two ? go(distill_kernel<T, 1, true>, true) : go(distill_kernel<T, 1, false>, true);
    if (!a.loss) return two ? go(distill_kernel<T, 2, true>, false) : go(distill_kernel<T, 2, false>, false);
    return two ? go(distill_kernel<T, 3, true>, true) : go(distill_kernel<T, 3, false>, true);
  });
}

}  // namespace apc
