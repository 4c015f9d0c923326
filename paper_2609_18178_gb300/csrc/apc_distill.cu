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
// CTAs exchange maxima and sums.  Its logits come once, by bulk copies into a
// ring of shared-memory chunks that runs ahead of the arithmetic into the next
// row, and stay there between the normaliser and the gradient; a part that the
// ring does not hold is loaded a second time, mostly from DRAM.  One warp copies, a few work on the
// teacher's entries some rows ahead, the others on the logits.
//
// Every wait on a barrier is bounded; one that gives up sets the device status
// word, and the CTA goes through its rows without waiting or copying further.
#include <cuda_runtime.h>

#include <type_traits>

#include "apc_distill_plan.h"
#include "apc_ops.cuh"
#include "apc_tcgen05.cuh"

namespace apc {

namespace {

constexpr int kThreads = kWorkers + 32 * kTeachers + 32;
constexpr int kMinPart = 16 * kWorkers;  // vectors of a row's part: 64 KB
constexpr int kMaxSplit = 8;
constexpr float kInf = __builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The largest logit m and the sums of exp((z - m)/tau) and exp(z - m).
struct Sum {
  float m, s, s1;
};

// A row whose logits are all masked, with infinities or a type's lowest value, has
// none above this.  Their sum's logarithm would be -3.4e38 + log(vocab): fp32 cannot
// hold it, and a gradient from it would take every place's q for 1.
constexpr float kMasked = -1e30f;

// What z's difference is taken to: m, or 0 where every logit is masked (the sums
// are 0 then).
__device__ __forceinline__ float reference(float m) { return m > kMasked ? m : 0.0f; }

// A sum about `from` as one about `to`, the larger.
__device__ __forceinline__ float moved(float s, float from, float to, float scale) {
  return s * exp2_approx((from - reference(to)) * scale);
}

template <int K>
__device__ __forceinline__ void join(Sum &a, const Sum &b, float scale) {
  const float t = fmaxf(a.m, b.m);
  a.s = moved(a.s, a.m, t, scale) + moved(b.s, b.m, t, scale);
  if (K) a.s1 = moved(a.s1, a.m, t, kLog2e) + moved(b.s1, b.m, t, kLog2e);
  a.m = t;
}

// Over the lanes of a warp (or the first `lanes` of them), the same in each.
template <int K>
__device__ __forceinline__ Sum joined(Sum a, float scale, int lanes = 32) {
  float t = a.m;
  for (int o = lanes / 2; o; o >>= 1) t = fmaxf(t, __shfl_xor_sync(~0u, t, o));
  a.s = moved(a.s, a.m, t, scale);
  if (K) a.s1 = moved(a.s1, a.m, t, kLog2e);
  for (int o = lanes / 2; o; o >>= 1) {
    a.s += __shfl_xor_sync(~0u, a.s, o);
    if (K) a.s1 += __shfl_xor_sync(~0u, a.s1, o);
  }
  a.m = t;
  return a;
}

// What a teacher's warp leaves of a row's entries; the label is entry k.
struct Entries {
  int32_t *id;           // -1: does not count
  float *p;              // the probability; the label's is 1
  float *z;              // the student's logit there
  float p_sum, entropy;  // sum of p and of p log p
  int32_t same;          // some place occurs twice
};

struct Shared {
  Entries e[kTeachers + 1];
  Sum part[kTeachers + 1][kWarps];
  Sum peer[kTeachers + 1][kMaxSplit];
  uint64_t full[kMaxChunks], empty[kMaxChunks], peer_full[kTeachers + 1];
  uint64_t read[kTeachers + 1];  // a row's loss no longer needs its entries
  int32_t dead;
  int32_t pad_;
};
static_assert(sizeof(Shared) <= kSharedBytes, "more than the layout keeps for it");

// A place in a ring of n and the parity of its use; no divisions: they and the other
// index arithmetic between two rows took a quarter of a row's time.
struct RingTurn {
  uint32_t at = 0, phase = 0;
  __device__ __forceinline__ void next(uint32_t n) {
    if (++at == n) at = 0, phase ^= 1;
  }
};

// wait_for, at once if another wait of this CTA has given up.
__device__ __noinline__ void wait_alive(uint32_t bar, uint32_t parity, volatile int32_t *dead, unsigned *status) {
  uint64_t t0 = 0;
  for (uint32_t it = 1; !*dead; ++it) {
    if (mbar_try_wait(bar, parity)) return;
    if (it == 1024) t0 = global_ns();
    if (it >= kWaitIterations && (it & 1023u) == 0 && global_ns() - t0 > kWaitNanoseconds) {
      *dead = 1;
      atomicOr(status, (unsigned)APC_ETIMEOUT);
    }
  }
}

__device__ __forceinline__ void wait(uint64_t *bar, uint32_t parity, Shared &sh, unsigned *status) {
  const uint32_t a = smem_addr(bar);
  if (!mbar_try_wait(a, parity) && !mbar_try_wait(a, parity)) wait_alive(a, parity, &sh.dead, status);
}

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
__device__ __noinline__ void teacher_entries(const DistillArgs &a, uint32_t row, Entries &e, int32_t *slot, uint32_t slots_log2,
                                             uint32_t lane) {
  const T *z = static_cast<const T *>(a.logits) + (int64_t)row * a.pitch;
  const int64_t at_id = (int64_t)row * a.ids_pitch, at_u = (int64_t)row * a.teacher_pitch;
  int32_t *ids = e.id;
  float *ps = e.p, *zs = e.z;
  float top = -kInf;
  // entries a lane has in flight: their ids, then the student's logits there (8
  // cost the rows' own arithmetic more than they saved: 268 us for 8192 x 32768 when 2 took 246)
  constexpr int kBatch = 2;
  for (uint32_t i0 = lane; i0 < a.k; i0 += 32 * kBatch) {
    int32_t id[kBatch];
    float u[kBatch], x[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const uint32_t i = i0 + 32 * b;
      const int64_t v = i < a.k ? index_at(a.ids, a.ids64, at_id + i) : -1;
      u[b] = i < a.k ? number_at(a.teacher, a.teacher_dtype, at_u + i) : -kInf;
      id[b] = v < 0 || v >= (int64_t)a.vocab || u[b] == -kInf ? -1 : (int32_t)v;
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) x[b] = id[b] >= 0 ? to_float(z[id[b]]) : 0.0f;
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const uint32_t i = i0 + 32 * b;
      if (id[b] < 0) u[b] = -kInf;
      if (i < a.k) ids[i] = id[b], ps[i] = u[b], zs[i] = x[b];
      top = fmaxf(top, u[b]);
    }
  }
  if (lane == 0) {
    int64_t y = a.labels ? index_at(a.labels, a.labels64, row) : -1;
    if (y >= (int64_t)a.vocab || y < 0) y = -1;
    ids[a.k] = (int32_t)y;
    ps[a.k] = 1.0f;
    zs[a.k] = y >= 0 ? to_float(z[y]) : 0.0f;
  }
  if (a.dlogits) {  // an empty table
    int4 *t = reinterpret_cast<int4 *>(slot);
    for (uint32_t i = lane; i < 1u << slots_log2 >> 2; i += 32) t[i] = make_int4(-1, -1, -1, -1);
  }
  for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
  float norm = 0.0f;
  if (a.teacher_lse) {
    top = 0.0f;
    norm = a.teacher_lse[row];
  } else {
    if (top == -kInf) top = 0.0f;
    float s = 0.0f;
    for (uint32_t i = lane; i < a.k; i += 32) s += exp2_approx((ps[i] - top) * a.scale2);
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    norm = logf(s);
  }
  float p_sum = 0.0f, entropy = 0.0f;
  bool same = false;
  __syncwarp();
  for (uint32_t i = lane; i <= a.k; i += 32) {
    const int32_t id = ids[i];
    if (i < a.k) {
      const float lp = id >= 0 ? __fmaf_rn(ps[i] - top, a.inv_tau, -norm) : -kInf, p = exp2_approx(lp * kLog2e);
      ps[i] = p;
      p_sum += p;
      if (p != 0.0f) entropy = __fmaf_rn(p, lp, entropy);
    }
    if (a.dlogits && id >= 0)
      for (uint32_t h = (uint32_t)id * 2654435761u >> (32 - slots_log2);; h = (h + 1) & ((1u << slots_log2) - 1)) {  // at most half full
        const int32_t was = atomicCAS(&slot[h], -1, id);
        same |= was == id;
        if (was == -1 || was == id) break;
      }
  }
  for (int o = 16; o; o >>= 1) {
    p_sum += __shfl_xor_sync(~0u, p_sum, o);
    entropy += __shfl_xor_sync(~0u, entropy, o);
  }
  same = __any_sync(~0u, same);
  if (lane == 0) e.p_sum = p_sum, e.entropy = entropy, e.same = same;
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

// A vector of elements that leave every maximum and sum alone.
template <typename T>
__device__ __forceinline__ uint4 nothing() {
  const uint32_t w = sizeof(T) == 4 ? 0xff800000u : __is_same(T, __half) ? 0xfc00fc00u : 0xff80ff80u;
  return {w, w, w, w};
}

// K: what the labels need beside the sums at tau.  0: nothing (no labels, or tau =
// 1); 1: exponentials of their own; 2, 4: tau is that number, and the exponential at
// 1 the power of the one at tau (17 instructions a pair of elements and both passes, for 23).
// The power's relative error is 2 or 4 times the function's 2^-22: below a rounding to
// 16 bits, and for fp32 within what an exponent of 8 rounded to fp32 costs anyway.

// A row's or a part's sums on the way: the largest logit and, in two fp32 lanes, the
// sums about it.
template <typename T, int K>
struct Running {
  float m;
  uint64_t s, s1;

  // One element to begin with, or none.
  __device__ __forceinline__ Running(float x, bool has, float scale2) : m(x), s(0), s1(0) {
    if (!has) return;
    s = pack2(exp2_approx((x - reference(x)) * scale2), 0.0f);
    if (K) s1 = pack2(exp2_approx((x - reference(x)) * kLog2e), 0.0f);
  }

  template <int N>
  __device__ __forceinline__ void add(const uint4 (&x)[N], float scale2) {
    const uint64_t scale = pack2(scale2, scale2), scale1 = pack2(kLog2e, kLog2e);
    const float top = largest<T>(x);
    if (top > m) {  // the sums move to the new maximum
      const float f = moved(1.0f, m, top, scale2);
      s = mul2(s, pack2(f, f));
      if (K) {
        const float f1 = moved(1.0f, m, top, kLog2e);
        s1 = mul2(s1, pack2(f1, f1));
      }
      m = top;
    }
    const uint64_t minus = pack2(-reference(m), -reference(m));
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
      for (int j = 0; j < 8 / (int)sizeof(T); ++j) {
        const uint64_t y = add2(pair<T>(x[i], j), minus), e = exp2_pair(mul2(y, scale));
        s = add2(s, e);
        if (K == 1) s1 = add2(s1, exp2_pair(mul2(y, scale1)));
        if (K == 2) s1 = fma2(e, e, s1);
        if (K == 4) s1 = fma2(mul2(e, e), mul2(e, e), s1);
      }
    }
  }

  __device__ __forceinline__ Sum sum() const {
    const float2 u = unpack2(s), u1 = unpack2(s1);
    return {m, u.x + u.y, u1.x + u1.y};
  }
};

__device__ __forceinline__ bool has_logits(const Sum &s) { return s.s != 0.0f; }  // a NaN has

// One warp: the row's loss and statistics, from its sums and entries.
template <int K>
__device__ __forceinline__ void store_loss(const DistillArgs &a, uint32_t row, const Sum &sum, const Entries &en, uint32_t lane) {
  const float from = reference(sum.m), log_s = log2f(sum.s) * kLn2, log_s1 = K ? log2f(sum.s1) * kLn2 : log_s;
  const bool some = has_logits(sum);
  float cross = 0.0f;
  for (uint32_t i = lane; i < a.k; i += 32)
    if (en.p[i] != 0.0f) cross = __fmaf_rn(a.loss_kd * en.p[i], __fmaf_rn(en.z[i] - from, a.inv_tau, -log_s), cross);
  for (int o = 16; o; o >>= 1) cross += __shfl_xor_sync(~0u, cross, o);
  if (lane == 0) {
    float loss = __fmaf_rn(a.loss_kd, en.entropy, -cross);
    if (en.id[a.k] >= 0 && a.loss_label != 0.0f) loss -= a.loss_label * (en.z[a.k] - from - log_s1);
    a.loss[row] = some ? loss : 0.0f;
    a.lse[row] = some ? __fmaf_rn(from, a.inv_tau, log_s) : -kInf;
    if (a.labels) a.lse[(int64_t)a.rows + row] = some ? from + log_s1 : -kInf;
  }
}

// A row's gradient without its entries' part: both temperatures' c 2^((z times +
// plus) scale), from the row's own maximum and sums or from the given logarithms.
template <bool LOSS, int K>
struct Whole {
  bool live;  // else zeros
  float g;
  uint64_t times, plus, plus1, scale, scale1, c0, c1;

  __device__ __forceinline__ Whole(const DistillArgs &a, uint32_t row, const Sum &sum, const Entries &en) {
    g = a.grad_loss[row];
    float k0 = g * a.grad_kd * en.p_sum, k1 = en.id[a.k] >= 0 ? g * a.loss_label : 0.0f, l = 0.0f, l1 = 0.0f;
    const float from = reference(sum.m);
    live = g != 0.0f;
    if (LOSS) {
      live = live && has_logits(sum);
      k0 /= sum.s, k1 /= K ? sum.s1 : sum.s;
    } else {
      l = a.lse[row];
      if (a.labels) l1 = a.lse[(int64_t)a.rows + row];
      live = live && !(l <= kMasked);
      if (K > 1 && k1 != 0.0f) k1 *= expf(__fmaf_rn((float)K, l, -l1));  // exp(z - l1) = exp(z/tau - l)^tau exp(tau l - l1)
    }
    if (K == 0) k0 += k1;  // one temperature for both
    const float t = LOSS ? 1.0f : a.inv_tau, p = LOSS ? -from : -l, p1 = LOSS ? -from : -l1, f = LOSS ? a.scale2 : kLog2e;
    times = pack2(t, t), plus = pack2(p, p), plus1 = pack2(p1, p1), scale = pack2(f, f), scale1 = pack2(kLog2e, kLog2e);
    c0 = pack2(k0, k0), c1 = pack2(k1, k1);
  }

  __device__ __forceinline__ uint64_t operator()(uint64_t y) const {
    const uint64_t t = LOSS ? add2(y, plus) : fma2(y, times, plus), e = exp2_pair(mul2(t, scale));
    if (K == 0) return mul2(c0, e);
    if (K == 1) return fma2(c1, exp2_pair(mul2(LOSS ? t : add2(y, plus1), scale1)), mul2(c0, e));
    if (K == 2) return mul2(e, fma2(c1, e, c0));
    return mul2(e, fma2(c1, mul2(e, mul2(e, e)), c0));
  }

  __device__ __forceinline__ float one(float y) const { return unpack2((*this)(pack2(y, y))).x; }
};

// The gradient at entry i's place, where this is the first entry there; false otherwise.
template <typename W>
__device__ __forceinline__ bool entry_gradient(const DistillArgs &a, const Entries &en, const W &whole, uint32_t i, float *out) {
  const int32_t id = en.id[i];
  float take = i == a.k ? a.loss_label : a.grad_kd * en.p[i];
  if (en.same) {  // entries of one place add up, in their order
    bool first = true;
    take = 0.0f;
    for (uint32_t j = 0; j <= a.k; ++j)
      if (en.id[j] == id) {
        first = first && j >= i;
        take += j == a.k ? a.loss_label : a.grad_kd * en.p[j];
      }
    if (!first) return false;
  }
  *out = __fmaf_rn(-whole.g, take, whole.one(en.z[i]));
  return true;
}

// Vector v to place k of a row's body: as it is where the gradient's rows are aligned
// as the logits' are, else element by element.
template <typename T>
__device__ __forceinline__ void store_vector(T *body, uint32_t k, const uint4 &v, bool alike) {
  constexpr int kPer = 16 / sizeof(T);
  if (alike) {
    __stcs(reinterpret_cast<uint4 *>(body) + k, v);
  } else {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if constexpr (sizeof(T) == 4) body[(int64_t)k * kPer + j] = __uint_as_float(w[j]);
      else reinterpret_cast<uint16_t *>(body)[(int64_t)k * kPer + j] = (uint16_t)(w[j / 2] >> (j % 2 * 16));
    }
  }
}

// ---------------------------------------------------------------------------
// Short rows, of which there are many: one warp a row, from its entries to its
// gradient.  A row's way takes some 6 us, most of it waiting, so what counts is how
// many are under way: 24 on an SM, where the kernel below has 2.  Up to
// kShortVectors of 16 bytes a lane stay in registers; a longer row's second sweep
// finds it in L2.  Loss and gradient of 8192 rows of bf16: 100 logits 19 us (79 by the
// kernel below), 5000 47 (85); 300 rows of 4000 10.5 (8.7), 4096 rows of 32768
// (loss) 58 (42): hence the limits on both sides.
constexpr int kShortWarps = 8, kShortVectors = 8, kShortCtas = 3;
constexpr uint32_t kShortBytes = 24576, kShortEntries = 256;

template <typename T, int FORM, int K>
__global__ void __launch_bounds__(32 * kShortWarps, kShortCtas)
    short_kernel(const __grid_constant__ DistillArgs a, const uint32_t room, const uint32_t slots_log2, const bool alike) {
  extern __shared__ __align__(16) uint8_t raw[];
  __shared__ Entries all[kShortWarps];
  constexpr int kPer = 16 / sizeof(T);
  constexpr bool kLoss = FORM & 1, kGrad = FORM & 2;
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  Entries &en = all[warp];
  int32_t *table = reinterpret_cast<int32_t *>(raw + warp * (room * 12 + (4u << slots_log2)));
  if (lane == 0) {
    uint8_t *at = reinterpret_cast<uint8_t *>(table) + (4u << slots_log2);
    en.id = reinterpret_cast<int32_t *>(at), en.p = reinterpret_cast<float *>(at + room * 4), en.z = reinterpret_cast<float *>(at + room * 8);
  }
  __syncwarp();
  for (uint64_t row = blockIdx.x * kShortWarps + warp; row < a.rows; row += gridDim.x * kShortWarps) {
    const T *z = static_cast<const T *>(a.logits) + (int64_t)row * a.pitch;
    const uint32_t head = min(a.vocab, (uint32_t)((16 - (uintptr_t)z % 16) % 16 / sizeof(T)));
    const uint32_t body = (a.vocab - head) / kPer, odd = a.vocab - body * kPer;
    const uint4 *zv = reinterpret_cast<const uint4 *>(z + head);
    const uint32_t odd_at = lane < head ? lane : body * kPer + lane;
    const float x_odd = lane < odd ? to_float(z[odd_at]) : -kInf;
    uint4 x[kShortVectors];
    auto load = [&](uint32_t at) {
#pragma unroll
      for (int i = 0; i < kShortVectors; ++i) x[i] = at + i * 32 + lane < body ? zv[at + i * 32 + lane] : nothing<T>();
    };
    load(0);
    __syncwarp();
    teacher_entries<T>(a, (uint32_t)row, en, table, slots_log2, lane);
    __syncwarp();
    Sum sum = {-kInf, 0.0f, 0.0f};
    if (kLoss) {
      Running<T, K> run(x_odd, lane < odd, a.scale2);
      for (uint32_t at = 0;;) {
        run.add(x, a.scale2);
        at += 32 * kShortVectors;
        if (at >= body) break;
        load(at);
      }
      sum = joined<K>(run.sum(), a.scale2);
      store_loss<K>(a, (uint32_t)row, sum, en, lane);
    }
    if (!kGrad) continue;
    const Whole<kLoss, K> whole(a, (uint32_t)row, sum, en);
    T *d = static_cast<T *>(a.dlogits) + (int64_t)row * a.dpitch;
    if (kLoss && body > 32 * kShortVectors) load(0);
    for (uint32_t at = 0;;) {
#pragma unroll
      for (int i = 0; i < kShortVectors; ++i)
        if (at + i * 32 + lane < body)
          store_vector<T>(d + head, at + i * 32 + lane, whole.live ? map<T>(x[i], whole) : make_uint4(0, 0, 0, 0), alike);
      at += 32 * kShortVectors;
      if (at >= body) break;
      load(at);
    }
    if (lane < odd) d[odd_at] = from_float<T>(whole.live ? whole.one(x_odd) : 0.0f);
    __syncwarp();  // the row is written but for its entries
    float v;
    if (whole.live)
      for (uint32_t i = lane; i <= a.k; i += 32)
        if (en.id[i] >= 0 && entry_gradient(a, en, whole, i, &v)) d[en.id[i]] = from_float<T>(v);
  }
}

// ---------------------------------------------------------------------------
// Longer rows.  Bound by issue: 60% of the issue slots with labels (17 instructions
// a pair of elements); the rest goes at the rows' turns.  Measured: loss
// and gradient of 8192 x 32768 with labels 199 us (5.4 TB/s), loss of 4096 x 32768 42 us
// (6.4 TB/s), gradient of 1021 x 100003 84 us (4.9 TB/s), loss and gradient of 1600 x
// 150000 226 us.
// FORM: 1 loss, 2 gradient, 3 both.  alike: the gradient's rows are aligned as the logits' are.
template <typename T, int FORM, int K>
__global__ void __launch_bounds__(kThreads, kCtas)
    distill_kernel(const __grid_constant__ DistillArgs a, const __grid_constant__ Layout layout, const uint32_t split_log2,
                   const bool alike) {
  extern __shared__ __align__(16) uint8_t raw[];
  Shared &sh = *reinterpret_cast<Shared *>(raw);
  uint4 *ring = reinterpret_cast<uint4 *>(raw + kSharedBytes);
  int32_t *tables = reinterpret_cast<int32_t *>(ring + layout.chunks * layout.chunk);
  float *sums = reinterpret_cast<float *>(tables + layout.tables) + (layout.teachers + 1) * layout.room * 3;
  const uint32_t kChunks = layout.chunks;
  constexpr int kPer = 16 / sizeof(T), kVectors = kVectorsOf<FORM>, kChunk = kWorkers * kVectors;
  constexpr bool kLoss = FORM & 1, kGrad = FORM & 2;
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32, split = 1u << split_log2;
  const uint32_t rank = blockIdx.x & (split - 1), first = blockIdx.x >> split_log2, step = gridDim.x >> split_log2;
  const bool together = kLoss && split > 1;  // the CTAs of a row are a cluster
  if (tid == 0) {
    for (uint32_t i = 0; i < kChunks; ++i) mbar_init(&sh.full[i], 1), mbar_init(&sh.empty[i], kWarps);
    for (int i = 0; i <= kTeachers; ++i) mbar_init(&sh.peer_full[i], 1), mbar_init(&sh.read[i], 1);
    sh.dead = 0;
    uint8_t *entries = reinterpret_cast<uint8_t *>(tables + layout.tables);
    for (uint32_t i = 0; i <= layout.teachers; ++i, entries += layout.room * 12) {
      sh.e[i].id = reinterpret_cast<int32_t *>(entries);
      sh.e[i].p = reinterpret_cast<float *>(entries + layout.room * 4);
      sh.e[i].z = reinterpret_cast<float *>(entries + layout.room * 8);
    }
    mbar_init_fence();
    if (together)
      for (uint32_t i = 0; i <= layout.teachers; ++i) mbar_arrive_expect_tx(&sh.peer_full[i], split * 12);
  }
  __syncthreads();
  if (together) cluster_arrive(), cluster_wait();  // the barriers are there before anyone sends

  // Vectors [v0, v1) of a row's 16-byte aligned body are this CTA's; the elements
  // outside the body are the first CTA's.
  struct Part {
    const T *z;
    uint32_t head, body, v0, v1, chunks;
    bool keeps;  // the ring holds the part: loss and gradient share one copy
  };
  auto part_of = [&](uint32_t row) {
    Part p;
    p.z = static_cast<const T *>(a.logits) + (int64_t)row * a.pitch;
    p.head = min(a.vocab, (uint32_t)((16 - (uintptr_t)p.z % 16) % 16 / sizeof(T)));
    p.body = (a.vocab - p.head) / kPer;
    p.v0 = (uint32_t)((uint64_t)p.body * rank >> split_log2), p.v1 = (uint32_t)((uint64_t)p.body * (rank + 1) >> split_log2);
    p.chunks = (p.v1 - p.v0 + kChunk - 1) / kChunk;
    p.keeps = p.chunks <= kChunks;
    return p;
  };

  if (warp == kWarps + kTeachers) {
    // copies
    if (lane == 0) {
      const uint64_t policy = l2_evict_first();
      RingTurn to;
      uint32_t issued = 0;
      for (uint32_t row = first; row < a.rows; row += step) {
        const Part p = part_of(row);
        for (int sweep = 0; sweep < (FORM == 3 && !p.keeps ? 2 : 1); ++sweep)
          for (uint32_t c = 0; c < p.chunks; ++c, ++issued, to.next(kChunks)) {
            const uint32_t from = p.v0 + c * kChunk, bytes = min((uint32_t)kChunk, p.v1 - from) * 16;
            wait(&sh.empty[to.at], to.phase ^ 1, sh, a.status);
            if (*(volatile int32_t *)&sh.dead) goto drain;
            mbar_arrive_expect_tx(&sh.full[to.at], bytes);
            bulk_g2s(ring + to.at * kChunk, reinterpret_cast<const uint4 *>(p.z + p.head) + from, bytes, &sh.full[to.at], policy);
          }
      }
    drain:
      if (*(volatile int32_t *)&sh.dead)
        for (uint32_t u = issued > kChunks ? issued - kChunks : 0; u < issued; ++u) wait_for(&sh.full[u % kChunks], u / kChunks & 1);
    }
  } else if (warp < kWarps + layout.teachers) {
    // Row i is teacher i's (modulo their number).  It meets the workers at a barrier
    // of its own when its entries are there and their sums are, and then goes on to
    // the entries of row i + teachers.  Entries, sums and the cluster's sums have one
    // place more than there are teachers: the entries of row i + teachers take row
    // i - 1's.  At row i's barrier the workers are through with row i - 1, but its own
    // teacher, who does not come to that barrier, may still be at its loss: `read` says when
    // it is done.  Sums are written again a row later, behind a barrier of that teacher's.
    const bool worker = warp < kWarps;
    const uint32_t teachers = layout.teachers, own = worker ? 0 : warp - kWarps;
    int32_t *table = tables + (own << layout.slots_log2);
    RingTurn ring_at;
    uint32_t done = own, turn = 0, round = 0, barrier = 2;
    if (!worker && first + (uint64_t)own * step < a.rows)
      teacher_entries<T>(a, first + own * step, sh.e[own], table, layout.slots_log2, lane);
    for (uint64_t row = first + (uint64_t)own * step; row < a.rows; row += worker ? step : (uint64_t)step * teachers, done += worker ? 1 : teachers) {
      if (!worker) {
        turn = done % (teachers + 1), round = done / (teachers + 1), barrier = 2 + own;
      } else if (done) {
        if (turn++ == teachers) turn = 0, ++round;
        if (++barrier == 2 + teachers) barrier = 2;
      }
      float *own_sums = sums + turn * (3 * kWorkers);  // the loss alone: every worker's
      const Part p = part_of(row);
      const uint32_t odd = a.vocab - p.body * kPer;
      const bool has_odd = worker && rank == 0 && tid < odd;
      const uint32_t odd_at = tid < p.head ? tid : p.body * kPer + tid;
      const float x_odd = has_odd ? to_float(p.z[odd_at]) : -kInf;
      Sum sum = {-kInf, 0.0f, 0.0f};
      if (kLoss) {
        if (worker) {
          Running<T, K> run(x_odd, has_odd, a.scale2);
          RingTurn at = ring_at;
          for (uint32_t c = 0; c < p.chunks; ++c) {
            const uint32_t s = at.at, n = p.v1 - p.v0 - c * kChunk;
            wait(&sh.full[s], at.phase, sh, a.status);
            at.next(kChunks);
            uint4 x[kVectors];
            const uint4 *from = ring + s * kChunk + tid;
            if (n >= kChunk) {
#pragma unroll
              for (int i = 0; i < kVectors; ++i) x[i] = from[i * kWorkers];
            } else {
#pragma unroll
              for (int i = 0; i < kVectors; ++i) x[i] = i * kWorkers + tid < n ? from[i * kWorkers] : nothing<T>();
            }
            run.add(x, a.scale2);
            if (FORM == 1 || !p.keeps) {
              __syncwarp();
              if (lane == 0) mbar_arrive(&sh.empty[s]);
            }
          }
          if (FORM == 1 || !p.keeps) ring_at = at;
          sum = run.sum();
          if (FORM == 1 && !together) {  // the teacher joins them
            own_sums[tid] = sum.m, own_sums[kWorkers + tid] = sum.s;
            if (K) own_sums[2 * kWorkers + tid] = sum.s1;
          } else {
            sum = joined<K>(sum, a.scale2);
            if (lane == 0) sh.part[turn][warp] = sum;
          }
        }
        asm volatile("bar.sync %0, %1;" ::"r"(barrier), "n"(kWorkers + 32) : "memory");
        if (FORM == 1 && worker && !together) continue;  // the rest is the teacher's
        if (FORM == 1 && !together) {
          sum = {-kInf, 0.0f, 0.0f};
#pragma unroll
          for (int w = 0; w < kWarps; ++w) sum.m = fmaxf(sum.m, own_sums[32 * w + lane]);
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            const float m = own_sums[32 * w + lane];
            sum.s += moved(own_sums[kWorkers + 32 * w + lane], m, sum.m, a.scale2);
            if (K) sum.s1 += moved(own_sums[2 * kWorkers + 32 * w + lane], m, sum.m, kLog2e);
          }
        } else {
          sum = lane < kWarps ? sh.part[turn][lane] : Sum{-kInf, 0.0f, 0.0f};
        }
        sum = joined<K>(sum, a.scale2);
        if (together) {
          if (tid < split) {
            const uint32_t at = map_rank(smem_addr(&sh.peer[turn][rank]), tid), bar = map_rank(smem_addr(&sh.peer_full[turn]), tid);
            store_async(at, sum.m, bar), store_async(at + 4, sum.s, bar), store_async(at + 8, sum.s1, bar);
          }
          wait(&sh.peer_full[turn], round & 1, sh, a.status);
          asm volatile("fence.acq_rel.cluster;" ::: "memory");
          if (tid == 0) mbar_arrive_expect_tx(&sh.peer_full[turn], split * 12);  // for the next round
          sum = sh.peer[turn][0];
          for (uint32_t k = 1; k < split; ++k) join<K>(sum, sh.peer[turn][k], a.scale2);
        }
      } else {
        asm volatile("bar.sync %0, %1;" ::"r"(barrier), "n"(kWorkers + 32) : "memory");
      }
      const Entries &en = sh.e[turn];
      if (!worker) {
        // the row's loss, then the next row's entries
        if (kLoss) {
          if (rank == 0) store_loss<K>(a, (uint32_t)row, sum, en, lane);
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.read[turn]);
        }
        if (row + (uint64_t)step * teachers < a.rows) {
          const uint32_t next = (done + teachers) % (teachers + 1), use = (done + teachers) / (teachers + 1);
          if (kLoss) wait(&sh.read[next], use & 1 ^ 1, sh, a.status);  // the first use passes
          teacher_entries<T>(a, (uint32_t)(row + (uint64_t)step * teachers), sh.e[next], table, layout.slots_log2, lane);
        }
        continue;
      }
      if (!kGrad) continue;
      const Whole<kLoss, K> whole(a, (uint32_t)row, sum, en);
      T *d = static_cast<T *>(a.dlogits) + (int64_t)row * a.dpitch;
      for (uint32_t c = 0; c < p.chunks; ++c, ring_at.next(kChunks)) {
        const uint32_t s = ring_at.at, at = p.v0 + c * kChunk;
        wait(&sh.full[s], ring_at.phase, sh, a.status);
        const uint4 *x = ring + s * kChunk + tid;
        if (alike && whole.live && p.v1 - at >= kChunk) {
          uint4 *to = reinterpret_cast<uint4 *>(d + p.head) + at + tid;
#pragma unroll
          for (int i = 0; i < kVectors; ++i) __stcs(to + i * kWorkers, map<T>(x[i * kWorkers], whole));
        } else {
          for (int i = 0; i < kVectors; ++i) {
            const uint32_t k = at + i * kWorkers + tid;
            if (k >= p.v1) break;
            store_vector<T>(d + p.head, k, whole.live ? map<T>(x[i * kWorkers], whole) : make_uint4(0, 0, 0, 0), alike);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.empty[s]);
      }
      if (has_odd) d[odd_at] = from_float<T>(whole.live ? whole.one(x_odd) : 0.0f);
      asm volatile("bar.sync 1, %0;" ::"n"(kWorkers) : "memory");  // the row is written but for its entries
      if (!whole.live) continue;
      for (uint32_t i = tid; i <= a.k; i += kWorkers) {
        const int32_t id = en.id[i];
        if (id < 0) continue;
        // whoever wrote the place writes it again
        const uint32_t v = ((uint32_t)id - p.head) / kPer;
        if (!((uint32_t)id < p.head || v >= p.body ? rank == 0 : v >= p.v0 && v < p.v1)) continue;
        float y;
        if (entry_gradient(a, en, whole, i, &y)) d[id] = from_float<T>(y);
      }
    }
  }
  __syncwarp();
  if (together) cluster_arrive(), cluster_wait();  // nobody writes to a CTA that has left
}

}  // namespace

namespace {

// A warp for each row where rows are short and enough of them to fill the GPU.
bool rows_are_short(const DistillArgs &a, unsigned sms) {
  return a.vocab * (a.dtype == APC_F32 ? 4u : 2u) <= kShortBytes && a.k <= kShortEntries && a.rows >= 4 * sms;
}

template <int V>
using Int = std::integral_constant<int, V>;

// f(FORM, K) of a call.
template <typename F>
int with_form(const DistillArgs &a, int k, F f) {
  auto with_power = [&](auto form) {
    switch (k) {
      case 0: return f(form, Int<0>{});
      case 2: return f(form, Int<2>{});
      case 4: return f(form, Int<4>{});
    }
    return f(form, Int<1>{});
  };
  return !a.dlogits ? with_power(Int<1>{}) : !a.loss ? with_power(Int<2>{}) : with_power(Int<3>{});
}

}  // namespace

int distill_per_sm(const DistillArgs &a, unsigned sms) { return rows_are_short(a, sms) ? kShortCtas : kCtas; }

int launch_distill(const DistillArgs &args, unsigned cap, unsigned sms, void *stream) {
  DistillArgs a = args;
  const int e = commit_status_word(&a.status);
  if (e) return e;
  return with_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    const uint32_t size = sizeof(T), body = a.vocab / (16 / size);
    const bool alike = a.dlogits && ((uintptr_t)a.dlogits - (uintptr_t)a.logits) % 16 == 0 && (a.dpitch - a.pitch) * size % 16 == 0;
    const int k = !a.labels || a.inv_tau == 1.0f ? 0 : a.inv_tau == 0.5f ? 2 : a.inv_tau == 0.25f ? 4 : 1;
    if (rows_are_short(a, sms)) {
      const uint32_t room = room_of(a.k), slots_log2 = slots_log2_of(a.k);
      const uint32_t bytes = kShortWarps * (room * 12 + (4u << slots_log2)), want = (a.rows + kShortWarps - 1) / kShortWarps;
      auto go = [&](auto kernel) {
        int e = (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e) return e;
        kernel<<<want < cap ? want : cap, 32 * kShortWarps, bytes, (cudaStream_t)stream>>>(a, room, slots_log2, alike);
        return (int)cudaGetLastError();
      };
      return with_form(a, k, [&](auto form, auto power) { return go(short_kernel<T, form.value, power.value>); });
    }
    const Layout l = distill_layout(a.k, a.loss, a.dlogits);
    // a row over more CTAs while they would not fill the GPU, but not into parts of
    // less than 64 KB
    uint32_t split_log2 = 0;
    while ((1u << split_log2) < (uint32_t)kMaxSplit && body >> (split_log2 + 1) >= kMinPart && (uint64_t)a.rows << split_log2 <= sms)
      ++split_log2;
    const uint32_t split = 1u << split_log2;
    const uint64_t most = cap >= split ? cap / split : 1;
    const unsigned grid = (unsigned)(a.rows < most ? a.rows : most) * split;
    auto go = [&](auto kernel, bool cluster) {
      int e = (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)l.bytes());
      if (e) return e;
      cudaLaunchAttribute attr = {};
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim = {split, 1, 1};
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(grid);
      cfg.blockDim = dim3(kThreads);
      cfg.dynamicSmemBytes = l.bytes();
      cfg.stream = (cudaStream_t)stream;
      cfg.attrs = &attr;
      cfg.numAttrs = cluster && split > 1 ? 1 : 0;
      return (int)cudaLaunchKernelEx(&cfg, kernel, a, l, split_log2, alike);
    };
    return with_form(a, k, [&](auto form, auto power) { return go(distill_kernel<T, form.value, power.value>, form.value != 2); });
  });
}

}  // namespace apc
