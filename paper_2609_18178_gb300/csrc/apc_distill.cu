// Distillation from a teacher's largest logits: loss and gradient
// (apc_distill_loss, apc_distill_grad, apc_distill_loss_grad).
//
// One CTA takes one row at a time.  The row's normalisers come from one sweep
// with a running maximum and sum per thread; the teacher's probabilities are
// few and the first warp's; the gradient is a second sweep, after which the
// entries' places are written once more.
#include <cuda_runtime.h>

#include "apc_ops.cuh"

namespace apc {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr float kInf = __builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The largest logit m and the sums of exp((z - m)/tau) and exp(z - m).  The
// difference comes before the scaling: logits at their type's lowest value
// would overflow the other way round.
struct Sum {
  float m, s, s1;
  __device__ __forceinline__ void add(const Sum &o, float scale2) {
    const float t = fmaxf(m, o.m), b = t == -kInf ? 0.0f : t, x = m - b, y = o.m - b;
    s = s * exp2_approx(x * scale2) + o.s * exp2_approx(y * scale2);
    s1 = s1 * exp2_approx(x * kLog2e) + o.s1 * exp2_approx(y * kLog2e);
    m = t;
  }
};

__device__ __forceinline__ Sum warp_sum(Sum a, float scale2) {
  for (int o = 16; o; o >>= 1)
    a.add({__shfl_xor_sync(~0u, a.m, o), __shfl_xor_sync(~0u, a.s, o), __shfl_xor_sync(~0u, a.s1, o)}, scale2);
  return a;
}

__device__ __forceinline__ float log_sum(float m, float s, float inv_tau) {
  return __fmaf_rn(m, inv_tau, log2f(s) * kLn2);
}

struct Shared {
  int32_t id[APC_DISTILL_MAX_K + 1];   // the entries' places, then the label's; -1: none
  float p[APC_DISTILL_MAX_K + 1];      // what each takes from the gradient, over grad_loss
  float z[APC_DISTILL_MAX_K + 1];
  Sum part[kWarps];
  float kd, p_sum;
};

__device__ __forceinline__ int64_t index_at(const void *p, bool wide, int64_t i) {
  return wide ? static_cast<const int64_t *>(p)[i] : static_cast<const int32_t *>(p)[i];
}

__device__ __forceinline__ float number_at(const void *p, uint32_t dtype, int64_t i) {
  return dtype == APC_F32 ? static_cast<const float *>(p)[i]
         : dtype == APC_BF16 ? to_float(static_cast<const __nv_bfloat16 *>(p)[i])
                             : to_float(static_cast<const __half *>(p)[i]);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) distill_kernel(const __grid_constant__ DistillArgs a) {
  __shared__ Shared sh;
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    __syncthreads();
    const T *z = static_cast<const T *>(a.logits) + row * a.pitch;
    // the normalisers
    float l, l1 = 0.0f;  // logarithms of the sums at tau and at 1
    if (a.loss) {
      Sum s = {-kInf, 0.0f, 0.0f};
      for (uint32_t i = tid; i < a.vocab; i += kThreads) s.add({to_float(z[i]), 1.0f, 1.0f}, a.scale2);
      s = warp_sum(s, a.scale2);
      if (lane == 0) sh.part[warp] = s;
      __syncthreads();
      s = warp_sum(lane < kWarps ? sh.part[lane] : Sum{-kInf, 0.0f, 0.0f}, a.scale2);
      l = log_sum(s.m, s.s, a.inv_tau);
      l1 = log_sum(s.m, s.s1, 1.0f);
      if (tid == 0) {
        a.lse[row] = l;
        if (a.labels) a.lse[a.rows + row] = l1;
      }
    } else {
      l = a.lse[row];
      if (a.labels) l1 = a.lse[a.rows + row];
    }
    const bool some = l != -kInf;
    // the teacher's probabilities
    if (warp == 0) {
      Sum t = {-kInf, 0.0f, 0.0f};
      for (uint32_t i = lane; i < a.k; i += 32) {
        const int64_t id = index_at(a.ids, a.ids64, row * a.ids_pitch + i);
        const float u = number_at(a.teacher, a.teacher_dtype, row * a.teacher_pitch + i);
        const bool counts = id >= 0 && id < a.vocab && u != -kInf;
        sh.id[i] = counts ? (int32_t)id : -1;
        sh.p[i] = u;
        if (counts) t.add({u, 1.0f, 0.0f}, a.scale2);
      }
      t = warp_sum(t, a.scale2);
      const float norm = a.teacher_lse ? a.teacher_lse[row] : log_sum(t.m, t.s, a.inv_tau);
      float kl = 0.0f, p_sum = 0.0f;
      for (uint32_t i = lane; i < a.k; i += 32)
        if (sh.id[i] >= 0) {
          const float lp = __fmaf_rn(sh.p[i], a.inv_tau, -norm), p = exp2f(lp * kLog2e), x = to_float(z[sh.id[i]]);
          sh.p[i] = a.grad_kd * p;
          sh.z[i] = x;
          p_sum += p;
          if (p != 0.0f) kl += p * (lp - __fmaf_rn(x, a.inv_tau, -l));
        }
      for (int o = 16; o; o >>= 1) {
        kl += __shfl_xor_sync(~0u, kl, o);
        p_sum += __shfl_xor_sync(~0u, p_sum, o);
      }
      if (lane == 0) {
        float loss = a.loss_kd * kl;
        int32_t y = -1;
        if (a.labels) {
          const int64_t id = index_at(a.labels, a.labels64, row);
          if (id >= 0 && id < a.vocab) {
            y = (int32_t)id;
            sh.z[a.k] = to_float(z[y]);
            sh.p[a.k] = a.loss_label;
            if (a.loss_label != 0.0f) loss += a.loss_label * (l1 - sh.z[a.k]);
          }
        }
        sh.id[a.k] = y;
        sh.p_sum = p_sum;
        if (a.loss) a.loss[row] = some ? loss : 0.0f;
      }
    }
    if (!a.dlogits) continue;
    __syncthreads();
    const float g = a.grad_loss[row];
    const bool live = g != 0.0f && some;
    const float c0 = g * a.grad_kd * sh.p_sum, c1 = sh.id[a.k] >= 0 ? g * a.loss_label : 0.0f;
    T *d = static_cast<T *>(a.dlogits) + row * a.dpitch;
    auto whole = [&](float x) {
      float v = c0 * exp2_approx(__fmaf_rn(x, a.inv_tau, -l) * kLog2e);
      if (c1 != 0.0f) v += c1 * exp2_approx((x - l1) * kLog2e);
      return v;
    };
    for (uint32_t i = tid; i < a.vocab; i += kThreads) d[i] = from_float<T>(live ? whole(to_float(z[i])) : 0.0f);
    __syncthreads();
    if (!live) continue;
    for (uint32_t i = tid; i <= a.k; i += kThreads) {
      if (sh.id[i] < 0) continue;
      float sum = 0.0f;
      bool first = true;
      for (uint32_t j = 0; j <= a.k; ++j)
        if (sh.id[j] == sh.id[i]) {
          first = first && j >= i;
          sum += sh.p[j];
        }
      if (first) d[sh.id[i]] = from_float<T>(whole(sh.z[i]) - g * sum);
    }
  }
}

}  // namespace

int distill_per_sm(const DistillArgs &) { return 4; }

int launch_distill(const DistillArgs &a, unsigned cap, void *stream) {
  return with_dtype(a.dtype, [&](auto t) {
    distill_kernel<decltype(t)><<<a.rows < cap ? a.rows : cap, kThreads, 0, (cudaStream_t)stream>>>(a);
    return (int)cudaGetLastError();
  });
}

}  // namespace apc
