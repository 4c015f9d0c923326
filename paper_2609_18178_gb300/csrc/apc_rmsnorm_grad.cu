// The gradient of the root-mean-square norm (apc_rms_norm_grad): with z = h * rstd and
// g = dout * weight,
//
//   dx = (g - z * mean of g*z) * rstd + dresidual,  dweight = sum over rows of dout * z
//
// One read of each input and one write of each output, a few operations for each element:
// bound by memory.
#include "apc_cluster.cuh"
#include "apc_rmsnorm.cuh"

namespace apc {

namespace {

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
  constexpr int kRes = kAgain ? 2 : V;
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
      uint32_t x[U][V][kWords], d[U][V][kWords], r[U][kRes][kWords];
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
        const auto late = [&](int v) {  // one ahead of the stores, which it might not pass
          if (kAgain && a.dresidual)
            load<T, WIDE>(r[u][v % kRes], static_cast<const T *>(a.dresidual) + (int64_t)row * a.dresidual_pitch + c[v], n[v]);
        };
        late(0);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          uint32_t o[kWords], (&res)[kWords] = r[u][v % kRes];
          uint64_t(&w)[4] = wt[kAgain ? 0 : v];
          if (kAgain) weights<WIDE>(w, a.weight, a.wdtype, a.weight_aligned, c[v], n[v]);
          if (v + 1 < V) late(v + 1);
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
    // wide units go by way of shared memory, a warp's stores to the workspace being neighbours: 4-byte
    // stores 32 bytes apart took 5 us more for 304 parts of 4,096 columns; but long rows' weights need L1
    const bool alone = !CLUSTER && (!WIDE || kAgain) && blockDim.y == 1;
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
  if (blockDim.y > 1) {  // the CTA's groups first
    __syncthreads();
    for (uint32_t k = threadIdx.y * blockDim.x + threadIdx.x; k < a.cols; k += blockDim.x * blockDim.y) {
      float s = 0.0f;
      for (uint32_t r = 0; r < blockDim.y; ++r) s += part_sums[r * a.cols + k];
      part_sums[k] = s;
    }
  }
  cluster_arrive();
  cluster_wait();
  // a slice of the columns for each CTA
  const uint32_t per = (a.cols + gridDim.x - 1) / gridDim.x, begin = blockIdx.x * per, end = min(a.cols, begin + per);
  for (uint32_t k = begin + threadIdx.y * blockDim.x + threadIdx.x; k < end; k += blockDim.x * blockDim.y) {
    const uint32_t at = smem_addr(part_sums + k);
    float s = 0.0f;
    for (uint32_t q = 0; q < gridDim.x; q += 8) {  // a power of two of CTAs
      float f[8];
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) f[i] = q + i < gridDim.x ? load_remote(map_rank(at, q + i)) : 0.0f;
      s += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
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
  if (a.partial) {
    wait_for_first();
    start_next();
  }
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

// dweight: the parts' sums, 32 columns a CTA, warp k those of parts k, k + 32, ..., ten loads of a
// lane under way, then the warps'.  Two CTAs on an SM pay once there are more than SMs: 300 x 4096
// took 8.5 us with both in place of 7.7, 1221 x 16384 69.9 in place of 73.3.
template <int PER_SM>
__global__ void __launch_bounds__(1024, PER_SM) parts_kernel(const float *partial, uint32_t parts, uint32_t cols, void *dweight, uint32_t dtype) {
  __shared__ float sums[32][33];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint32_t runs = (cols + 31) / 32;
  wait_for_first();
  for (uint32_t run = blockIdx.x; run < runs; run += gridDim.x) {
    const uint32_t c = run * 32 + lane;
    float s = 0.0f;
    if (c < cols)
      for (uint32_t p = warp; p < parts; p += 320) {
        float f[10];
#pragma unroll
        for (uint32_t i = 0; i < 10; ++i) f[i] = p + 32 * i < parts ? __ldcg(partial + (uint64_t)(p + 32 * i) * cols + c) : 0.0f;
        s += (((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]))) + (f[8] + f[9]);
      }
    __syncthreads();
    sums[warp][lane] = s;
    __syncthreads();
    float y = sums[lane][warp];  // column `warp`, a part of it in each lane
#pragma unroll
    for (int o = 16; o; o >>= 1) y += __shfl_xor_sync(~0u, y, o);
    if (lane == 0 && run * 32 + warp < cols) store_weight(dweight, dtype, run * 32 + warp, y);
  }
}

// A unit's elements from global memory.
template <typename T, bool WHOLE>
__device__ __forceinline__ void unit_load(uint32_t (&w)[8 / Word<T>::kPer], const T *row, const Unit<WHOLE> &u, uint32_t cols) {
  static_assert(sizeof(T) == 2, "");
  if (u.full) {
    const uint4 v = *reinterpret_cast<const uint4 *>(row + u.first);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = 0;
  if (WHOLE || !u.any) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int32_t c = u.first + i;
    if (c >= 0 && c < (int32_t)cols) w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[c] << (i % 2 * 16);
  }
}

// The gradient's rows through a ring of x, dout and dresidual.  Part p is rows p, p + parts,
// ...: rows of a part begin alike.  Rows of more than 1,024 units, two a thread (V): two stages of x
// and dout are what fits, dresidual comes into registers, and z and g are formed twice.  Bound:
// memory, at 5.8 TB/s for 8192 x 4096 (45.5 us of 50, then the parts); above 8,192 columns the wait
// for the one row under way: 1221 x 16384 in 49 us, by plain loads 67.
template <typename T, int V, bool WHOLE>
__global__ void __launch_bounds__(1024, 1) ring_grad_kernel(const __grid_constant__ GradArgs a, const __grid_constant__ Ring ring) {
  constexpr int kWords = 8 / Word<T>::kPer;
  constexpr bool kAgain = V > 1;
  extern __shared__ __align__(128) uint8_t s_ring[];
  __shared__ RingShared sh;
  const Group g{blockDim.x / 32, 0, threadIdx.x / 32, threadIdx.x % 32};
  const uint32_t units = V * blockDim.x;
  float *const laid = reinterpret_cast<float *>(s_ring + ring.stages * ring.stage());
  if (a.partial) start_next();
  constexpr int kMats = kAgain ? 2 : 3;
  Source src[kMats] = {{a.x, a.pitch}, {a.dout, a.dout_pitch}};
  if constexpr (!kAgain) src[2] = {a.dresidual, a.dresidual_pitch};
  uint32_t next_part = blockIdx.x, next = next_part, into = 0, issued = 0;
  const auto issue = [&]() {
    if (next_part < a.parts) {
      issued += ring_issue<kMats>(sh, src, ring, s_ring + into * ring.stage(), &sh.full[into], next, a.rows, a.cols, sizeof(T), l2_evict_first());
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
      if (!WHOLE && ring.edges) ring_edges<T, kMats>(src, ring, at, row, a.rows, a.cols);
      uint64_t z[kAgain ? 1 : V][4], gg[kAgain ? 1 : V][4], dot = 0;
      const auto form = [&](int v, auto each) {
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
          z_and_g<T>(x, d, rstd, wt, i, &z[kAgain ? 0 : v][i], &gg[kAgain ? 0 : v][i], &dd);
          each(i, dd);
        }
      };
      uint32_t res[kAgain ? V : 1][kWords];
      if (kAgain && a.dresidual)
#pragma unroll
        for (int v = 0; v < V; ++v)
          unit_load<T, WHOLE>(res[kAgain ? v : 0], static_cast<const T *>(a.dresidual) + (int64_t)row * a.dresidual_pitch,
                              Unit<WHOLE>(threadIdx.x + v * blockDim.x, skip / sizeof(T), a.cols), a.cols);
#pragma unroll
      for (int v = 0; v < V; ++v)
        form(v, [&](int i, uint64_t dd) {
          dot = fma2(gg[kAgain ? 0 : v][i], z[kAgain ? 0 : v][i], dot);
          acc[v][i] = fma2(dd, z[kAgain ? 0 : v][i], acc[v][i]);
        });
      const float2 both = unpack2(dot);
      const float mean = group_sum(both.x + both.y, g, sh.sums[turn ^= 1]) * a.inv_cols;
      if (threadIdx.x == 0) issue();  // into the stage of the row before, which all have left
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const uint32_t k = threadIdx.x + v * blockDim.x;
        const Unit<WHOLE> u(k, skip / sizeof(T), a.cols);
        if (kAgain) form(v, [](int, uint64_t) {});
        uint32_t o[kWords];
        uint32_t(&r)[kWords] = kAgain ? res[kAgain ? v : 0] : o;
        if (!kAgain && a.dresidual) ring_load<T, WHOLE>(o, at + 2 * ring.region, k, u, a.cols);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint64_t(&zv)[4] = z[kAgain ? 0 : v], (&gv)[4] = gg[kAgain ? 0 : v];
          float2 f = unpack2(mul2(fma2(zv[i], pack2(-mean, -mean), gv[i]), pack2(rstd, rstd)));
          if (a.dresidual) f.x += element<T>(r, 2 * i), f.y += element<T>(r, 2 * i + 1);
          round_pair<T>(o, i, f.x, f.y);
        }
        ring_store<T, WHOLE>(static_cast<T *>(a.dx) + (int64_t)row * a.dx_pitch, o, u, a.cols);
      }
      if (++stage == ring.stages) stage = 0, parity ^= 1;
    }
    if (!a.partial) continue;
    // by way of the stage that the last row has left, as in grad_kernel
    float *const sums = reinterpret_cast<float *>(s_ring + (stage ? stage - 1 : ring.stages - 1) * ring.stage());
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const Unit<WHOLE> u(threadIdx.x + v * blockDim.x, skip / sizeof(T), a.cols);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 f = unpack2(acc[v][i / 2]);
        if (u.first + i >= 0 && u.first + i < (int32_t)a.cols) sums[u.first + i] = i % 2 ? f.y : f.x;
      }
    }
    __syncthreads();
    for (uint32_t k = threadIdx.x; k < a.cols; k += blockDim.x) a.partial[(uint64_t)part * a.cols + k] = sums[k];
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the next copy comes behind a barrier
  }
  ring_end(sh, ring.stages, issued);
}

// Few rows: a cluster of so many CTAs (0: none) of so many groups, up to 8 rows for each.  It
// saves 2.4 us of host time: 64 x 1024 takes 4.6 us of kernel time (5.1 by two kernels), 64 x
// 4096 7.8 (6.4), 128 x 4096 would take 10.4 (6.5) and 1000 x 500 11.8 (7.3).
struct Few {
  uint32_t ctas, groups;
};

constexpr int kSumsBytes = 72 * 1024;  // shared memory of any launch of grad_kernel: 16,384 columns in one group

Shape grad_shape(uint32_t cols) { return shape_of(cols, cols <= 256 ? 1 : cols <= 8192 ? 2 : 4); }

uint32_t grad_ctas(uint32_t cols) { return cols <= 4096 ? 304 : 152; }

Few few_of(uint32_t rows, uint32_t cols) {
  const Shape s = grad_shape(cols);
  if (!rows || !s.fits || (uint64_t)rows * cols > 1u << 18) return {0, 0};
  Few f = {1, 1};
  while (f.ctas < 16 && f.ctas < rows) f.ctas *= 2;
  const uint32_t most = s.threads >= 512 ? 1 : 512 / s.threads, want = (rows + 15) / 16;
  if (rows > 16) f.groups = want < most ? want : most;
  return rows > 8 * f.ctas * f.groups ? Few{0, 0} : f;
}

}  // namespace

// Parts: two CTAs for every SM, above 4,096 columns one, which is what an SM then holds, or as
// many groups (the ring's CTAs are one); none where a cluster does it.
uint32_t rms_norm_parts(uint32_t rows, uint32_t cols) {
  if (few_of(rows, cols).ctas) return 0;
  const uint32_t parts = grad_ctas(cols) * grad_shape(cols).groups;
  return rows < parts ? rows : parts;
}

namespace {

template <typename K>
int grad_few(K kernel, const GradArgs &a, const Shape &s, const Few &few, cudaStream_t stream) {
  const uint32_t bytes = (2 * few.groups * (s.threads / 32) + few.groups * a.cols) * sizeof(float);
  int e = (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSumsBytes);
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
  // dx's bits are the same with dweight and without: few rows take the plain kernel either way
  // (400 x 601 bf16 without dweight 2.9 us, through the ring 4.5)
  const Few rows = few_of(n.rows, n.cols), few = n.dweight ? rows : Few{0, 0};
  a.parts = few.ctas ? few.ctas : n.rows < grad_ctas(n.cols) ? n.rows : grad_ctas(n.cols);
  if (few.ctas) a.partial = nullptr, a.dweight = n.dweight, a.dwdtype = n.dwdtype;
  a.weight_aligned = (uintptr_t)n.weight % 16 == 0;
  a.inv_cols = (float)(1.0 / n.cols);
  cudaStream_t s = (cudaStream_t)stream;
  const Shape sh = grad_shape(n.cols);
  const int e = !n.rows ? 0 : with_dtype(n.dtype, [&](auto t) {
    using T = decltype(t);
    const auto at = [](const void *p, int64_t pitch) { return aligned(p, pitch * (int64_t)sizeof(T)); };
    if (!sh.fits) {  // dweight's sums first: dx may take dout's place
      const unsigned grid = grid_of(n.rows, 1);
      if (!a.partial) {
        grad_long_kernel<T><<<grid, 1024, 0, s>>>(a);
        return (int)cudaGetLastError();
      }
      grad_long_parts_kernel<T><<<grid_of((uint64_t)((n.cols + 255) / 256) * a.parts, 8), 256, 0, s>>>(a);
      const int e = (int)cudaGetLastError();
      return e ? e : launch_after(grad_long_kernel<T>, grid, 1024, 0, s, a);
    }
    const auto alike = [&](const void *p, int64_t pitch) {
      return same_place(n.x, n.pitch * (int64_t)sizeof(T), p, pitch * (int64_t)sizeof(T));
    };
    const RingShape ring = ring_shape(n.x, n.pitch, n.rows, n.cols, sizeof(T), n.dresidual ? 3 : 2, 2 * sms, true,
                                      alike(n.dout, n.dout_pitch) && alike(n.dresidual, n.dresidual_pitch) && alike(n.dx, n.dx_pitch),
                                      n.cols >= 2048);
    if constexpr (sizeof(T) == 2) if (ring.threads && !rows.ctas) {
      a.parts = n.dweight ? rms_norm_parts(n.rows, n.cols) : n.rows;
      const uint32_t period = period_of(n.pitch * (int64_t)sizeof(T));
      if (ring.whole)
        return ring.v == 1 ? ring_launch(ring_grad_kernel<T, 1, true>, a, ring, a.parts, period, stream)
                           : ring_launch(ring_grad_kernel<T, 2, true>, a, ring, a.parts, period, stream);
      return ring.v == 1 ? ring_launch(ring_grad_kernel<T, 1, false>, a, ring, a.parts, period, stream)
                         : ring_launch(ring_grad_kernel<T, 2, false>, a, ring, a.parts, period, stream);
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
    return with_shape([&](auto kernel, auto) {
      const uint32_t room = (2 * sh.groups * (sh.threads / 32) + (a.partial && (sh.groups > 1 || (wide && sh.v < 4)) ? sh.groups * n.cols : 0)) * sizeof(float);
      const int e = room <= 48 * 1024 ? 0 : (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSumsBytes);
      if (e) return e;
      kernel<<<grid_of(a.parts, 2), dim3(sh.threads, sh.groups), room, s>>>(a);
      return (int)cudaGetLastError();
    });
  });
  if (e || !n.dweight || few.ctas) return e;
  const uint32_t runs = (n.cols + 31) / 32;
  const auto kernel = runs <= sms ? parts_kernel<1> : parts_kernel<2>;
  const unsigned grid = grid_of(runs, 2);
  const float *work = n.work;
  if (n.rows) return launch_after(kernel, grid, 1024, 0, s, work, a.parts, n.cols, n.dweight, n.dwdtype);
  kernel<<<grid, 1024, 0, s>>>(work, a.parts, n.cols, n.dweight, n.dwdtype);
  return (int)cudaGetLastError();
}

}  // namespace apc
