// The 2-norm of all elements of a list of buffers, per slot (apc_grad_norm):
//
//   norm = sqrt(sum of x^2)
//
// One read of every element and a multiply-add for it: bound by HBM.  The result
// does not depend on the grid, on how a list is split into launches or on where
// in memory a buffer lies, so replicas clip by the same factor:
//  * a tile is kNormTileBytes of one buffer, counted from its first element; a
//    warp sums a tile's squares in fp32 in a fixed order (16-byte chunk k of the
//    tile is lane k % 32's, whatever the buffer's alignment);
//  * tiles' sums are added exactly, as integers: a sum's 24 bits go into a
//    512-bit fixed-point number of which lane j of a warp holds the 32 bits
//    of weight 2^(32 j - kNormBias) on, in 64-bit registers.  Integer addition
//    has no order, so atomics may join the warps' numbers.
// A tile whose fp32 sum leaves [2^-90, largest finite] (values beyond 2^60 or below
// 2^-50) is summed again scaled by its largest magnitude.  The last CTA to finish
// turns the total into a norm.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "../../include/apc.h"
#include "apc_cluster.cuh"
#include "apc_device.cuh"
#include "apc_internal.h"
#include "apc_tma.cuh"

namespace apc {
namespace {

constexpr int kWarps = kNormThreads / 32;
constexpr int kBins = kNormWords;      // lanes 0-20 the number, 30 infinities, 31 NaNs
constexpr int kInf = 30, kNan = 31;
constexpr int kNormBias = 352;
static_assert(APC_GRAD_NORM_WORKSPACE == (APC_MAX_SLOTS * kBins + 1) * 8, "a ticket and each slot's words");

// A pair of 16-bit elements as fp32, or two fp32 elements.
template <uint32_t DTYPE>
__device__ __forceinline__ uint64_t widen(uint32_t w) {
  if (DTYPE == APC_BF16) return (uint64_t)(w & 0xffff0000u) << 32 | w << 16;
  const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
  return pack2(f.x, f.y);
}

// acc + the squares of a chunk's elements, each times scale^2, in two pairs of sums.
template <uint32_t DTYPE, bool SCALED>
__device__ __forceinline__ void squares(uint4 x, uint64_t (&acc)[2], uint64_t scale) {
  uint64_t v[4];
  int n = 4;
  if (DTYPE == APC_F32) {
    v[0] = (uint64_t)x.y << 32 | x.x, v[1] = (uint64_t)x.w << 32 | x.z;
    n = 2;
  } else {
    v[0] = widen<DTYPE>(x.x), v[1] = widen<DTYPE>(x.y), v[2] = widen<DTYPE>(x.z), v[3] = widen<DTYPE>(x.w);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i >= n) break;
    const uint64_t y = SCALED ? mul2(v[i], scale) : v[i];
    acc[i % 2] = fma2(y, y, acc[i % 2]);
  }
}

template <uint32_t DTYPE, bool SCALED>
__device__ __forceinline__ float warp_squares(const uint4 (&x)[kNormGroups], float scale) {
  uint64_t acc[2] = {0, 0};
  const uint64_t both = pack2(scale, scale);
#pragma unroll
  for (int j = 0; j < kNormGroups; ++j) squares<DTYPE, SCALED>(x[j], acc, both);
  float s = (lane0(acc[0]) + lane1(acc[0])) + (lane0(acc[1]) + lane1(acc[1]));
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
  return s;
}

// Magnitude of the largest element of a chunk, as fp32 bits (NaNs largest).
template <uint32_t DTYPE>
__device__ __forceinline__ uint32_t largest(uint4 x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DTYPE == APC_F32) {
      m = max(m, w[i] & 0x7fffffffu);
    } else {
      const uint64_t v = widen<DTYPE>(w[i]) & 0x7fffffff7fffffffull;
      m = max(m, max((uint32_t)v, (uint32_t)(v >> 32)));
    }
  }
  return m;
}

// sum * 2^(2 shift) into the lanes' words.
__device__ __forceinline__ void add_exact(uint64_t &word, float sum, int shift, uint32_t lane) {
  const uint32_t b = __float_as_uint(sum), e = b >> 23;
  const uint32_t m = e ? (b & 0x7fffffu) | 0x800000u : b;
  const uint32_t at = (uint32_t)((int)max(e, 1u) - 150 + 2 * shift + kNormBias);
  const uint64_t v = (uint64_t)m << (at & 31);
  if (lane == at >> 5) word += (uint32_t)v;
  if (lane == (at >> 5) + 1) word += v >> 32;
}

// A tile whose plain sum is zero, tiny, infinite or NaN.
template <uint32_t DTYPE>
__device__ __forceinline__ void awkward(const uint4 (&x)[kNormGroups], uint64_t &word, uint32_t lane) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < kNormGroups; ++j) m = max(m, largest<DTYPE>(x[j]));
  m = __reduce_max_sync(~0u, m);
  if (m == 0) return;
  if (m >= 0x7f800000u) {
    word += lane == (m > 0x7f800000u ? kNan : kInf);
    return;
  }
  // the largest magnitude to [1, 2); subnormal ones by 2^126 at most, which makes them normal
  const int shift = min(max((int)(m >> 23) - 127, -126), 126);
  add_exact(word, warp_squares<DTYPE, true>(x, __uint_as_float((uint32_t)(127 - shift) << 23)), shift, lane);
}

template <uint32_t DTYPE>
__device__ __forceinline__ void add_tile(const uint4 (&x)[kNormGroups], uint64_t &word, uint32_t lane) {
  const float s = warp_squares<DTYPE, false>(x, 1.0f);
  if (s >= 0x1p-90f && s <= 3.402823466e38f) add_exact(word, s, 0, lane);
  else awkward<DTYPE>(x, word, lane);
}

// The aligned 16-byte block at p, with what lies outside [lo, hi) as zeros.
__device__ __forceinline__ uint4 block(const uint8_t *p, const uint8_t *lo, const uint8_t *hi) {
  if (p + 16 <= lo || p >= hi) return make_uint4(0, 0, 0, 0);
  if (p >= lo && p + 16 <= hi) return __ldcs(reinterpret_cast<const uint4 *>(p));
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (p + 2 * i >= lo && p + 2 * i < hi) w[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t *>(p + 2 * i) << (i % 2 * 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// 16 bytes from byte `off` (1 to 15, even) of two neighbouring blocks.
__device__ __forceinline__ uint4 cut(uint4 a, uint4 b, uint32_t off) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (off & 8) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (off & 4) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  const uint32_t bits = (off & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                    __funnelshift_r(w[3], w[4], bits));
}

// A tile that begins at no 16-byte boundary or ends with its buffer: the blocks that hold it,
// and a lane's chunk cut from its own and the next lane's, four shuffles each (60 M in 291 odd
// entries 32 us; 45 with the second block loaded again).  Zeros behind the end.
template <uint32_t DTYPE>
__device__ __noinline__ uint64_t other_tile(const uint8_t *at, const uint8_t *lo, const uint8_t *end, uint64_t word, uint32_t lane) {
  const uint32_t off = (uint32_t)((uintptr_t)at & 15);
  const uint8_t *p = at - off + 16 * lane;
  uint4 x[kNormGroups], more = make_uint4(0, 0, 0, 0);  // more: lane 0's block behind lane 31's last
  if (at - off >= lo && at - off + kNormTileBytes + 16 <= end) {
#pragma unroll
    for (int j = 0; j < kNormGroups; ++j) x[j] = __ldcs(reinterpret_cast<const uint4 *>(p) + j * 32);
    if (lane == 0) more = __ldcs(reinterpret_cast<const uint4 *>(p + kNormTileBytes));
  } else {
#pragma unroll
    for (int j = 0; j < kNormGroups; ++j) x[j] = block(p + j * 512, lo, end);
    if (lane == 0 && off) more = block(p + kNormTileBytes, lo, end);
  }
  if (off) {
    const int next = (int)(lane + 1) & 31;
#pragma unroll
    for (int j = 0; j < kNormGroups; ++j) {
      const uint4 from = lane ? x[j] : j + 1 < kNormGroups ? x[(j + 1) % kNormGroups] : more;
      x[j] = cut(x[j], make_uint4(__shfl_sync(~0u, from.x, next), __shfl_sync(~0u, from.y, next), __shfl_sync(~0u, from.z, next),
                                  __shfl_sync(~0u, from.w, next)), off);
    }
  }
  add_tile<DTYPE>(x, word, lane);
  return word;
}

template <uint32_t DTYPE>
__device__ __noinline__ uint64_t awkward_tile(const uint8_t *at, uint64_t word, uint32_t lane) {
  uint4 x[kNormGroups];
#pragma unroll
  for (int j = 0; j < kNormGroups; ++j) x[j] = __ldcs(reinterpret_cast<const uint4 *>(at) + j * 32 + lane);
  awkward<DTYPE>(x, word, lane);
  return word;
}

// The tiles at `at`, `at` + step, ... of a buffer, `count` of them, into the lanes' words.
template <uint32_t DTYPE>
__device__ __forceinline__ uint64_t add_tiles(const uint8_t *at, const uint8_t *lo, const uint8_t *end, uint32_t count, uint32_t step,
                                              uint64_t word, uint32_t lane) {
  const bool aligned = ((uintptr_t)at & 15) == 0;
  for (; count; --count, at += step) {
    if (!aligned || at + kNormTileBytes > end) {
      word = other_tile<DTYPE>(at, lo, end, word, lane);
      continue;
    }
    uint4 x[kNormGroups];
#pragma unroll
    for (int j = 0; j < kNormGroups; ++j) x[j] = __ldcs(reinterpret_cast<const uint4 *>(at) + j * 32 + lane);
    const float s = warp_squares<DTYPE, false>(x, 1.0f);
    if (s >= 0x1p-90f && s <= 3.402823466e38f) add_exact(word, s, 0, lane);
    else word = awkward_tile<DTYPE>(at, word, lane);
  }
  return word;
}

// A slot's number as a norm: its words, highest first, in double; one rounding to fp32.
__device__ __forceinline__ float norm_of(unsigned long long word, uint32_t lane) {
  double v = lane < (uint32_t)kInf ? (double)word * scalbn(1.0, 32 * (int)lane - kNormBias) : 0.0;
  const bool nan = __shfl_sync(~0u, word, kNan) != 0, inf = __shfl_sync(~0u, word, kInf) != 0;
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return nan ? __uint_as_float(0x7fffffffu) : inf ? __uint_as_float(0x7f800000u) : (float)sqrt(v);
}

// The entry whose tiles hold `tile`, at or after entry `lo`.
template <int MAXE>
__device__ __forceinline__ uint32_t norm_entry(const NormPlan<MAXE> &plan, uint32_t lo, uint32_t tile) {
  uint32_t hi = plan.count;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (plan.tile_begin[mid] <= tile) lo = mid;
    else hi = mid;
  }
  return lo;
}

// CLUSTER: all CTAs are one cluster, which joins its numbers in shared memory; no workspace.
// A small list then takes one launch and nothing else.
template <int MAXE, bool CLUSTER>
__global__ void __launch_bounds__(kNormThreads, 1) norm_kernel(const __grid_constant__ NormPlan<MAXE> plan, unsigned long long *work,
                                                               float *out, uint32_t slots) {
  __shared__ unsigned long long s_bins[APC_MAX_SLOTS * kBins];
  __shared__ bool s_last;
  if (!CLUSTER && plan.more) chain_start_next();
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x < APC_MAX_SLOTS * kBins) s_bins[threadIdx.x] = 0;
  if (CLUSTER) cluster_arrive();
  else __syncthreads();
  // this CTA's run of tiles: its warps walk it interleaved or, where each has few of them, in
  // runs of their own, over entries that follow one another
  const uint32_t per = plan.total_tiles / gridDim.x, rem = plan.total_tiles % gridDim.x;
  const uint32_t t_begin = blockIdx.x * per + min(blockIdx.x, rem), run = per + (blockIdx.x < rem ? 1 : 0);
  const bool short_run = run < 16 * kWarps;
  const uint32_t step = short_run ? 1 : kWarps, len = short_run ? run * (warp + 1) / kWarps : run;
  uint32_t cur = 0, r = short_run ? run * warp / kWarps : warp;
  int slot = -1;
  uint64_t word = 0;
  bool waited = !CLUSTER;
  const auto flush_word = [&]() {
    if (!waited) {
      cluster_wait();
      waited = true;
    }
    if (slot >= 0 && word) atomicAdd(&s_bins[slot * kBins + lane], (unsigned long long)word);
    word = 0;
  };
  while (r < len) {
    if (slot < 0 || !short_run) cur = norm_entry(plan, cur, t_begin + r);
    const uint64_t kind = plan.kind[cur];
    const uint32_t dtype = (uint32_t)(kind & 3), begin = plan.tile_begin[cur];
    const uint32_t stop = min(len, (cur + 1 < plan.count ? plan.tile_begin[cur + 1] : plan.total_tiles) - t_begin);
    if ((int)(kind >> 2 & 7) != slot) {
      flush_word();
      slot = (int)(kind >> 2 & 7);
    }
    const uint8_t *lo = static_cast<const uint8_t *>(plan.data[cur]), *end = lo + (kind >> 5) * (dtype == APC_F32 ? 4 : 2);
    const uint8_t *at = lo + (uint64_t)(t_begin + r - begin) * kNormTileBytes;
    const uint32_t count = (stop - r + step - 1) / step;
    if (dtype == APC_BF16) word = add_tiles<APC_BF16>(at, lo, end, count, step * kNormTileBytes, word, lane);
    else if (dtype == APC_F32) word = add_tiles<APC_F32>(at, lo, end, count, step * kNormTileBytes, word, lane);
    else word = add_tiles<APC_F16>(at, lo, end, count, step * kNormTileBytes, word, lane);
    r += count * step;
    cur += short_run;
  }
  flush_word();
  __syncthreads();
  if (CLUSTER) {
    if (cluster_rank() && threadIdx.x < slots * kBins && s_bins[threadIdx.x])
      asm volatile("red.relaxed.cluster.shared::cluster.add.u64 [%0], %1;" ::"r"(map_rank(smem_addr(&s_bins[threadIdx.x]), 0)),
                   "l"(s_bins[threadIdx.x])
                   : "memory");
    cluster_arrive();
    cluster_wait();
    if (cluster_rank() || warp >= slots) return;
    const float n = norm_of(s_bins[warp * kBins + lane], lane);
    if (lane == 0) out[warp] = n;
    return;
  }
  chain_wait();
  if (threadIdx.x < slots * kBins && s_bins[threadIdx.x]) atomicAdd(&work[1 + threadIdx.x], s_bins[threadIdx.x]);
  if (!plan.last) return;
  // the last CTA of the last launch: what the others added is behind their tickets
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) s_last = atomicAdd(work, 1ull) == gridDim.x - 1;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  if (warp < slots) {
    const float n = norm_of(__ldcg(&work[1 + warp * kBins + lane]), lane);
    if (lane == 0) out[warp] = n;
  }
}

template <int MAXE>
int launch_n(const void *plan, unsigned grid, void *stream, unsigned long long *work, float *out, unsigned slots) {
  const NormPlan<MAXE> &p = *static_cast<const NormPlan<MAXE> *>(plan);
  cudaLaunchAttribute attr = {};
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kNormThreads);
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = &attr;
  if (!work) {
    cfg.gridDim = dim3(norm_cluster(p.total_tiles));
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim = {cfg.gridDim.x, 1, 1};
    cfg.numAttrs = 1;
    const int e = (int)cudaFuncSetAttribute(norm_kernel<MAXE, true>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return e ? e : (int)cudaLaunchKernelEx(&cfg, norm_kernel<MAXE, true>, p, work, out, slots);
  }
  cfg.gridDim = dim3(grid);
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = p.chained ? 1 : 0;
  return (int)cudaLaunchKernelEx(&cfg, norm_kernel<MAXE, false>, p, work, out, slots);
}

}  // namespace

int launch_norm(const void *plan, int size, unsigned grid, void *stream, unsigned long long *work, float *out, unsigned slots) {
  return size == kNormSmall ? launch_n<kNormSmall>(plan, grid, stream, work, out, slots)
         : size == kNormMid ? launch_n<kNormMid>(plan, grid, stream, work, out, slots)
                            : launch_n<kNormLarge>(plan, grid, stream, work, out, slots);
}

}  // namespace apc
