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
#include "apc_device.cuh"
#include "apc_internal.h"
#include "apc_launch.cuh"

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
__device__ __noinline__ uint4 edge_block(const uint8_t *p, const uint8_t *lo, const uint8_t *hi) {
  uint32_t w[4] = {0, 0, 0, 0};
  for (int i = 0; i < 16; i += 2)
    if (p + i >= lo && p + i < hi) w[i / 4] |= (uint32_t)*reinterpret_cast<const uint16_t *>(p + i) << (i % 4 * 8);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ uint4 block(const uint8_t *p, const uint8_t *lo, const uint8_t *hi) {
  if (p >= lo && p + 16 <= hi) return __ldcs(reinterpret_cast<const uint4 *>(p));
  return p + 16 > lo && p < hi ? edge_block(p, lo, hi) : make_uint4(0, 0, 0, 0);
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

// A warp's tile that begins at `at` in a buffer that ends at `end`: zeros behind the end.
__device__ __forceinline__ void load_tile(uint4 (&x)[kNormGroups], const uint8_t *at, const uint8_t *lo, const uint8_t *end,
                                          uint32_t lane) {
  const uint32_t off = (uint32_t)((uintptr_t)at & 15);
  if (off == 0 && at + kNormTileBytes <= end) {
#pragma unroll
    for (int j = 0; j < kNormGroups; ++j) x[j] = __ldcs(reinterpret_cast<const uint4 *>(at) + j * 32 + lane);
    return;
  }
  // lane 0 holds one block more: the one behind lane 31's last
  const uint8_t *p = at - off + 16 * lane;
#pragma unroll
  for (int j = 0; j < kNormGroups; ++j) x[j] = block(p + j * 512, lo, end);
  if (off == 0) return;
  uint4 more = make_uint4(0, 0, 0, 0);
  if (lane == 0) more = block(p + kNormTileBytes, lo, end);
#pragma unroll
  for (int j = 0; j < kNormGroups; ++j) {
    const uint4 from = lane ? x[j] : j + 1 < kNormGroups ? x[j + 1] : more;
    const int next = (int)(lane + 1) & 31;
    const uint4 b = make_uint4(__shfl_sync(~0u, from.x, next), __shfl_sync(~0u, from.y, next), __shfl_sync(~0u, from.z, next),
                               __shfl_sync(~0u, from.w, next));
    x[j] = cut(x[j], b, off);
  }
}

// A slot's number as a norm: its words, highest first, in double; one rounding to fp32.
__device__ __forceinline__ float norm_of(unsigned long long word, uint32_t lane) {
  double v = lane < (uint32_t)kInf ? (double)word * scalbn(1.0, 32 * (int)lane - kNormBias) : 0.0;
  const bool nan = __shfl_sync(~0u, word, kNan) != 0, inf = __shfl_sync(~0u, word, kInf) != 0;
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return nan ? __uint_as_float(0x7fffffffu) : inf ? __uint_as_float(0x7f800000u) : (float)sqrt(v);
}

template <int MAXE>
__global__ void __launch_bounds__(kNormThreads, 1) norm_kernel(const __grid_constant__ DigestPlan<MAXE> plan,
                                                               unsigned long long *work, float *out, uint32_t slots) {
  __shared__ unsigned long long s_bins[APC_MAX_SLOTS][kBins];
  __shared__ bool s_last;
  if (plan.more) chain_start_next();
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x < APC_MAX_SLOTS * kBins) s_bins[threadIdx.x / kBins][threadIdx.x % kBins] = 0;
  __syncthreads();
  // this CTA's run of tiles, walked by its warps
  const uint64_t per = plan.total_tiles / gridDim.x, rem = plan.total_tiles % gridDim.x;
  const uint64_t t_begin = blockIdx.x * per + (blockIdx.x < rem ? blockIdx.x : rem);
  const uint32_t len = (uint32_t)(per + (blockIdx.x < rem ? 1 : 0));
  uint32_t cur = 0, r = warp;
  int slot = -1;
  uint64_t word = 0;
  while (r < len) {
    cur = entry_of(plan, cur, t_begin + r);
    const DigestEntry &E = plan.e[cur];
    const uint64_t left = (cur + 1 < plan.count ? plan.e[cur + 1].tile_begin : plan.total_tiles) - t_begin;
    const uint32_t stop = left < len ? (uint32_t)left : len;
    if ((int)E.slot != slot) {
      if (slot >= 0 && word) atomicAdd(&s_bins[slot][lane], (unsigned long long)word);
      word = 0;
      slot = E.slot;
    }
    const uint8_t *lo = static_cast<const uint8_t *>(E.data), *end = lo + E.n * (E.dtype == APC_F32 ? 4 : 2);
    const uint8_t *at = lo + (t_begin + r - E.tile_begin) * kNormTileBytes;
    for (; r < stop; r += kWarps, at += kWarps * kNormTileBytes) {
      uint4 x[kNormGroups];
      load_tile(x, at, lo, end, lane);
      if (E.dtype == APC_BF16) add_tile<APC_BF16>(x, word, lane);
      else if (E.dtype == APC_F32) add_tile<APC_F32>(x, word, lane);
      else add_tile<APC_F16>(x, word, lane);
    }
  }
  if (slot >= 0 && word) atomicAdd(&s_bins[slot][lane], (unsigned long long)word);
  __syncthreads();
  chain_wait();
  if (threadIdx.x < slots * kBins) {
    const unsigned long long b = s_bins[threadIdx.x / kBins][threadIdx.x % kBins];
    if (b) atomicAdd(&work[1 + threadIdx.x], b);
  }
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
  const DigestPlan<MAXE> &p = *static_cast<const DigestPlan<MAXE> *>(plan);
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kNormThreads);
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = &attr;
  cfg.numAttrs = p.chained ? 1 : 0;
  return (int)cudaLaunchKernelEx(&cfg, norm_kernel<MAXE>, p, work, out, slots);
}

}  // namespace

int launch_norm(const void *plan, int size, unsigned grid, void *stream, unsigned long long *work, float *out, unsigned slots) {
  return size == kDigestSmall ? launch_n<kDigestSmall>(plan, grid, stream, work, out, slots)
         : size == kDigestMid ? launch_n<kDigestMid>(plan, grid, stream, work, out, slots)
                              : launch_n<kDigestLarge>(plan, grid, stream, work, out, slots);
}

}  // namespace apc
