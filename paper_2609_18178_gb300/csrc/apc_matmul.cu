// The product of two block-scaled 8-bit matrices (apc_matmul_fp8).
//
// One CTA computes a 64 x 64 tile of out: operands are widened into shared
// memory, a block of 128 k at a time, its products summed in fp32, and the
// sums added with both scales.
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include "apc_ops.cuh"

namespace apc {

namespace {

constexpr int kTile = 64, kStep = 32;

__device__ __forceinline__ float widen(uint8_t v, bool e5m2) {
  const __half_raw h = __nv_cvt_fp8_to_halfraw(v, e5m2 ? __NV_E5M2 : __NV_E4M3);
  return __half2float(__half(h));
}

template <typename T>
__global__ void __launch_bounds__(256) matmul_kernel(const __grid_constant__ MatmulArgs p) {
  __shared__ float sa[kStep][kTile + 1], sb[kStep][kTile + 1];
  const uint32_t tm = (p.m + kTile - 1) / kTile, tn = (p.n + kTile - 1) / kTile;
  const uint32_t tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (uint64_t tile = blockIdx.x; tile < (uint64_t)tm * tn; tile += gridDim.x) {
    const uint32_t m0 = (uint32_t)(tile / tn) * kTile, n0 = (uint32_t)(tile % tn) * kTile;
    float acc[4][4] = {};
    for (uint32_t kb = 0; kb * kBlock < p.k; ++kb) {
      float part[4][4] = {};
      for (uint32_t k0 = kb * kBlock; k0 < min(p.k, (kb + 1) * kBlock); k0 += kStep) {
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < kTile * kStep; i += 256) {
          const uint32_t r = i / kStep, c = i % kStep;
          const bool in = k0 + c < p.k;
          sa[c][r] = in && m0 + r < p.m ? widen(p.a[(m0 + r) * p.a_pitch + k0 + c], p.a_e5m2) : 0.0f;
          sb[c][r] = in && n0 + r < p.n ? widen(p.b[(n0 + r) * p.b_pitch + k0 + c], p.b_e5m2) : 0.0f;
        }
        __syncthreads();
        for (int c = 0; c < kStep; ++c)
          for (int i = 0; i < 4; ++i)
            for (int j = 0; j < 4; ++j) part[i][j] = __fmaf_rn(sa[c][ty * 4 + i], sb[c][tx + 16 * j], part[i][j]);
      }
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
          const uint32_t m = m0 + ty * 4 + i, n = n0 + tx + 16 * j;
          if (m < p.m && n < p.n)
            acc[i][j] = __fmaf_rn(part[i][j], p.a_scale[kb * p.a_scale_pitch + (m >> p.a_shift)] *
                                                  p.b_scale[kb * p.b_scale_pitch + (n >> p.b_shift)], acc[i][j]);
        }
    }
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j) {
        const uint32_t m = m0 + ty * 4 + i, n = n0 + tx + 16 * j;
        if (m < p.m && n < p.n) static_cast<T *>(p.out)[m * p.out_pitch + n] = from_float<T>(acc[i][j]);
      }
  }
}

}  // namespace

int launch_matmul(const MatmulArgs &a, unsigned cap, void *stream) {
  const uint64_t tiles = (uint64_t)((a.m + kTile - 1) / kTile) * ((a.n + kTile - 1) / kTile);
  return with_dtype(a.out_dtype, [&](auto t) {
    const uint64_t most = (uint64_t)cap * 4;
    matmul_kernel<decltype(t)><<<(unsigned)(tiles < most ? tiles : most), 256, 0, (cudaStream_t)stream>>>(a);
    return (int)cudaGetLastError();
  });
}

}  // namespace apc
