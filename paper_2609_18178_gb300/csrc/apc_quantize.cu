// Quantization to 8 bits with a power-of-two scale per block (apc_quantize_fp8).
//
// One CTA takes one block at a time: 1 x 128 values of a row of x (or, for the
// transpose, 128 x 1 of a column) or a 128 x 128 tile.
#include <cuda_runtime.h>

#include "apc_ops.cuh"

namespace apc {

namespace {

constexpr int kThreads = 128;

// 2^e with 2^e * top >= amax > 2^(e-1) * top, e >= -126; 1 for amax = 0.  top is
// 1.75 * 2^8 (E4M3) or 1.75 * 2^15 (E5M2), so only fractions above 1.75 need
// the next power.
__device__ __forceinline__ float scale_of(float amax, bool e5m2) {
  if (amax == 0.0f) return 1.0f;
  int x = 0;
  if (amax < 1.1754944e-38f) amax *= 16777216.0f, x = -24;
  const uint32_t b = __float_as_uint(amax);
  int e = (int)(b >> 23) - 127 + x - (e5m2 ? 15 : 8) + ((b & 0x7fffffu) > 0x600000u);
  e = e < -126 ? -126 : e;
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

__device__ __forceinline__ uint8_t quantize_one(float x, float inv, bool e5m2) {
  const uint32_t b = __float_as_uint(x);
  if ((b & 0x7fffffffu) == 0x7f800000u) return (uint8_t)((e5m2 ? 0x7c : 0x7f) | (b >> 24 & 0x80));
  return (uint8_t)to_fp8x2(x * inv, 0.0f, e5m2);
}

// x viewed with strides: the transpose swaps them.
template <typename T>
__global__ void __launch_bounds__(kThreads) quantize_kernel(const T *x, int64_t sr, int64_t sc, uint32_t rows,
                                                            uint32_t cols, uint32_t height, QuantOut q) {
  __shared__ float s_max[kThreads / 32];
  const uint32_t across = (cols + kBlock - 1) / kBlock;
  const uint64_t blocks = (uint64_t)across * ((rows + height - 1) / height);
  for (uint64_t i = blockIdx.x; i < blocks; i += gridDim.x) {
    const uint32_t bc = (uint32_t)(i % across), br = (uint32_t)(i / across);
    const uint32_t c = bc * kBlock + threadIdx.x, r1 = min(rows, (br + 1) * height);
    float amax = 0.0f;
    if (c < cols)
      for (uint32_t r = br * height; r < r1; ++r) {
        const float v = fabsf(to_float(x[r * sr + c * sc]));
        amax = v <= 3.402823466e38f ? fmaxf(amax, v) : amax;
      }
    for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, o));
    __syncthreads();
    if (threadIdx.x % 32 == 0) s_max[threadIdx.x / 32] = amax;
    __syncthreads();
    amax = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
    const float s = scale_of(amax, q.e5m2), inv = 1.0f / s;
    if (threadIdx.x == 0) q.scale[bc * q.scale_pitch + br] = s;
    if (c < cols)
      for (uint32_t r = br * height; r < r1; ++r)
        q.data[r * q.pitch + c] = quantize_one(to_float(x[r * sr + c * sc]), inv, q.e5m2);
  }
}

}  // namespace

int quantize_per_sm(const QuantArgs &) { return 16; }

int launch_quantize(const QuantArgs &a, unsigned cap, void *stream) {
  const uint32_t height = a.square ? kBlock : 1;
  return with_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    for (int k = 0; k < (a.qt.data ? 2 : 1); ++k) {
      const uint32_t rows = k ? a.cols : a.rows, cols = k ? a.rows : a.cols;
      const uint64_t blocks = (uint64_t)((cols + kBlock - 1) / kBlock) * ((rows + height - 1) / height);
      quantize_kernel<T><<<(unsigned)(blocks < cap ? blocks : cap), kThreads, 0, (cudaStream_t)stream>>>(
          static_cast<const T *>(a.x), k ? 1 : a.pitch, k ? a.pitch : 1, rows, cols, height, k ? a.qt : a.q);
      const int e = (int)cudaGetLastError();
      if (e) return e;
    }
    return 0;
  });
}

}  // namespace apc
