// What the norm's kernels (apc_rmsnorm.cu) and its gradient's (apc_rmsnorm_grad.cu) share:
// a row over a group of threads, the ring of shared memory that many rows come through,
// shapes and launches.
#pragma once

#include <cuda_runtime.h>

#include "../../include/apc.h"
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

// Plain loads: outputs may take the place of what is read.
template <typename T, bool WIDE>
__device__ __forceinline__ void load(uint32_t (&w)[8 / Word<T>::kPer], const T *x, int n) {
  if (WIDE) {
    load8<T, Read::kPlain>(w, x, n, true);
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

__device__ __forceinline__ void group_sync(uint32_t id, uint32_t threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// A group of threads that share a row.
struct Group {
  uint32_t warps, id, warp, lane;

  __device__ void sync() const {
    if (warps > 1) group_sync(id, warps * 32);
  }
  // for those who do not wait in a sync() of the others, and a barrier of its own behind it
  __device__ void arrive() const { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(warps * 32) : "memory"); }
  __device__ void sync_again() const { group_sync(id + 8, warps * 32); }
};

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

constexpr uint32_t kStagesMost = 3, kRingBytes = 220 * 1024;

struct Ring {
  uint32_t stages, region, mats;  // region: bytes of a matrix's part of a stage
  uint32_t weights;               // bytes of the weights
  uint32_t edges;                 // 1: the first row's first block begins in front of the matrix, 2: the last one's last ends behind
  unsigned *status;

  __host__ __device__ uint32_t stage() const { return region * mats; }
  __host__ __device__ uint32_t bytes() const { return stages * stage() + weights; }
};

// A warp's sum of squares: (sum + low * 2^-20) * 2^(e - 152).
struct __align__(16) Stat {
  uint32_t sum, e;
  int32_t low;
};

struct RingShared {
  uint64_t full[kStagesMost];
  Stat stats[2][33];
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

// The bounded wait for a stage.  After one that gave up nothing more is copied and no stage
// waited for; what follows is not to be used, as the status word says.  Copies that are under way
// have to land before the CTA ends (ring_end).
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

// One thread: copy a row of each matrix into a stage.  How many rows that were: 1, or 0 after a
// wait that gave up.
template <int M>
__device__ __forceinline__ uint32_t ring_issue(RingShared &sh, const Source (&src)[M], const Ring &ring, uint8_t *stage, uint64_t *full,
                                           uint32_t row, uint32_t rows, uint32_t cols, uint32_t size, uint64_t policy) {
  if (*(volatile int *)&sh.dead) return 0;
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
  return 1;
}

// The thread that issued: after a wait that gave up, the (bounded) ones for the last copy into each
// stage, of `issued` rows that went into the stages in turn.
__device__ __forceinline__ void ring_end(RingShared &sh, uint32_t stages, uint32_t issued) {
  if (threadIdx.x || !*(volatile int *)&sh.dead) return;
  for (uint32_t u = issued > stages ? issued - stages : 0; u < issued; ++u) mbar_wait(&sh.full[u % stages], u / stages & 1);
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

bool aligned(const void *p, int64_t pitch_bytes) { return (uintptr_t)p % 16 == 0 && pitch_bytes % 16 == 0; }

// More rows than `least`, of 16 bits, alike within 16 bytes: the ring's shape, or none (threads
// 0).  Where rows begin at blocks and end with them, plain loads by more warps keep up with it
// for some (pays): 8192 x 4096 to 8 bits takes 45 us (47 by plain loads), to 16 bits without a residual
// 31 (34), its gradient 50 (60), but the gradient of 16384 x 1024 33 (30).  To 16 bits with a residual
// plain loads are ahead, and this rule takes the ring all the same: 8192 x 4096 48 us (45), 1221 x
// 16384 44 (34).  fp32 rows do better without it too: 4883 x 4096 52 us (60).  Elsewhere in the matrix
// 16-bit rows need it: 4001 x 5001 to 16 bits 36 us (41), its gradient 49 (94).
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
  // units a thread: with more than registers have room for, or barriers to wait for, fewer threads do more
  s.v = grad ? units <= 1024 ? 1 : 2 : units <= 512 && mats == 2 ? 1 : 2;
  if (grad && s.v == 2) mats = 2;
  s.threads = 32 * ((units + 32 * s.v - 1) / (32 * s.v));
  s.ring.region = (cols * size + 15 + 15) / 16 * 16 + 16;
  s.ring.mats = mats;
  s.ring.weights = s.threads * s.v * 32;
  s.ring.edges = ((uintptr_t)x % 16 != 0) | (((uintptr_t)x + ((int64_t)(rows - 1) * pitch + cols) * size) % 16 != 0) << 1;
  for (s.ring.stages = 3; s.ring.stages > 1 && s.ring.bytes() > kRingBytes; --s.ring.stages) {}
  if (s.ring.stages < 2) s.threads = 0;
  return s;
}

// The launch of a ring kernel: persistent, in so many CTAs as an SM holds, rows of a CTA
// beginning alike where the grid allows.
template <typename K, typename A>
int ring_launch(K kernel, const A &a, RingShape s, uint32_t work, uint32_t period, void *stream) {
  const uint32_t bytes = s.ring.bytes();
  int e = commit_status_word(&s.ring.status), per_sm = 1;
  // the limit is what any launch takes: a call of another thread sets it too
  if (!e) e = (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes);
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

}  // namespace
}  // namespace apc
