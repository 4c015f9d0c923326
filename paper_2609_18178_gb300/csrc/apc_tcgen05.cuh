// Inline-PTX helpers for the tensor-core kernels: tiled TMA loads, tensor
// memory, tcgen05.mma of 8-bit operands, and barriers across a cluster.
#pragma once

#include <cuda.h>
#include <stdint.h>

#include "apc_cluster.cuh"
#include "apc_tma.cuh"

namespace apc {

// The loops around tcgen05 and TMA run in a whole warp, so that barriers,
// coordinates and descriptors stay in uniform registers, and the instructions
// themselves are elected (elect.sync): with a loop in one lane the issue of
// four products took 600 cycles, more than the products.

// ---- arrivals and copies across a cluster
__device__ __forceinline__ void arrive_remote(uint32_t mapped) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(mapped) : "memory");
}

// The same where nothing but tensor memory was read, which tcgen05.fence orders.  A
// release at cluster scope waits for the thread's memory operations, 1,000
// cycles and more, and would bound the product kernel (1,136 TFLOP/s with it).
__device__ __forceinline__ void arrive_remote_relaxed(uint32_t mapped) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(mapped) : "memory");
}

// Stores a word into another CTA's shared memory and counts its 4 bytes there.
__device__ __forceinline__ void store_async(uint32_t mapped, float v, uint32_t mapped_bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(mapped),
               "r"(__float_as_uint(v)), "r"(mapped_bar)
               : "memory");
}

// Copies `bytes` (a multiple of 16) of this CTA's shared memory into another CTA's
// and counts them there.  One barrier update for the whole copy: 4-byte st.async
// updates one a word, and 16,384 of them took 10 us.
__device__ __forceinline__ void bulk_s2s(uint32_t mapped, uint32_t from, uint32_t bytes, uint32_t mapped_bar) {
  asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(mapped),
               "r"(from), "r"(bytes), "r"(mapped_bar)
               : "memory");
}

// mbar_wait with the clock read only once a wait is a long one: the loops here
// wait for a few hundred cycles again and again, and reading %globaltimer takes
// longer than that.
// dead: given up by another wait of this CTA, which ends this one too.
__device__ __forceinline__ bool wait_for(uint64_t *bar, uint32_t parity, const volatile int32_t *dead = nullptr) {
  const uint32_t a = smem_addr(bar);
  if (mbar_try_wait(a, parity) || mbar_try_wait(a, parity)) return true;
  uint64_t t0 = 0;
  for (uint32_t it = 1;; ++it) {
    if (mbar_try_wait(a, parity)) return true;
    if (dead && *dead) return false;
    if (it == 1024) t0 = global_ns();
    if (it >= kWaitIterations && (it & 1023u) == 0 && global_ns() - t0 > kWaitNanoseconds) return false;
  }
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// ---- tensor memory
template <int PAIR>
__device__ __forceinline__ void tmem_alloc(uint32_t *at, uint32_t columns) {  // a whole warp
  if (PAIR == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(at)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(at)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
}

template <int PAIR>
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {  // the same warp
  if (PAIR == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
  else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of this thread's lane.
__device__ __forceinline__ void tmem_load(uint32_t (&r)[32], uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
      "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at));
}

__device__ __forceinline__ void tmem_load(uint32_t (&r)[16], uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at));
}

__device__ __forceinline__ void tmem_load(uint32_t (&r)[8], uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(at));
}

// Until the loads have landed; r passes through, so that no use of it moves ahead.
__device__ __forceinline__ void tmem_landed(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                 "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                 "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}

__device__ __forceinline__ void tmem_landed(uint32_t (&r)[8]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])
               :
               : "memory");
}

__device__ __forceinline__ void tmem_landed(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}

// ---- tcgen05.mma of 8-bit operands, both K-major in 128-byte rows under the
// 128-byte swizzle (tiles of 8 rows are 1,024 bytes apart).
__device__ __forceinline__ uint64_t operand_desc(uint32_t smem) {
  return (uint64_t)(smem >> 4 & 0x3fff) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}

// One thread of a converged warp issues the four products of a block of 128 k
// (overwriting the accumulator first) and both commits: `done` is arrived on once
// they are complete, `read` too.  Predicated as a whole: a branch around them and
// the warp's return from it cost as much as the products' issue.
template <int PAIR>
__device__ __forceinline__ void mma_block(uint32_t d, uint64_t a, uint64_t b, uint32_t instruction, uint32_t done, uint32_t read) {
  if (PAIR == 2)
    asm volatile(
        "{\n\t.reg .pred q, no, yes;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t.reg .b16 both;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 no, 0, 0;\n\tsetp.eq.b32 yes, 0, 0;\n\tmov.b16 both, 3;\n\t"
        "add.s64 a1, %1, 2;\n\tadd.s64 a2, %1, 4;\n\tadd.s64 a3, %1, 6;\n\t"
        "add.s64 b1, %2, 2;\n\tadd.s64 b2, %2, 4;\n\tadd.s64 b3, %2, 6;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, no;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a1, b1, %3, yes;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a2, b2, %3, yes;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a3, b3, %3, yes;\n\t"
        "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%4], both;\n\t"
        "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%5], both;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(instruction), "r"(done), "r"(read)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred q, no, yes;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 no, 0, 0;\n\tsetp.eq.b32 yes, 0, 0;\n\t"
        "add.s64 a1, %1, 2;\n\tadd.s64 a2, %1, 4;\n\tadd.s64 a3, %1, 6;\n\t"
        "add.s64 b1, %2, 2;\n\tadd.s64 b2, %2, 4;\n\tadd.s64 b3, %2, 6;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, no;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a1, b1, %3, yes;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a2, b2, %3, yes;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a3, b3, %3, yes;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%4];\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(instruction), "r"(done), "r"(read)
        : "memory");
}

// Scales in the tensor cores: E8M0 bytes (a float's biased exponent), one word of
// four for each row, rows l, l + 32, l + 64, l + 96 of 128 side by side in 16 bytes.

// One thread of a converged warp copies three tiles of 128 rows' words, 512 bytes
// apart, to four columns of tensor memory each, in both CTAs of the pair.
__device__ __forceinline__ void copy_scales_pair(uint32_t columns, uint32_t smem) {
  const uint64_t d = (uint64_t)(smem >> 4 & 0x3fff) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
  asm volatile(
      "{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
      "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %3;\n\t"
      "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%1], %4;\n\t"
      "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%2], %5;\n\t}" ::"r"(columns),
      "r"(columns + 4), "r"(columns + 8), "l"(d), "l"(d + 32), "l"(d + 64)
      : "memory");
}

// fp32 accumulators, E8M0 scales; formats: a's << 7 | b's << 10, 0 E4M3, 1 E5M2; byte:
// which of a word's four scales.
__device__ __forceinline__ uint32_t scaled_instruction(uint32_t formats, uint32_t m, uint32_t n, uint32_t byte) {
  return formats | byte << 4 | (n >> 3) << 17 | 1u << 23 | (m >> 7) << 27 | byte << 29;
}

// The four products of a block of 128 k, scaled, added to the accumulator unless
// `first`; `read` is arrived on in both CTAs once they are complete.
__device__ __forceinline__ void mma_scaled_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t instruction, uint32_t scales,
                                                bool first, uint32_t read) {
  asm volatile(
      "{\n\t.reg .pred q, more, yes;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t.reg .b16 both;\n\t"
      "elect.sync _|q, 0xffffffff;\n\t"
      "setp.eq.b32 more, %6, 0;\n\tsetp.eq.b32 yes, 0, 0;\n\tmov.b16 both, 3;\n\t"
      "add.s64 a1, %1, 2;\n\tadd.s64 a2, %1, 4;\n\tadd.s64 a3, %1, 6;\n\t"
      "add.s64 b1, %2, 2;\n\tadd.s64 b2, %2, 4;\n\tadd.s64 b3, %2, 6;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], more;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a1, b1, %3, [%4], [%5], yes;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a2, b2, %3, [%4], [%5], yes;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a3, b3, %3, [%4], [%5], yes;\n\t"
      "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%7], both;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(instruction), "r"(scales), "r"(scales + 4), "r"((uint32_t)first), "r"(read)
      : "memory");
}

// One thread's products and copies so far, in both CTAs.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t.reg .b16 both;\n\telect.sync _|q, 0xffffffff;\n\tmov.b16 both, 3;\n\t"
      "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], both;\n\t}" ::"r"(bar)
      : "memory");
}

// One thread of a converged warp announces `bytes` on `bar` and loads a box of each
// operand, both in the same columns.
__device__ __forceinline__ void load_block(uint32_t dst, const CUtensorMap *r, int32_t r0, uint32_t c_dst, const CUtensorMap *c,
                                           int32_t c0, int32_t x, uint32_t bar, uint32_t bytes) {
  asm volatile(
      "{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
      "@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%7], %8;\n\t"
      "@q cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%6, %2}], [%7];\n\t"
      "@q cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%3], [%4, {%6, %5}], [%7];\n\t}" ::"r"(dst),
      "l"(r), "r"(r0), "r"(c_dst), "l"(c), "r"(c0), "r"(x), "r"(bar), "r"(bytes)
      : "memory");
}

// The same for a pair of CTAs, whose first one's barrier `first_bar` counts both's
// boxes; bytes: announced on this CTA's `bar`, 0 in the second.
__device__ __forceinline__ void load_block_pair(uint32_t dst, const CUtensorMap *r, int32_t r0, uint32_t c_dst, const CUtensorMap *c,
                                                int32_t c0, int32_t x, uint32_t first_bar, uint32_t bar, uint32_t bytes) {
  asm volatile(
      "{\n\t.reg .pred q, t;\n\telect.sync _|q, 0xffffffff;\n\tsetp.ne.and.b32 t, %9, 0, q;\n\t"
      "@t mbarrier.arrive.expect_tx.shared::cta.b64 _, [%8], %9;\n\t"
      "@q cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%6, %2}], [%7];\n\t"
      "@q cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%3], [%4, {%6, %5}], "
      "[%7];\n\t}" ::"r"(dst),
      "l"(r), "r"(r0), "r"(c_dst), "l"(c), "r"(c0), "r"(x), "r"(first_bar), "r"(bar), "r"(bytes)
      : "memory");
}

// A place in a ring and the parity of its current use.  A consumer waits for
// `phase`, a producer for the use before: phase ^ 1, which a new barrier passes.
template <int N>
struct Turn {
  uint32_t at = 0, phase = 0;
  __device__ __forceinline__ void next() {
    if (++at == N) at = 0, phase ^= 1;
  }
  __device__ __forceinline__ void skip(uint32_t n) {
    at += n;
    phase ^= at / N & 1;
    at %= N;
  }
  __device__ __forceinline__ void back() {
    if (at-- == 0) at = N - 1, phase ^= 1;
  }
};

// ---- a word from global to shared memory without a register, and the arrival of
// the calling thread's words so far
__device__ __forceinline__ void copy_word(uint32_t dst, const float *src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

__device__ __forceinline__ void arrive_with_words(uint64_t *bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}

__device__ __forceinline__ void words_landed() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// ---- two fp32 lanes in one instruction
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}

__device__ __forceinline__ uint64_t pack2(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}

__device__ __forceinline__ float2 unpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}

__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

}  // namespace apc
