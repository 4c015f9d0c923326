// The product of two block-scaled 8-bit matrices (apc_matmul_fp8) on the
// 5th-generation tensor cores.
//
//   out[i, j] = sum over blocks c of 128 k:
//                 (sum over k in c of a[i, k] b[j, k]) sb[c, j] sa[c, i]
//
// The inner sum is four tcgen05.mma (K = 32 each) into tensor memory, in fp32.
// Its accumulator is then read back, multiplied by the scales and added into
// fp32 registers while the tensor core fills other accumulators: the scales are
// arbitrary fp32 numbers, and no sum of more than 128 products is left to the
// tensor core's own rounding.  Large products to 16 bits whose scales are powers of two,
// as quantization makes them, leave scaling and sums to the tensor cores (may_go_by_exponents).
//
// Two kernels, warp-specialized alike: one warp issues TMA loads into a ring of
// shared-memory stages (128 bytes of k a row, 128-byte swizzle, zeros beyond
// the edges), one copies the blocks' scales into a ring of their own, one thread
// issues the products, the others add up.  (With the scales loaded by the adding
// warps a block ahead, each block took a trip to memory: 1,600 cycles for
// few columns, 900 for large products.)
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

#include "apc_ops.cuh"
#include "apc_tcgen05.cuh"

namespace apc {

namespace {

// What both kernels take.  "r" is the operand on the accumulator's lanes, "c"
// the one on its columns.
struct ProductPlan {
  const float *r_scale, *c_scale;
  int64_t r_scale_pitch, c_scale_pitch;
  uint32_t r_shift, c_shift;
  uint32_t rows, cols;      // of the product's lanes and columns
  uint32_t row_tiles, col_tiles;
  uint32_t blocks;          // of 128 k
  uint32_t instruction;
  uint32_t formats;         // of the operands, in the instruction's bits
  bool by_exponent;         // large products: scales that are powers of two may be the tensor cores'
  void *out;
  int64_t row_step, col_step;  // elements of out
  unsigned *status;
};

// A whole warp's wait: its lanes give up together.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity) {
  return __all_sync(~0u, mbar_try_wait(smem_addr(bar), parity)) || __all_sync(~0u, wait_for(bar, parity));
}

__device__ __forceinline__ void give_up(unsigned *status) { atomicOr(status, (unsigned)APC_ETIMEOUT); }

constexpr int kScaleSlots = 8;  // blocks whose scales are on their way or in use

// ---------------------------------------------------------------------------
// The kernel for few columns: 128 rows of the wide operand (a weight's outputs)
// on the lanes, BN columns (tokens) beside them.
//
// The k blocks of a tile are split evenly over a cluster's CTAs, so that few
// tiles still keep all SMs loading: each CTA sums its share in registers, leaves it
// in shared memory and sends every CTA the columns that it owns (one bulk copy
// each, counted by an mbarrier); the owner adds the shares in the order of their
// ranks and stores.  The loads of the next tile run meanwhile.
//
// Bound by memory while it streams, and by launch, first loads and exchange, some 7 us.
// Measured: 1 x 14336 x 4096 14.0 us (4.2 TB/s), 37 x 4096 x 14336 17.2 us (3.5 TB/s),
// 777 x 1001 x 2500 to fp32 10.6 us.
//
// A wait that gives up marks the CTA dead: it stops loading and issuing, waits for
// what is in flight, and its sums go on without waiting, so that every barrier is
// reached.
constexpr int kMidThreads = 352;  // warps: copies, products, scales; 8 that add

template <int BN, bool SPLIT>
struct MidShape {
  static constexpr int kRowBytes = 128 * kBlock, kColBytes = BN * kBlock;
  static constexpr int kStageBytes = kRowBytes + kColBytes;
  static constexpr int kShareBytes = SPLIT ? BN * 128 * 4 : 0;
  static constexpr int kScaleBytes = kScaleSlots * (128 + BN) * 4;
  static constexpr int kRoom = 224 * 1024 - 2 * kShareBytes - kScaleBytes;
  static constexpr int kStages = kRoom / kStageBytes > 12 ? 12 : kRoom / kStageBytes;
  static constexpr int kBytes = 1024 + kStages * kStageBytes + 2 * kShareBytes + kScaleBytes;
  // accumulators: a block's way from its products through the sums and back takes
  // many times as long as either
  static constexpr int kAcc = 512 / BN < 8 ? 512 / BN : 8;
  static constexpr int kTmem = kAcc * BN;
  static constexpr int kCols = BN / 2, kLoad = kCols < 32 ? kCols : 32;  // a warp adds half the columns
};

template <int BN, bool SPLIT, typename T>
__global__ void __launch_bounds__(kMidThreads, 1)
    mid_kernel(const __grid_constant__ CUtensorMap map_r, const __grid_constant__ CUtensorMap map_c,
               const __grid_constant__ ProductPlan p, const uint32_t split_log2) {
  using S = MidShape<BN, SPLIT>;
  constexpr int kLog2Bn = BN == 16 ? 4 : BN == 32 ? 5 : BN == 64 ? 6 : 7;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[S::kStages], empty[S::kStages], acc_full[S::kAcc], acc_empty[S::kAcc], recv_full, recv_free;
  __shared__ uint64_t scale_full[kScaleSlots], scale_empty[kScaleSlots];
  __shared__ uint32_t tmem_at;
  __shared__ volatile int32_t dead;
  uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  float *share = reinterpret_cast<float *>(smem + S::kStages * S::kStageBytes);  // [column][row]
  float *recv = share + S::kShareBytes / 4;                                       // [rank][own column][row]
  float *scales = recv + S::kShareBytes / 4;                                     // [slot][128 rows, BN columns]
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t split = SPLIT ? 1u << split_log2 : 1, rank = SPLIT ? cluster_rank() : 0;
  const uint32_t first = blockIdx.x / split, step = gridDim.x / split;
  const uint32_t tiles = p.row_tiles * p.col_tiles;
  const uint32_t b0 = (uint32_t)((uint64_t)p.blocks * rank / split), b1 = (uint32_t)((uint64_t)p.blocks * (rank + 1) / split);

  if (threadIdx.x == 32) prefetch_map(&map_r), prefetch_map(&map_c);
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kStages; ++i) mbar_init(&full[i], 1), mbar_init(&empty[i], 1);
    for (int i = 0; i < S::kAcc; ++i) mbar_init(&acc_full[i], 1), mbar_init(&acc_empty[i], 8);
    for (int i = 0; i < kScaleSlots; ++i) mbar_init(&scale_full[i], 32), mbar_init(&scale_empty[i], 8);
    mbar_init(&recv_full, 1);
    mbar_init(&recv_free, 8 * split);
    dead = 0;
    mbar_init_fence();
  }
  if (warp == 1) tmem_alloc<1>(&tmem_at, S::kTmem);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (SPLIT) cluster_arrive(), cluster_wait();  // the barriers are there before anyone sends
  const uint32_t tmem = tmem_at;
  // A whole warp's wait.
  auto alive = [&](uint64_t *bar, uint32_t parity) {
    if (__all_sync(~0u, mbar_try_wait(smem_addr(bar), parity))) return true;
    const bool ok = __all_sync(~0u, wait_for(bar, parity, &dead));
    if (!ok && !dead) {
      dead = 1;
      give_up(p.status);
    }
    return ok;
  };

  if (warp == 0) {
    Turn<S::kStages> st;
    uint32_t issued = 0;
    bool ok = true;
    for (uint32_t t = first; t < tiles && ok; t += step) {
      const int32_t r0 = (int32_t)(t % p.row_tiles) * 128, c0 = (int32_t)(t / p.row_tiles) * BN;
      for (uint32_t b = b0; b < b1; ++b, st.next(), ++issued) {
        if (!(ok = alive(&empty[st.at], st.phase ^ 1))) break;
        const uint32_t at = smem_addr(smem) + st.at * S::kStageBytes;
        load_block(at, &map_r, r0, at + S::kRowBytes, &map_c, c0, (int32_t)(b * kBlock), smem_addr(&full[st.at]), S::kStageBytes);
      }
    }
    if (!ok)  // let the copies in flight land
      for (uint32_t i = min(issued, (uint32_t)S::kStages); i; --i) st.back(), wait_for(&full[st.at], st.phase);
  } else if (warp == 1) {
    Turn<S::kStages> st;
    Turn<S::kAcc> acc;
    uint32_t issued = 0;
    bool ok = true;
    const uint64_t r_desc = operand_desc(smem_addr(smem)), c_desc = operand_desc(smem_addr(smem) + S::kRowBytes);
    for (uint32_t t = first; t < tiles && ok; t += step)
      for (uint32_t b = b0; b < b1; ++b, st.next(), acc.next(), ++issued) {
        if (!(ok = alive(&acc_empty[acc.at], acc.phase ^ 1) && alive(&full[st.at], st.phase))) break;
        tc_fence_after();
        const uint64_t off = st.at * (S::kStageBytes >> 4);
        mma_block<1>(tmem + acc.at * BN, r_desc + off, c_desc + off, p.instruction, smem_addr(&acc_full[acc.at]), smem_addr(&empty[st.at]));
      }
    if (!ok)  // let the products in flight end
      for (uint32_t i = min(issued, (uint32_t)S::kAcc); i; --i) acc.back(), wait_for(&acc_full[acc.at], acc.phase);
  } else if (warp == 2) {
    Turn<kScaleSlots> slot;
    for (uint32_t t = first; t < tiles && !dead; t += step) {
      const uint32_t r0 = t % p.row_tiles * 128 + lane, c0 = t / p.row_tiles * BN + lane;
      for (uint32_t b = b0; b < b1; ++b, slot.next()) {
        const uint32_t at = smem_addr(scales + slot.at * (128 + BN) + lane);
        if (!alive(&scale_empty[slot.at], slot.phase ^ 1)) break;
        const float *rs = p.r_scale + b * p.r_scale_pitch, *cs = p.c_scale + b * p.c_scale_pitch;
#pragma unroll
        for (int i = 0; i < 128; i += 32) copy_word(at + i * 4, rs + (min(r0 + i, p.rows - 1) >> p.r_shift));
#pragma unroll
        for (int i = 0; i < BN; i += 32)
          if (BN >= 32 || lane < BN) copy_word(at + (128 + i) * 4, cs + (min(c0 + i, p.cols - 1) >> p.c_shift));
        arrive_with_words(&scale_full[slot.at]);
      }
    }
    words_landed();
  } else {
    constexpr int kCols = S::kCols, kLoad = S::kLoad;
    const uint32_t quad = warp & 3, row = quad * 32 + lane, half = (warp - 3) / 4;
    Turn<S::kAcc> buf;
    Turn<kScaleSlots> slot;
    uint32_t done = 0;
    if (SPLIT && threadIdx.x == 96) mbar_arrive_expect_tx(&recv_full, S::kShareBytes);
    for (uint32_t t = first; t < tiles; t += step, ++done) {
      const uint32_t r0 = t % p.row_tiles * 128, c0 = t / p.row_tiles * BN;
      uint64_t acc[kCols / 2];
#pragma unroll
      for (int i = 0; i < kCols / 2; ++i) acc[i] = 0;
      for (uint32_t b = b0; b < b1; ++b, buf.next(), slot.next()) {
        alive(&scale_full[slot.at], slot.phase);
        const float *line = scales + slot.at * (128 + BN), *s = line + 128 + half * kCols;
        const uint64_t sr = pack2(line[row], line[row]);
        alive(&acc_full[buf.at], buf.phase);
        tc_fence_after();
        const uint32_t at = tmem + buf.at * BN + half * kCols + (quad << 21);  // lane 32 * quad in bits 16 up
#pragma unroll
        for (int c = 0; c < kCols; c += kLoad) {
          uint32_t d[kLoad];
          tmem_load(d, at + c);
          tmem_landed(d);
          if (c + kLoad == kCols) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_empty[buf.at]);
          }
#pragma unroll
          for (int i = 0; i < kLoad; i += 4) {
            const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(s + c + i);
            acc[(c + i) / 2] = fma2(mul2(pack2(d[i], d[i + 1]), sr), v.x, acc[(c + i) / 2]);
            acc[(c + i) / 2 + 1] = fma2(mul2(pack2(d[i + 2], d[i + 3]), sr), v.y, acc[(c + i) / 2 + 1]);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&scale_empty[slot.at]);
      }
      T *out = static_cast<T *>(p.out) + (int64_t)(r0 + row) * p.row_step;
      const bool in = r0 + row < p.rows;
      if (!SPLIT) {
        const uint32_t c1 = c0 + half * kCols;
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          const float2 v = unpack2(acc[i / 2]);
          if (in && c1 + i < p.cols) out[(int64_t)(c1 + i) * p.col_step] = from_float<T>(i % 2 ? v.y : v.x);
        }
        continue;
      }
      // a share to each CTA of the cluster, once all have read the tile before
      if (done) alive(&recv_free, (done + 1) & 1);
#pragma unroll
      for (int i = 0; i < kCols; ++i) {
        const float2 v = unpack2(acc[i / 2]);
        share[(half * kCols + i) * 128 + row] = i % 2 ? v.y : v.x;
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      asm volatile("bar.sync 1, 256;" ::: "memory");
      const uint32_t per = 1u << (kLog2Bn - split_log2);  // columns that a CTA owns
      if (threadIdx.x - 96 < split) {
        const uint32_t owner = threadIdx.x - 96;
        bulk_s2s(map_rank(smem_addr(recv + rank * per * 128), owner), smem_addr(share + owner * per * 128), per * 512,
                 map_rank(smem_addr(&recv_full), owner));
      }
      alive(&recv_full, done & 1);
      if (threadIdx.x == 96) mbar_arrive_expect_tx(&recv_full, S::kShareBytes);
      for (uint32_t c = half * (per / 2); c < (half + 1) * (per / 2); ++c) {
        float sum = recv[c * 128 + row];
        for (uint32_t k = 1; k < split; ++k) sum += recv[(k * per + c) * 128 + row];
        const uint32_t col = c0 + rank * per + c;
        if (in && col < p.cols) out[(int64_t)col * p.col_step] = from_float<T>(sum);
      }
      __syncwarp();
      if (lane < split) arrive_remote(map_rank(smem_addr(&recv_free), lane));
    }
    if (SPLIT && dead && done) wait_for(&recv_full, (done - 1) & 1);  // let the shares in flight land
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (SPLIT) cluster_arrive(), cluster_wait();  // nobody sends to a CTA that has left
  tc_fence_after();
  if (warp == 1) tmem_free<1>(tmem, S::kTmem);
}

// ---------------------------------------------------------------------------
// The kernel for large products: a pair of CTAs computes 256 x 256 of out, each
// CTA 128 rows of a on its lanes and all 256 rows of b on its columns, of which
// it holds half in shared memory (tcgen05.mma.cta_group::2 reads both halves).
// The first CTA's thread issues for both.  Persistent: the pair's next tile is
// loaded while the epilogue stores.
//
// A tile goes one of two ways.
//  * By exponents, where every scale in its rows' and columns' blocks is a power of two:
//    mxf8f6f4 products multiply by the scales' exponents and add up in the accumulator
//    over all of k.  One warp packs the exponents of four blocks at a time, tcgen05.cp
//    takes them to the columns of the accumulator that is not in use.
//  * In general, block by block: two accumulators, read back, scaled and added in
//    registers.  Bound by an accumulator's way: products (512 cycles), commit, drain and
//    the pair's arrival take 2,000, of which two overlap; with a scale for every column
//    by the fp32 pipe too.
// While a tile's products run, its next one's scales are looked at and both CTAs told:
// in a tile by exponents by the adding warps, which wait then, in a general one by the
// exponents' warp, which has nothing else to do there.
// A tile's way is its own scales' alone, whatever its pair did before, so results do
// not depend on which tiles a pair gets.
// Measured: 4096 x 32768 x 4096 by exponents 322 us (3.4 PFLOP/s; the tensor cores busy for
// 75% of the cycles, at 8192 columns), in general 567; 14336 x 4096 x 8192 with a
// scale for every column 290 us (3.3 PFLOP/s), 724; 4096 x 8192 x 4096 to fp32 167.  Back to
// back for seconds the GPU's power limit takes the clock to 1.5 GHz: 380 and 339 us.
// Warps 0 to 3 load and issue with 56 registers a thread, 4 to 11 add with 224 (of
// the launch's 168 each: 128 x 56 + 256 x 224 = 384 x 168).
constexpr int kBigWarps = 8, kBigThreads = 128 + 32 * kBigWarps, kBigStages = 6;
constexpr int kBigCols = 1024 / kBigWarps;  // columns that a warp adds
constexpr int kBigHalf = 128 * kBlock, kBigStageBytes = 2 * kBigHalf;
constexpr int kBigScaleBytes = kScaleSlots * (128 + 256) * 4;
constexpr int kBigTurnBytes = 32 * 68;  // a warp's, for its way to out
constexpr int kExpSlots = 2, kExpBytes = 3 * 512;  // exponents of four blocks: 128 rows, 256 columns
constexpr int kBigBytes = 1024 + kBigStages * kBigStageBytes + kBigScaleBytes + kBigWarps * kBigTurnBytes + kExpSlots * kExpBytes;
constexpr uint32_t kBigGroup = 16;  // row tiles that are walked together
// Tiles whose way is told and not yet read by all: of one block each, the exponents' warp can
// be as many ahead as there are slots of scales, and the pair's other one a tile beside that.
constexpr uint32_t kModes = 16;

// Tile t of the walk: groups of row tiles, in each the row tile first, so that
// the tiles in flight share few rows of both operands in L2.
__device__ __forceinline__ void big_tile(const ProductPlan &p, uint32_t t, uint32_t *r, uint32_t *c) {
  const uint32_t group = t / (kBigGroup * p.col_tiles), first = group * kBigGroup;
  const uint32_t height = min(kBigGroup, p.row_tiles - first), i = t - first * p.col_tiles;
  *r = first + i % height;
  *c = i / height;
}

// A warp's 32 rows of kBigCols sums, a row a lane, to out (lane 0's row), of which
// `count` columns and the rows of `rows` exist.  They go through shared memory, 64
// bytes of each row at a time, so that a store instruction writes neighbours in a
// row: 8 rows' 64 bytes where rows start on 16-byte boundaries, one row's otherwise.
// (Stored by their own lanes, 16 bytes in each of 32 rows, a tile took 9 us.)
template <bool ALIGNED, typename T>
__device__ __forceinline__ void store_rows(T *out, const uint64_t (&acc)[kBigCols / 2], uint32_t count, uint32_t rows, int64_t step,
                                           float *turn, uint32_t lane) {
  constexpr int kPer = 16 / sizeof(T), kTurnCols = 64 / sizeof(T);
  constexpr int kTurnPitch = (ALIGNED ? 64 : 68) / sizeof(T);  // aligned: 16-byte pieces, swizzled over the banks
  T *mine = reinterpret_cast<T *>(turn);
#pragma unroll
  for (int c = 0; c < kBigCols; c += kTurnCols) {
    if constexpr (ALIGNED) {
#pragma unroll
      for (int i = 0; i < kTurnCols; i += kPer) {
        union {
          T v[kPer];
          uint4 q;
        } u;
#pragma unroll
        for (int j = 0; j < kPer; j += 2) {
          const float2 v = unpack2(acc[(c + i + j) / 2]);
          u.v[j] = from_float<T>(v.x);
          u.v[j + 1] = from_float<T>(v.y);
        }
        *reinterpret_cast<uint4 *>(mine + lane * kTurnPitch + (i / kPer ^ (lane >> 1 & 3)) * kPer) = u.q;
      }
      __syncwarp();
      const uint32_t col = lane % 4 * kPer;
#pragma unroll
      for (uint32_t r = lane / 4; r < 32; r += 8) {
        const T *from = mine + r * kTurnPitch + (lane % 4 ^ (r >> 1 & 3)) * kPer;
        T *to = out + (int64_t)r * step + c + col;
        if (!(rows >> r & 1)) continue;
        if (c + col + kPer <= count) {
          *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from);
        } else {
          for (int j = 0; j < kPer; ++j)
            if (c + col + j < count) to[j] = from[j];
        }
      }
    } else {
      constexpr int kRows = 32 / kTurnCols;  // rows a store writes
#pragma unroll
      for (int i = 0; i < kTurnCols; i += 2) {
        const float2 v = unpack2(acc[(c + i) / 2]);
        mine[lane * kTurnPitch + i] = from_float<T>(v.x);
        mine[lane * kTurnPitch + i + 1] = from_float<T>(v.y);
      }
      __syncwarp();
      const uint32_t col = lane % kTurnCols;
#pragma unroll 8
      for (uint32_t r = lane / kTurnCols; r < 32; r += kRows)
        if ((rows >> r & 1) && c + col < count) out[(int64_t)r * step + c + col] = mine[r * kTurnPitch + col];
    }
    __syncwarp();
  }
}

// ROWS: the scales of b change from column to column.  ALIGNED: every row of out
// starts on a 16-byte boundary.
template <typename T, bool ROWS, bool ALIGNED>
__global__ void __launch_bounds__(kBigThreads, 1)
    big_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ ProductPlan p) {
  constexpr int kLoad = ROWS ? 32 : 16;  // columns in a load from the accumulator
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kBigStages], empty[kBigStages], acc_full[2], acc_empty[2];
  __shared__ uint64_t scale_full[kScaleSlots], scale_empty[kScaleSlots];
  __shared__ uint64_t exp_full[kExpSlots], exp_empty[kExpSlots], mode_full[kModes];
  __shared__ volatile uint32_t general[kModes];  // n where the pair's nth tile's scales are not all powers of two, at n mod kModes
  __shared__ uint32_t tmem_at;
  uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  float *scales = reinterpret_cast<float *>(smem + kBigStages * kBigStageBytes);  // [slot][128 rows, 256 columns]
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, rank = cluster_rank();
  const uint32_t first = blockIdx.x / 2, step = gridDim.x / 2, tiles = p.row_tiles * p.col_tiles;

  if (threadIdx.x == 32) prefetch_map(&map_a), prefetch_map(&map_b);
  if (threadIdx.x == 0) {
    for (int i = 0; i < kBigStages; ++i) mbar_init(&full[i], 1), mbar_init(&empty[i], 1);
    for (int i = 0; i < 2; ++i) mbar_init(&acc_full[i], 1), mbar_init(&acc_empty[i], 2 * kBigWarps);
    for (int i = 0; i < kScaleSlots; ++i) mbar_init(&scale_full[i], 32), mbar_init(&scale_empty[i], kBigWarps + p.by_exponent);
    for (int i = 0; i < kExpSlots; ++i) mbar_init(&exp_full[i], 2), mbar_init(&exp_empty[i], 1);
    for (uint32_t i = 0; i < kModes; ++i) mbar_init(&mode_full[i], 2 * kBigWarps);
    for (uint32_t i = 0; i < kModes; ++i) general[i] = ~0u;
    mbar_init_fence();
  }
  if (warp == 1) tmem_alloc<2>(&tmem_at, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  cluster_arrive(), cluster_wait();
  const uint32_t tmem = tmem_at;
  uint8_t *exps = reinterpret_cast<uint8_t *>(scales) + kBigScaleBytes + kBigWarps * kBigTurnBytes;
  // Whether the pair's nth tile goes by exponents; `ok` false if the wait gave up.
  auto by_exponent = [&](uint32_t n, bool &ok) {
    if (!p.by_exponent) return false;
    ok = warp_wait(&mode_full[n % kModes], n / kModes & 1);
    return general[n % kModes] != n;
  };
  // kBigWarps threads of each CTA tell both CTAs whether the pair's nth tile goes by
  // exponents.  No release where there is nothing to see: it would wait for the last tile's
  // stores.
  auto tell = [&](uint32_t n, bool good) {
    const uint32_t at = (uint32_t)__cvta_generic_to_shared((const void *)general) + n % kModes * 4, bar = smem_addr(mode_full) + n % kModes * 8;
    if (!good) {
      general[n % kModes] = n;
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_rank(at, rank ^ 1)), "r"(n) : "memory");
      asm volatile("fence.acq_rel.cluster;" ::: "memory");
    }
    arrive_remote_relaxed(map_rank(bar, 0));
    arrive_remote_relaxed(map_rank(bar, 1));
  };
  // 0 for a float 2^-126 to 2^63: the tensor cores' product of two larger ones may be an
  // infinity, and an infinity times 0 is no 0.  (Small ones they multiply exactly, below
  // 2^-126 too.)  Without a branch: the loads before stay together.
  auto no_exponent = [](uint32_t bits) { return bits & 0x807fffffu | (uint32_t)(bits - 1u >= (63 + 127 << 23)); };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0) {
      Turn<kBigStages> st;
      uint32_t issued = 0;
      bool ok = true;
      const uint32_t bars = map_rank(smem_addr(full), 0);
      for (uint32_t t = first; t < tiles && ok; t += step) {
        uint32_t tr, tc;
        big_tile(p, t, &tr, &tc);
        const int32_t r0 = (int32_t)(tr * 256 + rank * 128), c0 = (int32_t)(tc * 256 + rank * 128);
        for (uint32_t b = 0; b < p.blocks; ++b, st.next(), ++issued) {
          if (!(ok = warp_wait(&empty[st.at], st.phase ^ 1))) break;
          const uint32_t at = smem_addr(smem) + st.at * kBigStageBytes;
          load_block_pair(at, &map_a, r0, at + kBigHalf, &map_b, c0, (int32_t)(b * kBlock), bars + st.at * 8, smem_addr(&full[st.at]),
                          rank == 0 ? 2 * kBigStageBytes : 0);
        }
      }
      if (!ok) {  // let the copies in flight land, the other CTA's too
        give_up(p.status);
        if (rank == 0)
          for (uint32_t i = min(issued, (uint32_t)kBigStages); i; --i) st.back(), wait_for(&full[st.at], st.phase);
        const uint64_t t0 = global_ns();
        for (uint32_t i = 0; i < kWaitIterations && global_ns() - t0 < 1000000; ++i) __nanosleep(1000);
      }
    }
    if (warp == 2) {
      Turn<kScaleSlots> slot;
      bool ok = true;
      for (uint32_t t = first; t < tiles && ok; t += step) {
        uint32_t tr, tc;
        big_tile(p, t, &tr, &tc);
        const uint32_t r0 = tr * 256 + rank * 128 + lane, c0 = tc * 256 + lane;
        for (uint32_t b = 0; b < p.blocks; ++b, slot.next()) {
          const uint32_t at = smem_addr(scales + slot.at * 384 + lane);
          if (!(ok = warp_wait(&scale_empty[slot.at], slot.phase ^ 1))) break;
          const float *rs = p.r_scale + b * p.r_scale_pitch, *cs = p.c_scale + b * p.c_scale_pitch;
#pragma unroll
          for (int i = 0; i < 128; i += 32) copy_word(at + i * 4, rs + (min(r0 + i, p.rows - 1) >> p.r_shift));
          if (ROWS) {
#pragma unroll
            for (int i = 0; i < 256; i += 32) copy_word(at + (128 + i) * 4, cs + min(c0 + i, p.cols - 1));
          } else if (lane < 2) {  // one for each 128 columns
            copy_word(at + 128 * 4, cs + (min(tc * 256 + lane * 128, p.cols - 1) >> 7));
          }
          arrive_with_words(&scale_full[slot.at]);
        }
      }
      words_landed();
      if (!ok) give_up(p.status);
    }
    if (warp == 3) {
      // exponents of four blocks at a time, in tiles that go by them; in the others every
      // block's slot is passed on, and a block of the next tile's scales is looked at
      Turn<kScaleSlots> slot;
      Turn<kExpSlots> exp;
      bool ok = true;
      uint32_t n = 0;
      const uint32_t bars = map_rank(smem_addr(exp_full), 0);
      for (uint32_t t = first; t < tiles && ok && p.by_exponent; t += step, ++n) {
        if (!by_exponent(n, ok)) {
          const bool more = t + step < tiles;
          uint32_t tr, tc, seen = more ? 0 : p.blocks;  // blocks of the next tile
          if (more) big_tile(p, t + step, &tr, &tc);
          const uint32_t r0 = tr * 256 + rank * 128 + lane, c0 = tc * 256 + rank * 128 + lane;
          for (uint32_t b = 0; b < p.blocks && ok; ++b, slot.next()) {
            if (seen < p.blocks) {
              const float *rs = p.r_scale + seen * p.r_scale_pitch, *cs = p.c_scale + seen * p.c_scale_pitch;
              uint32_t v[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const uint32_t o = i % 4 * 32;
                v[i] = __float_as_uint(__ldg(i < 4 ? rs + (min(r0 + o, p.rows - 1) >> p.r_shift) : cs + (min(c0 + o, p.cols - 1) >> p.c_shift)));
              }
              uint32_t bad = 0;
#pragma unroll
              for (int i = 0; i < 8; ++i) bad |= no_exponent(v[i]);
              const bool good = __all_sync(~0u, bad == 0);
              seen = good ? seen + 1 : ~0u;
              if (seen >= p.blocks && lane < kBigWarps) tell(n + 1, good);
            }
            if (!(ok = warp_wait(&scale_full[slot.at], slot.phase))) break;
            if (lane == 0) mbar_arrive(&scale_empty[slot.at]);
          }
          continue;
        }
        for (uint32_t b = 0; b < p.blocks && ok; b += 4, exp.next()) {
          if (!(ok = warp_wait(&exp_empty[exp.at], exp.phase ^ 1))) break;
          uint32_t w[12];
#pragma unroll
          for (int j = 0; j < 12; ++j) w[j] = 0;
          for (uint32_t i = 0; i < min(4u, p.blocks - b); ++i, slot.next()) {
            if (!(ok = warp_wait(&scale_full[slot.at], slot.phase))) break;
            const float *line = scales + slot.at * 384;
#pragma unroll
            for (int j = 0; j < 12; ++j) {
              const float s = j < 4 || ROWS ? line[32 * j + lane] : line[128 + (j - 4) / 4];
              w[j] |= (__float_as_uint(s) >> 23 & 0xff) << 8 * i;
            }
            __syncwarp();
            if (lane < kBigWarps + 1) mbar_arrive(&scale_empty[slot.at]);  // for the adding warps too
          }
          uint4 *to = reinterpret_cast<uint4 *>(exps + exp.at * kExpBytes) + lane;
#pragma unroll
          for (int j = 0; j < 3; ++j) to[32 * j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) arrive_remote(bars + exp.at * 8);
        }
      }
      if (!ok) give_up(p.status);
    }
    if (warp == 1 && rank == 0) {
      Turn<kBigStages> st;
      Turn<2> acc;
      uint32_t issued = 0;
      bool ok = true;
      const uint64_t da = operand_desc(smem_addr(smem)), db = operand_desc(smem_addr(smem) + kBigHalf);
      Turn<kExpSlots> exp;
      uint32_t n = 0;
      for (uint32_t t = first; t < tiles && ok; t += step, ++n) {
        const bool exponents = by_exponent(n, ok);
        if (!ok) break;
        if (exponents) {
          // one accumulator, the exponents in the other's columns
          Turn<2> other = acc;
          other.next();
          if (!(ok = warp_wait(&acc_empty[acc.at], acc.phase ^ 1) && warp_wait(&acc_empty[other.at], other.phase ^ 1))) break;
          const uint32_t columns = tmem + (acc.at ^ 1) * 256;
          for (uint32_t b = 0; b < p.blocks && ok; b += 4, exp.next()) {
            if (!(ok = warp_wait(&exp_full[exp.at], exp.phase))) break;
            tc_fence_after();
            copy_scales_pair(columns, smem_addr(exps + exp.at * kExpBytes));
            for (uint32_t i = 0; i < min(4u, p.blocks - b); ++i, st.next()) {
              if (!(ok = warp_wait(&full[st.at], st.phase))) break;
              tc_fence_after();
              const uint64_t off = st.at * (kBigStageBytes >> 4);
              mma_scaled_pair(tmem + acc.at * 256, da + off, db + off, scaled_instruction(p.formats, 256, 256, i), columns, b + i == 0,
                              smem_addr(&empty[st.at]));
            }
            commit_pair(smem_addr(&exp_empty[exp.at]));
          }
          commit_pair(smem_addr(&acc_full[acc.at]));
          acc.next(), ++issued;
          continue;
        }
        for (uint32_t b = 0; b < p.blocks && ok; ++b, st.next(), acc.next(), ++issued) {
          if (!(ok = warp_wait(&full[st.at], st.phase) && warp_wait(&acc_empty[acc.at], acc.phase ^ 1))) break;
          tc_fence_after();
          const uint64_t off = st.at * (kBigStageBytes >> 4);
          mma_block<2>(tmem + acc.at * 256, da + off, db + off, p.instruction, smem_addr(&acc_full[acc.at]), smem_addr(&empty[st.at]));
        }
      }
      if (!ok) {  // let the products in flight end
        give_up(p.status);
        for (uint32_t i = min(issued, 2u); i; --i) acc.back(), wait_for(&acc_full[acc.at], acc.phase);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    const uint32_t quad = warp & 3, part = (warp - 4) / 4, row = quad * 32 + lane;
    const uint32_t empty_bars = map_rank(smem_addr(acc_empty), 0);
    float *turn = scales + kBigScaleBytes / 4 + (warp - 4) * (kBigTurnBytes / 4);
    Turn<2> buf;
    Turn<kScaleSlots> slot;
    bool ok = true;
    // Looks at the scales of the pair's nth tile, t, and tells: this CTA at its 128 rows' and
    // at those of its half of the columns, a thread at one.
    auto look = [&](uint32_t t, uint32_t n) {
      uint32_t tr, tc;
      big_tile(p, t, &tr, &tc);
      const uint32_t k = threadIdx.x - 128;  // 128 rows, 128 columns
      const bool col = k >= 128;
      const uint32_t at = col ? min(tc * 256 + rank * 128 + k - 128, p.cols - 1) >> p.c_shift : min(tr * 256 + rank * 128 + k, p.rows - 1) >> p.r_shift;
      const float *s = (col ? p.c_scale : p.r_scale) + at;
      const int64_t pitch = col ? p.c_scale_pitch : p.r_scale_pitch;
      uint32_t bad = 0;
      for (uint32_t b = 0; b < p.blocks; b += 16) {
        uint32_t v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__ldg(s + min(b + i, p.blocks - 1) * pitch));
#pragma unroll
        for (int i = 0; i < 16; ++i) bad |= no_exponent(v[i]);
      }
      const bool good = __all_sync(~0u, bad == 0);
      if (lane == 0) tell(n, good);
    };
    uint32_t n = 0;
    if (p.by_exponent && first < tiles) look(first, 0);
    for (uint32_t t = first; t < tiles && ok; t += step, ++n) {
      uint32_t tr, tc;
      big_tile(p, t, &tr, &tc);
      const uint32_t r0 = tr * 256 + rank * 128, c0 = tc * 256 + part * kBigCols;
      uint64_t acc[kBigCols / 2];
#pragma unroll
      for (int i = 0; i < kBigCols / 2; ++i) acc[i] = 0;
      // adds some columns of a sum of 128 products, scaled; c: the first, within the warp's.  The
      // sums are multiplied by b's scale and then by a's: their product may leave fp32's range
      // where a sum is 0 or the result small.  (With the product first, which without scales of the
      // columns is one for all of them: 523 us for 4096 x 32768 x 4096 in place of 568.)
      auto add = [&](const uint32_t (&d)[kLoad], int c, uint64_t sr, uint64_t sc, const float *s) {
#pragma unroll
        for (int i = 0; i < kLoad; i += 4) {
          uint64_t x = sc, y = sc;
          if (ROWS) {
            const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(s + c + i);
            x = v.x, y = v.y;
          }
          acc[(c + i) / 2] = fma2(mul2(pack2(d[i], d[i + 1]), x), sr, acc[(c + i) / 2]);
          acc[(c + i) / 2 + 1] = fma2(mul2(pack2(d[i + 2], d[i + 3]), y), sr, acc[(c + i) / 2 + 1]);
        }
      };
      const bool exponents = by_exponent(n, ok);
      if (!ok) break;
      if (exponents) {
        if (t + step < tiles) look(t + step, n + 1);
        if (!(ok = warp_wait(&acc_full[buf.at], buf.phase))) break;
        tc_fence_after();
        const uint32_t at = tmem + buf.at * 256 + part * kBigCols + (quad << 21);
#pragma unroll
        for (int c = 0; c < kBigCols; c += 32) {
          uint32_t d[32];
          tmem_load(d, at + c);
          tmem_landed(d);
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[c / 2 + i] = pack2(d[2 * i], d[2 * i + 1]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_remote_relaxed(empty_bars + buf.at * 8);
        buf.next();
        slot.skip(p.blocks);  // the exponents' warp took them
      } else {
        for (uint32_t b = 0; b < p.blocks; ++b, buf.next(), slot.next()) {
          const float *s = scales + slot.at * 384 + 128 + (ROWS ? part * kBigCols : part * kBigCols / 128);
          if (!(ok = warp_wait(&scale_full[slot.at], slot.phase))) break;
          const float mine = scales[slot.at * 384 + row];
          const uint64_t sr = pack2(mine, mine), sc = ROWS ? 0 : pack2(s[0], s[0]);
          if (!(ok = warp_wait(&acc_full[buf.at], buf.phase))) break;
          tc_fence_after();
          const uint32_t at = tmem + buf.at * 256 + part * kBigCols + (quad << 21);
          // each load runs under the additions of the one before
          uint32_t d[2][kLoad];
          tmem_load(d[0], at);
#pragma unroll
          for (int c = 0; c < kBigCols; c += kLoad) {
            const int i = c / kLoad % 2;
            tmem_landed(d[i]);
            if (c + kLoad < kBigCols) {
              tmem_load(d[i ^ 1], at + c + kLoad);
            } else {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) arrive_remote_relaxed(empty_bars + buf.at * 8);
            }
            add(d[i], c, sr, sc, s);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&scale_empty[slot.at]);
        }
      }
      if (!ok) break;
      if (c0 < p.cols)
        store_rows<ALIGNED>(static_cast<T *>(p.out) + (int64_t)(r0 + quad * 32) * p.row_step + c0, acc,
                            min((uint32_t)kBigCols, p.cols - c0), __ballot_sync(~0u, r0 + row < p.rows), p.row_step, turn, lane);
    }
    if (!ok) give_up(p.status);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_arrive(), cluster_wait();
  tc_fence_after();
  if (warp == 1) tmem_free<2>(tmem, 512);
}

// ---------------------------------------------------------------------------

int encode(CUtensorMap *map, const uint8_t *data, uint32_t rows, uint32_t cols, int64_t pitch, uint32_t box_rows) {
  static const PFN_cuTensorMapEncodeTiled_v12000 tiled = [] {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult st = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &st) != cudaSuccess) cudaGetLastError();
    return st == cudaDriverEntryPointSuccess ? (PFN_cuTensorMapEncodeTiled_v12000)fn : nullptr;
  }();
  if (!tiled) return (int)cudaErrorNotSupported;
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {rows > 1 ? (cuuint64_t)pitch : ((cuuint64_t)cols + 15) / 16 * 16};
  const cuuint32_t box[2] = {kBlock, box_rows}, steps[2] = {1, 1};
  const CUresult r = tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(data), dims, strides, box, steps,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? 0 : (int)cudaErrorInvalidValue;
}

template <typename K, typename... A>
int launch_cluster(K kernel, unsigned grid, unsigned threads, unsigned smem, unsigned cluster, void *stream, A... args) {
  int e = (int)cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e) return e;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim = {cluster, 1, 1};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = &attr;
  cfg.numAttrs = cluster > 1 ? 1 : 0;
  return (int)cudaLaunchKernelEx(&cfg, kernel, args...);
}

uint32_t ceil_div(uint64_t a, uint64_t b) { return (uint32_t)((a + b - 1) / b); }

// Whether a large product's sums over all of k may be the tensor cores' own.  These cut off
// each of the k/32 additions at up to 2^-23 of the sum so far, which over terms of one
// sign makes k 2^-29 of the result at most (measured with positive values: 1.5e-6 at 4,096, 3.9e-6
// at 8,192; with both signs 2.2e-7 and 4.9e-7; sums in registers 1e-7 and less, with no bias).
// That is to stay below a sixteenth of the rounding to out's type, 2^-8 or 2^-11: up to
// 131,072 in bf16 and 16,384 in fp16.  fp32 results are not rounded and never take them.
bool may_go_by_exponents(uint32_t out_dtype, uint32_t blocks) {
  return out_dtype == APC_BF16 ? blocks <= 1024 : out_dtype == APC_F16 ? blocks <= 128 : false;
}

// Which kernel, and for few columns how many and how far k is split: the least of
// the estimated times, in nanoseconds, of measured parts (one GB300, 152 SMs):
//   a block of 128 k takes a CTA 270, 330, 385 and 535 ns with 16, 32, 64 and 128
//   columns, a pair with a tile of 256 x 256 350 ns where it may go by exponents (the
//   scales are not known here), else 600 and, with a scale for every column, 900, and
//   1.8 us between tiles;
//   a cluster's exchange 2.2, 3 and 6.5 us for 2, 4 and 8 CTAs; a call 4 us beside
//   that, 8 with pairs.
// For example 100 x 4096 x 4096: 64 columns in two halves 13.8 us, whole 16.7, tiles
// of 128 22.0, of 256 x 256 19.6; 512 x 4096 x 4096: 30.7, 22.6 and 20.8 with tiles
// of 64, 128 and 256 (12.8 and 17.0 since for the two that are taken).  By sizes, out's type
// and the GPU's SMs alone: the cap of a grid does not change results.
struct Choice {
  uint32_t cols, split_log2;  // cols 256: the pairs' kernel
};

Choice choose(uint32_t m, uint32_t n, uint32_t blocks, uint32_t pair_ns, uint32_t sms) {
  static constexpr uint32_t kBlockNs[4] = {270, 330, 385, 535}, kExchangeNs[4] = {0, 2200, 3000, 6500};
  const uint64_t pairs = sms / 2 ? sms / 2 : 1;
  Choice best = {256, 0};
  uint64_t least = 8000 + ceil_div((uint64_t)ceil_div(m, 256) * ceil_div(n, 256), pairs) * ((uint64_t)blocks * pair_ns + 1800);
  for (uint32_t c = 0; c < 4; ++c)
    for (uint32_t s = 0; s <= (c == 3 ? 0u : 3u) && (1u << s) <= blocks && (1u << s) <= sms; ++s) {
      const uint64_t tiles = (uint64_t)ceil_div(n, 128) * ceil_div(m, 16u << c);
      const uint64_t t = 4000 + ceil_div(tiles, sms >> s) * ((uint64_t)ceil_div(blocks, 1u << s) * kBlockNs[c] + kExchangeNs[s]);
      if (t < least) least = t, best = {16u << c, s};
    }
  return best;
}

template <int BN, typename T>
int launch_mid(const MatmulArgs &a, ProductPlan p, uint32_t best, unsigned cap, void *stream) {
  p.r_scale = a.b_scale, p.c_scale = a.a_scale;
  p.r_scale_pitch = a.b_scale_pitch, p.c_scale_pitch = a.a_scale_pitch;
  p.r_shift = a.b_shift, p.c_shift = a.a_shift;
  p.rows = a.n, p.cols = a.m;
  p.row_tiles = ceil_div(a.n, 128), p.col_tiles = ceil_div(a.m, BN);
  p.instruction = 1u << 4 | a.b_e5m2 << 7 | a.a_e5m2 << 10 | (uint32_t)(BN >> 3) << 17 | 8u << 24;
  p.row_step = 1, p.col_step = a.out_pitch;
  CUtensorMap r, c;
  int e = encode(&r, a.b, a.n, a.k, a.b_pitch, 128);
  if (!e) e = encode(&c, a.a, a.m, a.k, a.a_pitch, BN);
  if (e) return e;
  const uint64_t tiles = (uint64_t)p.row_tiles * p.col_tiles;
  const uint64_t clusters = tiles < (cap >> best) ? tiles : (cap >> best);
  const unsigned grid = (unsigned)(clusters ? clusters : 1) << best;
  if (BN < 128 && best)
    return launch_cluster(mid_kernel<BN, BN < 128, T>, grid, kMidThreads, MidShape<BN, BN < 128>::kBytes, 1u << best, stream, r, c, p, best);
  return launch_cluster(mid_kernel<BN, false, T>, grid, kMidThreads, MidShape<BN, false>::kBytes, 1, stream, r, c, p, 0u);
}

template <typename T>
int launch_big(const MatmulArgs &a, ProductPlan p, unsigned cap, void *stream) {
  p.r_scale = a.a_scale, p.c_scale = a.b_scale;
  p.r_scale_pitch = a.a_scale_pitch, p.c_scale_pitch = a.b_scale_pitch;
  p.r_shift = a.a_shift, p.c_shift = a.b_shift;
  p.rows = a.m, p.cols = a.n;
  p.row_tiles = ceil_div(a.m, 256), p.col_tiles = ceil_div(a.n, 256);
  p.formats = a.a_e5m2 << 7 | a.b_e5m2 << 10;
  p.instruction = 1u << 4 | p.formats | (256u >> 3) << 17 | (256u >> 4) << 24;
  p.by_exponent = may_go_by_exponents(a.out_dtype, p.blocks);
  p.row_step = a.out_pitch, p.col_step = 1;
  const uint64_t size = a.out_dtype == APC_F32 ? 4 : 2;
  const bool aligned = (uintptr_t)a.out % 16 == 0 && (a.m <= 1 || (uint64_t)a.out_pitch * size % 16 == 0);
  CUtensorMap ma, mb;
  int e = encode(&ma, a.a, a.m, a.k, a.a_pitch, 128);
  if (!e) e = encode(&mb, a.b, a.n, a.k, a.b_pitch, 128);
  if (e) return e;
  const uint64_t tiles = (uint64_t)p.row_tiles * p.col_tiles, pairs = cap >= 2 ? cap / 2 : 1;
  const unsigned grid = (unsigned)(tiles < pairs ? tiles : pairs) * 2;
  auto go = [&](auto kernel) { return launch_cluster(kernel, grid, kBigThreads, kBigBytes, 2, stream, ma, mb, p); };
  if (aligned) return a.b_shift ? go(big_kernel<T, false, true>) : go(big_kernel<T, true, true>);
  return a.b_shift ? go(big_kernel<T, false, false>) : go(big_kernel<T, true, false>);
}

}  // namespace

int launch_matmul(const MatmulArgs &a, unsigned cap, unsigned sms, void *stream) {
  if (a.k == 0) {
    const size_t size = a.out_dtype == APC_F32 ? 4 : 2;
    return (int)cudaMemset2DAsync(a.out, (size_t)a.out_pitch * size, 0, a.n * size, a.m, (cudaStream_t)stream);
  }
  ProductPlan p = {};
  p.blocks = ceil_div(a.k, kBlock);
  p.out = a.out;
  int e = commit_status_word(&p.status);
  if (e) return e;
  const uint32_t pair_ns = may_go_by_exponents(a.out_dtype, p.blocks) ? 350 : a.b_shift ? 600 : 900;
  const Choice c = choose(a.m, a.n, p.blocks, pair_ns, sms);
  return with_dtype(a.out_dtype, [&](auto t) {
    using T = decltype(t);
    switch (c.cols) {
      case 16: return launch_mid<16, T>(a, p, c.split_log2, cap, stream);
      case 32: return launch_mid<32, T>(a, p, c.split_log2, cap, stream);
      case 64: return launch_mid<64, T>(a, p, c.split_log2, cap, stream);
      case 128: return launch_mid<128, T>(a, p, c.split_log2, cap, stream);
    }
    return launch_big<T>(a, p, cap, stream);
  });
}

}  // namespace apc
