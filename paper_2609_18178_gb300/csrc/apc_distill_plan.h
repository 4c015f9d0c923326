// How the distillation kernel for longer rows (apc_distill.cu) shares out a CTA's
// shared memory.  Plain C++, so that the CPU's tests can ask it too.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define APC_BOTH __host__ __device__
#else
#define APC_BOTH
#endif

namespace apc {

// Warps on the logits and on the teacher's entries, CTAs on an SM.  Measured on loss
// and gradient of 8192 x 32768 with labels, when this shape took 254 us: 1 CTA of 16
// warps 310, 12 warps 275, 4 warps 282 and, with 3 CTAs, 313.  Since then (199 us): 3
// teachers 215, 2 252.
constexpr int kWarps = 8, kWorkers = 32 * kWarps, kTeachers = 4, kCtas = 2;
constexpr int kMaxChunks = 16;
constexpr uint32_t kSharedBytes = 1536;  // of barriers, sums and pointers
// Vectors of 16 bytes that each thread on the logits takes of a chunk.  Loss and
// gradient hold a row between their passes, and smaller chunks let more of the next
// row in meanwhile: 199 us on the same case (8 vectors 208, 5 219, 2 230).  The others let
// chunks go at once and want fewer turns: loss of 4096 x 32768 41.9 us (4 vectors
// 43.9), gradient of 1021 x 100003 83.7 (85.1).
template <int FORM>
constexpr int kVectorsOf = FORM == 3 ? 4 : 8;

// Behind those: the ring, each teacher's table of ids (for a gradient), the entries of one
// row more than there are teachers and, for the loss alone, as many rows' sums of every
// worker.  room: entries of a row, the label's among them; tables, sums: words of them all
// and of a row's; chunk: vectors.
struct Layout {
  uint32_t chunk, chunks, teachers, room, slots_log2, tables, sums;
  APC_BOTH uint32_t bytes() const {
    return kSharedBytes + chunks * chunk * 16 + (teachers + 1) * (room * 12 + sums * 4) + tables * 4;
  }
};

// Slots of a row's table of ids: at most half of them are taken.
inline uint32_t slots_log2_of(uint32_t k) {
  uint32_t n = 6;
  while ((1u << n) < 2 * (k + 1)) ++n;
  return n;
}

inline uint32_t room_of(uint32_t k) { return (k + 1 + 3) / 4 * 4; }

// As many teachers as leave the ring 32 KB.  With large k their reads are the bound: 4096 x
// 32768 with k = 513, loss 135 us with four, 421 with one; gradient 199 and 505 (with k = 512
// and two, for a ring of two chunks, 293).  The loss alone from k = 256 on takes no second
// chunk either: the copies ahead are in the teachers' way (k = 256 77 us for 81, 400 112 for 116).
inline Layout distill_layout(uint32_t k, bool loss, bool grad) {
  constexpr uint32_t kRoom = 228 * 1024 / kCtas - 1024;  // an SM's shared memory; 1 KB of each CTA's is the system's
  Layout l = {};
  l.chunk = (loss && grad ? kVectorsOf<3> : kVectorsOf<1>) * kWorkers;
  l.room = room_of(k);
  l.slots_log2 = slots_log2_of(k);
  l.sums = grad ? 0 : 3 * kWorkers;
  for (l.teachers = kTeachers;; --l.teachers) {
    l.tables = grad ? l.teachers << l.slots_log2 : 0;
    if (l.teachers == 1 || l.bytes() + 32 * 1024 <= kRoom) break;
  }
  const uint32_t fit = (kRoom - l.bytes()) / (l.chunk * 16);
  l.chunks = !grad && k >= 256 ? 1 : fit < (uint32_t)kMaxChunks ? fit : (uint32_t)kMaxChunks;
  return l;
}

}  // namespace apc
