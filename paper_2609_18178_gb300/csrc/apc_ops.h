// The operators around the output head (quantization, 8-bit product,
// distillation): what their host side (apc_ops_host.cpp), their kernels
// (apc_quantize.cu, apc_matmul.cu, apc_distill.cu) and apc_host.cpp share.
#pragma once

#include <stdint.h>

#include "../../include/apc.h"

namespace apc {

// ---- of apc_host.cpp: the error text, the pointer checks, the persistent grid
struct OpRange {
  uintptr_t lo, hi;  // [lo, hi), not empty
  uintptr_t width, pitch;  // rows of so many bytes, so far apart; a single one: pitch 0
  const char *name;
  bool written;

  // Column ranges of one buffer lie between each other's rows.
  bool overlaps(const OpRange &o) const {
    if (lo >= o.hi || o.lo >= hi) return false;
    if (!pitch || pitch != o.pitch) return true;
    const uintptr_t at = (lo > o.lo ? lo - o.lo : pitch - (o.lo - lo) % pitch) % pitch;  // this one's columns behind the other's
    return at < o.width || at + width > pitch;
  }
};

void op_begin();
__attribute__((format(printf, 2, 3))) apc_status op_fail(apc_status s, const char *fmt, ...);
apc_status op_cuda_fail(int err, const char *what);
apc_status op_ranges(const OpRange *r, int n);
// CTAs of a persistent grid with so many resident per SM, after
// apc_set_reserved_sms and APC_GRID_LIMIT.
apc_status op_grid(int per_sm, unsigned *cap, unsigned *sms = nullptr);

// ---- the gradients' norm: planned by apc_host.cpp like the other buffer lists,
// launched by apc_gradnorm.cu.  plan: a NormPlan of so many entries; work null: a small list.
typedef int (*NormLaunch)(const void *plan, int size, unsigned grid, void *stream, unsigned long long *work, float *out,
                          unsigned slots);
int launch_norm(const void *plan, int size, unsigned grid, void *stream, unsigned long long *work, float *out, unsigned slots);
apc_status grad_norm(const apc_buffer *bufs, int32_t num_bufs, int32_t num_slots, void *work, apc_stream_t stream, float *out,
                     NormLaunch launch);
int64_t grad_norm_workspace(const apc_buffer *bufs, int32_t num_bufs);

constexpr int kBlock = 128;  // columns (and, in square blocks, rows) that share a scale

// ---- quantization
struct QuantOut {
  uint8_t *data;
  float *scale;
  int64_t pitch, scale_pitch;
  uint32_t e5m2;
};

struct QuantArgs {
  const void *x;
  int64_t pitch;  // elements
  uint32_t rows, cols;
  uint32_t dtype;
  uint32_t square;  // 128 x 128 blocks
  QuantOut q, qt;   // qt.data null: no transpose
};

int launch_quantize(const QuantArgs &a, unsigned cap, void *stream);
int quantize_per_sm(const QuantArgs &a);

// ---- root-mean-square norm
struct NormArgs {
  const void *x, *residual, *weight;  // residual null: none, and no sum
  void *sum;
  void *out;        // null: y in 8 bits
  QuantOut q, qt;   // qt.data null: no transpose
  float *rstd;
  int64_t pitch, residual_pitch, sum_pitch, out_pitch;
  uint32_t rows, cols, dtype, wdtype;
  double eps;
};

int launch_rms_norm(const NormArgs &a, unsigned sms, void *stream);

struct NormGradArgs {
  const void *dout, *x, *weight, *dresidual;  // dresidual null: none
  const float *rstd;
  void *dx;
  void *dweight;    // null: not wanted
  float *work;      // rms_norm_parts(rows, cols) x cols; null where that is none
  int64_t dout_pitch, pitch, dresidual_pitch, dx_pitch;
  uint32_t rows, cols, dtype, wdtype, dwdtype;
};

// Runs of rows whose sums of the weight's gradient are kept apart.
uint32_t rms_norm_parts(uint32_t rows, uint32_t cols);
int launch_rms_norm_grad(const NormGradArgs &a, unsigned sms, void *stream);

// ---- product
struct MatmulArgs {
  const uint8_t *a, *b;
  const float *a_scale, *b_scale;
  int64_t a_pitch, b_pitch, a_scale_pitch, b_scale_pitch;
  uint32_t a_shift, b_shift;  // log2 of the rows of a scale: 0 or 7
  uint32_t a_e5m2, b_e5m2;
  uint32_t m, n, k;
  void *out;
  int64_t out_pitch;
  uint32_t out_dtype;
};

// cap: CTAs of the persistent grid; sms: the device's SMs, by which sizes alone choose
// a kernel and a split.  Returns a cudaError_t value, as the others do.
int launch_matmul(const MatmulArgs &a, unsigned cap, unsigned sms, void *stream);
// The device status word of apc_device_status (apc_commit.cu) on the current device.
int commit_status_word(unsigned **out);

// ---- distillation
struct DistillArgs {
  const void *logits, *ids, *teacher, *labels;
  const float *teacher_lse;
  const float *grad_loss;  // null: loss alone
  float *loss;             // null: gradient alone
  float *lse;              // written with the loss, else read
  void *dlogits;
  int64_t pitch, ids_pitch, teacher_pitch, dpitch;
  uint32_t rows, vocab, k;
  uint32_t dtype, teacher_dtype;
  uint32_t ids64, labels64;
  float inv_tau;             // 1/tau
  float scale2;              // log2(e)/tau
  float loss_kd, loss_label; // kd_weight*tau^2, label_weight
  float grad_kd;             // kd_weight*tau
  unsigned *status;          // the device status word
};

int launch_distill(const DistillArgs &a, unsigned cap, unsigned sms, void *stream);
int distill_per_sm(const DistillArgs &a, unsigned sms);

}  // namespace apc
