// Host side of the operators around the output head: argument validation and
// launches.  Errors, pointer checks and grid sizes are apc_host.cpp's.
#include <cmath>
#include <cstddef>
#include <initializer_list>

#include "apc_ops.h"

#define APC_EXPORT extern "C" __attribute__((visibility("default")))

namespace {

using apc::OpRange;
using apc::op_fail;

constexpr int64_t kMaxSize = INT32_MAX;
constexpr int64_t kMaxPitch = (int64_t)1 << 40;

int64_t size_of(uint32_t dtype) { return dtype == APC_F32 ? 4 : 2; }

struct Ranges {
  OpRange r[12];
  int n = 0;

  // A matrix of so many rows, `width` bytes each, `pitch` bytes apart.
  void add(const char *name, const void *p, int64_t rows, int64_t width, int64_t pitch, bool written) {
    if (rows > 0 && width > 0)
      r[n++] = {(uintptr_t)p, (uintptr_t)p + (uintptr_t)((rows - 1) * pitch + width), (uintptr_t)width, rows > 1 ? (uintptr_t)pitch : 0, name, written};
  }
};

apc_status check_size(const char *name, int64_t v) {
  if (v < 0) return op_fail(APC_EINVAL, "%s %lld < 0", name, (long long)v);
  if (v > kMaxSize) return op_fail(APC_ERANGE, "%s %lld above 2^31 - 1", name, (long long)v);
  return APC_OK;
}

// A matrix of elements of `size` bytes, pitch in elements.
apc_status check_matrix(const char *name, const void *p, int64_t rows, int64_t cols, int64_t pitch, int64_t size) {
  if (rows == 0 || cols == 0) return APC_OK;
  if (!p) return op_fail(APC_EINVAL, "%s pointer is null", name);
  if (pitch < cols && rows > 1) return op_fail(APC_EINVAL, "%s: pitch %lld below its %lld columns", name, (long long)pitch, (long long)cols);
  if (pitch > kMaxPitch) return op_fail(APC_ERANGE, "%s: pitch %lld too large", name, (long long)pitch);
  if ((uintptr_t)p % (uintptr_t)size) return op_fail(APC_EALIGN, "%s not %d-byte aligned", name, (int)size);
  const uint64_t step = rows > 1 ? (uint64_t)pitch : 0;
  const bool huge = step > ((uint64_t)1 << 58) / (uint64_t)rows;
  if (huge || ((uint64_t)(rows - 1) * step + (uint64_t)cols) * (uint64_t)size > UINTPTR_MAX - (uintptr_t)p)
    return op_fail(APC_ERANGE, "%s: address range overflows", name);
  return APC_OK;
}

// One with a single row may have any pitch.
int64_t pitch_of(int64_t rows, int64_t cols, int64_t pitch) { return rows > 1 ? pitch : cols; }

apc_status check_fp8(const char *name, const apc_fp8_matrix *q, int64_t rows, int64_t cols, bool written, Ranges *rs) {
  if (!q) return op_fail(APC_EINVAL, "%s pointer is null", name);
  if (q->format > APC_E5M2) return op_fail(APC_EINVAL, "%s: unknown format %u", name, q->format);
  if (q->block_rows != 1 && q->block_rows != (uint32_t)apc::kBlock)
    return op_fail(APC_EINVAL, "%s: block_rows %u is neither 1 nor %d", name, q->block_rows, apc::kBlock);
  if (rows == 0 || cols == 0) return APC_OK;
  apc_status st = check_matrix(name, q->data, rows, cols, q->pitch, 1);
  if (st != APC_OK) return st;
  if ((uintptr_t)q->data % 16 || (rows > 1 && q->pitch % 16))
    return op_fail(APC_EALIGN, "%s: data or its pitch is not a multiple of 16 bytes", name);
  const int64_t lines = (cols + apc::kBlock - 1) / apc::kBlock, width = (rows + q->block_rows - 1) / q->block_rows;
  if ((st = check_matrix(name, q->scale, lines, width, q->scale_pitch, 4)) != APC_OK) return st;
  rs->add(name, q->data, rows, cols, q->pitch, written);
  rs->add(name, q->scale, lines, width * 4, q->scale_pitch * 4, written);
  return APC_OK;
}

apc::QuantOut quant_out(const apc_fp8_matrix *q) {
  return {static_cast<uint8_t *>(q->data), q->scale, q->pitch, q->scale_pitch, q->format == APC_E5M2};
}

}  // namespace

APC_EXPORT apc_status apc_quantize_fp8(const void *x, int64_t rows, int64_t cols, int64_t pitch, uint32_t dtype,
                                       const apc_fp8_matrix *q, const apc_fp8_matrix *qt, apc_stream_t stream) {
  apc::op_begin();
  apc_status st;
  if ((st = check_size("rows", rows)) != APC_OK || (st = check_size("cols", cols)) != APC_OK) return st;
  if (dtype > APC_F16) return op_fail(APC_EINVAL, "unknown dtype %u", dtype);
  Ranges rs;
  if ((st = check_matrix("x", x, rows, cols, pitch, size_of(dtype))) != APC_OK) return st;
  rs.add("x", x, rows, cols * size_of(dtype), pitch * size_of(dtype), false);
  if ((st = check_fp8("q", q, rows, cols, true, &rs)) != APC_OK) return st;
  if (qt) {
    if ((st = check_fp8("qt", qt, cols, rows, true, &rs)) != APC_OK) return st;
    if (qt->block_rows != q->block_rows || qt->format != q->format)
      return op_fail(APC_EINVAL, "q and qt differ in block_rows (%u, %u) or format (%u, %u)", q->block_rows, qt->block_rows,
                     q->format, qt->format);
  }
  if (rows == 0 || cols == 0) return APC_OK;
  if ((st = apc::op_ranges(rs.r, rs.n)) != APC_OK) return st;
  apc::QuantArgs a = {};
  a.x = x;
  a.pitch = pitch_of(rows, cols, pitch);
  a.rows = (uint32_t)rows;
  a.cols = (uint32_t)cols;
  a.dtype = dtype;
  a.square = q->block_rows != 1;
  a.q = quant_out(q);
  if (qt) a.qt = quant_out(qt);
  unsigned cap = 0;
  if ((st = apc::op_grid(apc::quantize_per_sm(a), &cap)) != APC_OK) return st;
  const int e = apc::launch_quantize(a, cap, stream);
  return e ? apc::op_cuda_fail(e, "quantize kernel launch") : APC_OK;
}

namespace {

// Sizes, types and inputs of a norm, and its sum.
apc_status check_norm(const apc_norm *d, Ranges *rs, apc::NormArgs *a) {
  apc_status st;
  if (!d) return op_fail(APC_EINVAL, "descriptor pointer is null");
  if ((st = check_size("rows", d->rows)) != APC_OK || (st = check_size("cols", d->cols)) != APC_OK) return st;
  if (d->dtype > APC_F16 || d->weight_dtype > APC_F16)
    return op_fail(APC_EINVAL, "unknown dtype %u or weight_dtype %u", d->dtype, d->weight_dtype);
  if (!((float)d->eps >= 1e-20f) || !std::isfinite((float)d->eps))
    return op_fail(APC_EINVAL, "eps %g is not a binary32 number from 1e-20 on", d->eps);
  const int64_t es = size_of(d->dtype), ws = size_of(d->weight_dtype), r = d->rows, c = d->cols;
  const bool adds = d->residual != nullptr;
  if (d->sum && !adds) return op_fail(APC_EINVAL, "sum without a residual");
  if ((st = check_matrix("x", d->x, r, c, d->pitch, es)) != APC_OK) return st;
  if (adds && (st = check_matrix("residual", d->residual, r, c, d->residual_pitch, es)) != APC_OK) return st;
  if (adds && (st = check_matrix("sum", d->sum, r, c, d->sum_pitch, es)) != APC_OK) return st;
  if ((st = check_matrix("weight", d->weight, r ? 1 : 0, c, c, ws)) != APC_OK) return st;
  // the sum may take the place of either of its terms
  const auto place = [&](const void *p, int64_t pitch) { return adds && p == d->sum && (pitch == d->sum_pitch || r <= 1); };
  if (!place(d->x, d->pitch)) rs->add("x", d->x, r, c * es, d->pitch * es, false);
  if (adds && !place(d->residual, d->residual_pitch))
    rs->add("residual", d->residual, r, c * es, d->residual_pitch * es, false);
  if (adds) rs->add("sum", d->sum, r, c * es, d->sum_pitch * es, true);
  rs->add("weight", d->weight, r ? 1 : 0, c * ws, 0, false);
  a->x = d->x;
  a->residual = d->residual;
  a->weight = d->weight;
  a->sum = d->sum;
  a->pitch = pitch_of(r, c, d->pitch);
  a->residual_pitch = adds ? pitch_of(r, c, d->residual_pitch) : 0;  // else whatever the caller left there
  a->sum_pitch = adds ? pitch_of(r, c, d->sum_pitch) : 0;
  a->rows = (uint32_t)r;
  a->cols = (uint32_t)c;
  a->dtype = d->dtype;
  a->wdtype = d->weight_dtype;
  a->eps = d->eps;
  return APC_OK;
}

apc_status run_norm(const apc::NormArgs &a, const Ranges &rs, apc_stream_t stream) {
  apc_status st = apc::op_ranges(rs.r, rs.n);
  unsigned cap = 0, sms = 0;
  if (st != APC_OK || (st = apc::op_grid(1, &cap, &sms)) != APC_OK) return st;
  const int e = apc::launch_rms_norm(a, sms, stream);
  return e ? apc::op_cuda_fail(e, "norm kernel launch") : APC_OK;
}

apc_status check_rstd(const float *rstd, int64_t rows, int64_t cols, bool written, Ranges *rs) {
  const apc_status st = check_matrix("rstd", rstd, cols ? 1 : 0, rows, rows, 4);
  if (st == APC_OK) rs->add("rstd", rstd, cols ? 1 : 0, rows * 4, 0, written);
  return st;
}

}  // namespace

APC_EXPORT apc_status apc_rms_norm(const apc_norm *d, void *out, int64_t out_pitch, float *rstd, apc_stream_t stream) {
  apc::op_begin();
  Ranges rs;
  apc::NormArgs a = {};
  apc_status st = check_norm(d, &rs, &a);
  if (st != APC_OK) return st;
  const int64_t es = size_of(d->dtype);
  if ((st = check_matrix("out", out, d->rows, d->cols, out_pitch, es)) != APC_OK) return st;
  rs.add("out", out, d->rows, d->cols * es, out_pitch * es, true);
  if ((st = check_rstd(rstd, d->rows, d->cols, true, &rs)) != APC_OK) return st;
  if (d->rows == 0 || d->cols == 0) return APC_OK;
  a.out = out;
  a.out_pitch = pitch_of(d->rows, d->cols, out_pitch);
  a.rstd = rstd;
  return run_norm(a, rs, stream);
}

APC_EXPORT apc_status apc_rms_norm_fp8(const apc_norm *d, const apc_fp8_matrix *q, const apc_fp8_matrix *qt, float *rstd,
                                       apc_stream_t stream) {
  apc::op_begin();
  Ranges rs;
  apc::NormArgs a = {};
  apc_status st = check_norm(d, &rs, &a);
  if (st != APC_OK) return st;
  if ((st = check_fp8("q", q, d->rows, d->cols, true, &rs)) != APC_OK) return st;
  if (q->block_rows != 1) return op_fail(APC_EINVAL, "q: block_rows %u is not 1", q->block_rows);
  if (qt) {
    if ((st = check_fp8("qt", qt, d->cols, d->rows, true, &rs)) != APC_OK) return st;
    if (qt->block_rows != 1 || qt->format != q->format)
      return op_fail(APC_EINVAL, "qt: block_rows %u is not 1 or its format (%u) is not q's (%u)", qt->block_rows, qt->format, q->format);
  }
  if ((st = check_rstd(rstd, d->rows, d->cols, true, &rs)) != APC_OK) return st;
  if (d->rows == 0 || d->cols == 0) return APC_OK;
  a.q = quant_out(q);
  if (qt) a.qt = quant_out(qt);
  a.rstd = rstd;
  return run_norm(a, rs, stream);
}

APC_EXPORT int64_t apc_rms_norm_grad_workspace(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || rows > kMaxSize || cols > kMaxSize) return 0;
  return (int64_t)apc::rms_norm_parts((uint32_t)rows, (uint32_t)cols) * cols * 4;
}

APC_EXPORT apc_status apc_rms_norm_grad(const apc_norm_grad *d, void *dx, int64_t dx_pitch, void *dweight, uint32_t dweight_dtype,
                                        float *workspace, apc_stream_t stream) {
  apc::op_begin();
  apc_status st;
  if (!d) return op_fail(APC_EINVAL, "descriptor pointer is null");
  if ((st = check_size("rows", d->rows)) != APC_OK || (st = check_size("cols", d->cols)) != APC_OK) return st;
  if (d->dtype > APC_F16 || d->weight_dtype > APC_F16 || (dweight && dweight_dtype > APC_F16))
    return op_fail(APC_EINVAL, "unknown dtype %u, weight_dtype %u or dweight_dtype %u", d->dtype, d->weight_dtype, dweight_dtype);
  const int64_t es = size_of(d->dtype), ws = size_of(d->weight_dtype), r = d->rows, c = d->cols;
  Ranges rs;
  // dx may take the place of dout or of dresidual
  const auto place = [&](const void *p, int64_t pitch) { return p == dx && (pitch == dx_pitch || r <= 1); };
  if ((st = check_matrix("dout", d->dout, r, c, d->dout_pitch, es)) != APC_OK) return st;
  if (!place(d->dout, d->dout_pitch)) rs.add("dout", d->dout, r, c * es, d->dout_pitch * es, false);
  if ((st = check_matrix("x", d->x, r, c, d->pitch, es)) != APC_OK) return st;
  rs.add("x", d->x, r, c * es, d->pitch * es, false);
  if (d->dresidual) {
    if ((st = check_matrix("dresidual", d->dresidual, r, c, d->dresidual_pitch, es)) != APC_OK) return st;
    if (!place(d->dresidual, d->dresidual_pitch)) rs.add("dresidual", d->dresidual, r, c * es, d->dresidual_pitch * es, false);
  }
  if ((st = check_matrix("weight", d->weight, r ? 1 : 0, c, c, ws)) != APC_OK) return st;
  rs.add("weight", d->weight, r ? 1 : 0, c * ws, 0, false);
  if ((st = check_rstd(d->rstd, r, c, false, &rs)) != APC_OK) return st;
  if ((st = check_matrix("dx", dx, r, c, dx_pitch, es)) != APC_OK) return st;
  rs.add("dx", dx, r, c * es, dx_pitch * es, true);
  if (dweight) {
    const int64_t dws = size_of(dweight_dtype), work = apc_rms_norm_grad_workspace(r, c);
    if ((st = check_matrix("dweight", dweight, 1, c, c, dws)) != APC_OK) return st;
    rs.add("dweight", dweight, 1, c * dws, 0, true);
    if ((st = check_matrix("workspace", workspace, 1, work / 4, work / 4, 4)) != APC_OK) return st;
    rs.add("workspace", workspace, 1, work, 0, true);
  }
  if (c == 0 || (r == 0 && !dweight)) return APC_OK;
  unsigned cap = 0, sms = 0;
  if ((st = apc::op_ranges(rs.r, rs.n)) != APC_OK || (st = apc::op_grid(1, &cap, &sms)) != APC_OK) return st;
  apc::NormGradArgs a = {};
  a.dout = d->dout;
  a.x = d->x;
  a.weight = d->weight;
  a.dresidual = d->dresidual;
  a.rstd = d->rstd;
  a.dx = dx;
  a.dweight = dweight;
  a.work = workspace;
  a.dout_pitch = pitch_of(r, c, d->dout_pitch);
  a.pitch = pitch_of(r, c, d->pitch);
  a.dresidual_pitch = d->dresidual ? pitch_of(r, c, d->dresidual_pitch) : 0;
  a.dx_pitch = pitch_of(r, c, dx_pitch);
  a.rows = (uint32_t)r;
  a.cols = (uint32_t)c;
  a.dtype = d->dtype;
  a.wdtype = d->weight_dtype;
  a.dwdtype = dweight_dtype;
  const int e = apc::launch_rms_norm_grad(a, sms, stream);
  return e ? apc::op_cuda_fail(e, "norm gradient kernel launch") : APC_OK;
}

APC_EXPORT apc_status apc_matmul_fp8(const apc_fp8_matrix *a, const apc_fp8_matrix *b, int64_t m, int64_t n, int64_t k,
                                     void *out, int64_t out_pitch, uint32_t out_dtype, apc_stream_t stream) {
  apc::op_begin();
  apc_status st;
  if ((st = check_size("m", m)) != APC_OK || (st = check_size("n", n)) != APC_OK || (st = check_size("k", k)) != APC_OK)
    return st;
  if (out_dtype > APC_F16) return op_fail(APC_EINVAL, "unknown out_dtype %u", out_dtype);
  const int64_t os = size_of(out_dtype);
  Ranges rs;
  if ((st = check_fp8("a", a, m, k, false, &rs)) != APC_OK || (st = check_fp8("b", b, n, k, false, &rs)) != APC_OK) return st;
  if ((st = check_matrix("out", out, m, n, out_pitch, os)) != APC_OK) return st;
  rs.add("out", out, m, n * os, out_pitch * os, true);
  if (m == 0 || n == 0) return APC_OK;
  if ((st = apc::op_ranges(rs.r, rs.n)) != APC_OK) return st;
  apc::MatmulArgs p = {};
  p.a = static_cast<const uint8_t *>(a->data);
  p.b = static_cast<const uint8_t *>(b->data);
  p.a_scale = a->scale;
  p.b_scale = b->scale;
  p.a_pitch = a->pitch;
  p.b_pitch = b->pitch;
  p.a_scale_pitch = a->scale_pitch;
  p.b_scale_pitch = b->scale_pitch;
  p.a_shift = a->block_rows == 1 ? 0 : 7;
  p.b_shift = b->block_rows == 1 ? 0 : 7;
  p.a_e5m2 = a->format == APC_E5M2;
  p.b_e5m2 = b->format == APC_E5M2;
  p.m = (uint32_t)m;
  p.n = (uint32_t)n;
  p.k = (uint32_t)k;
  p.out = out;
  p.out_pitch = pitch_of(m, n, out_pitch);
  p.out_dtype = out_dtype;
  unsigned cap = 0;
  unsigned sms = 0;
  if ((st = apc::op_grid(1, &cap, &sms)) != APC_OK) return st;
  const int e = apc::launch_matmul(p, cap, sms, stream);
  return e ? apc::op_cuda_fail(e, "product kernel launch") : APC_OK;
}

APC_EXPORT int64_t apc_grad_norm_workspace(const apc_buffer *bufs, int32_t num_bufs) {
  return apc::grad_norm_workspace(bufs, num_bufs);
}

APC_EXPORT apc_status apc_grad_norm(const apc_buffer *bufs, int32_t num_bufs, int32_t num_slots, void *workspace,
                                    apc_stream_t stream, float *out_norms) {
  apc::op_begin();
  return apc::grad_norm(bufs, num_bufs, num_slots, workspace, stream, out_norms, apc::launch_norm);
}

namespace {

apc_status distill(const apc_distill *d, const float *grad_loss, float *loss, float *lse, void *dlogits, int64_t dpitch,
                   apc_stream_t stream) {
  apc_status st;
  if (!d) return op_fail(APC_EINVAL, "descriptor pointer is null");
  if ((st = check_size("rows", d->rows)) != APC_OK || (st = check_size("vocab", d->vocab)) != APC_OK ||
      (st = check_size("k", d->k)) != APC_OK)
    return st;
  if (d->k > APC_DISTILL_MAX_K) return op_fail(APC_EINVAL, "k %lld above %d", (long long)d->k, APC_DISTILL_MAX_K);
  if (d->dtype > APC_F16) return op_fail(APC_EINVAL, "unknown dtype %u", d->dtype);
  if (d->k && (d->teacher_dtype > APC_F16 || d->ids_dtype > APC_I64))
    return op_fail(APC_EINVAL, "unknown teacher_dtype %u or ids_dtype %u", d->teacher_dtype, d->ids_dtype);
  if (d->labels && d->labels_dtype > APC_I64) return op_fail(APC_EINVAL, "unknown labels_dtype %u", d->labels_dtype);
  const double tau = d->temperature;
  if (!std::isfinite(tau) || !((float)tau > 0.0f) || !std::isfinite((float)(1.0 / tau) * 1.4426950408889634f))
    return op_fail(APC_EINVAL, "temperature %g is not a positive binary32 number with a finite reciprocal", tau);
  for (const double w : {d->kd_weight, d->kd_weight * tau, d->kd_weight * tau * tau, d->label_weight})
    if (!std::isfinite(w) || w < 0 || !std::isfinite((float)w))
      return op_fail(APC_EINVAL, "weight %g is negative or too large (the teacher's is taken times the temperature's square)", w);
  const int64_t es = size_of(d->dtype), ts = size_of(d->teacher_dtype), is = d->ids_dtype == APC_I64 ? 8 : 4;
  const int64_t ls = d->labels_dtype == APC_I64 ? 8 : 4, rows = d->rows, v = d->vocab;
  if (rows > 0 && v == 0) return op_fail(APC_EINVAL, "vocab is 0");
  Ranges rs;
  // the logits' own memory may take the gradient
  const bool in_place = dlogits && dlogits == d->logits && (dpitch == d->pitch || rows <= 1);
  if ((st = check_matrix("logits", d->logits, rows, v, d->pitch, es)) != APC_OK) return st;
  if (!in_place) rs.add("logits", d->logits, rows, v * es, d->pitch * es, false);
  if ((st = check_matrix("ids", d->ids, rows, d->k, d->ids_pitch, is)) != APC_OK) return st;
  rs.add("ids", d->ids, rows, d->k * is, d->ids_pitch * is, false);
  if ((st = check_matrix("teacher", d->teacher, rows, d->k, d->teacher_pitch, ts)) != APC_OK) return st;
  rs.add("teacher", d->teacher, rows, d->k * ts, d->teacher_pitch * ts, false);
  if (d->teacher_lse && d->k) {
    if ((st = check_matrix("teacher_lse", d->teacher_lse, 1, rows, rows, 4)) != APC_OK) return st;
    rs.add("teacher_lse", d->teacher_lse, 1, rows * 4, 0, false);
  }
  if (d->labels) {
    if ((st = check_matrix("labels", d->labels, 1, rows, rows, ls)) != APC_OK) return st;
    rs.add("labels", d->labels, 1, rows * ls, 0, false);
  }
  if (loss || !grad_loss) {
    if ((st = check_matrix("loss", loss, 1, rows, rows, 4)) != APC_OK) return st;
    rs.add("loss", loss, 1, rows * 4, 0, true);
  }
  const int64_t stats = d->labels ? 2 : 1;
  if ((st = check_matrix("lse", lse, stats, rows, rows, 4)) != APC_OK) return st;
  rs.add("lse", lse, 1, stats * rows * 4, 0, loss != nullptr);
  if (dlogits || grad_loss) {
    if ((st = check_matrix("grad_loss", grad_loss, 1, rows, rows, 4)) != APC_OK) return st;
    rs.add("grad_loss", grad_loss, 1, rows * 4, 0, false);
    if ((st = check_matrix("dlogits", dlogits, rows, v, dpitch, es)) != APC_OK) return st;
    rs.add("dlogits", dlogits, rows, v * es, dpitch * es, true);
  }
  if (rows == 0) return APC_OK;
  if ((st = apc::op_ranges(rs.r, rs.n)) != APC_OK) return st;
  apc::DistillArgs a = {};
  // without a weight there is no teacher's part: its probabilities times 0 would be NaN where
  // a logarithm is infinite
  const int64_t k = (float)d->kd_weight != 0.0f ? d->k : 0;
  a.logits = d->logits;
  a.ids = d->ids;
  a.teacher = d->teacher;
  a.labels = d->labels;
  a.teacher_lse = k ? d->teacher_lse : nullptr;
  a.grad_loss = grad_loss;
  a.loss = loss;
  a.lse = lse;
  a.dlogits = dlogits;
  a.pitch = pitch_of(rows, v, d->pitch);
  a.ids_pitch = pitch_of(rows, k, d->ids_pitch);
  a.teacher_pitch = pitch_of(rows, k, d->teacher_pitch);
  a.dpitch = pitch_of(rows, v, dpitch);
  a.rows = (uint32_t)rows;
  a.vocab = (uint32_t)v;
  a.k = (uint32_t)k;
  a.dtype = d->dtype;
  a.teacher_dtype = d->teacher_dtype;
  a.ids64 = d->ids_dtype == APC_I64;
  a.labels64 = d->labels_dtype == APC_I64;
  a.inv_tau = (float)(1.0 / tau);
  a.scale2 = (float)(1.4426950408889634 / tau);
  a.loss_kd = (float)(d->kd_weight * tau * tau);
  a.grad_kd = (float)(d->kd_weight * tau);
  a.loss_label = (float)d->label_weight;
  unsigned cap = 0;
  unsigned sms = 0;
  if ((st = apc::op_grid(1, &cap, &sms)) != APC_OK || (st = apc::op_grid(apc::distill_per_sm(a, sms), &cap)) != APC_OK) return st;
  const int e = apc::launch_distill(a, cap, sms, stream);
  return e ? apc::op_cuda_fail(e, "distillation kernel launch") : APC_OK;
}

}  // namespace

APC_EXPORT apc_status apc_distill_loss(const apc_distill *d, float *loss, float *lse, apc_stream_t stream) {
  apc::op_begin();
  if (!loss && d && d->rows > 0) return op_fail(APC_EINVAL, "loss pointer is null");
  return distill(d, nullptr, loss, lse, nullptr, 0, stream);
}

APC_EXPORT apc_status apc_distill_grad(const apc_distill *d, const float *lse, const float *grad_loss, void *dlogits,
                                       int64_t dlogits_pitch, apc_stream_t stream) {
  apc::op_begin();
  if ((!grad_loss || !dlogits) && d && d->rows > 0) return op_fail(APC_EINVAL, "grad_loss or dlogits pointer is null");
  return distill(d, grad_loss, nullptr, const_cast<float *>(lse), dlogits, dlogits_pitch, stream);
}

APC_EXPORT apc_status apc_distill_loss_grad(const apc_distill *d, const float *grad_loss, float *loss, float *lse,
                                            void *dlogits, int64_t dlogits_pitch, apc_stream_t stream) {
  apc::op_begin();
  if ((!grad_loss || !dlogits || !loss) && d && d->rows > 0)
    return op_fail(APC_EINVAL, "grad_loss, loss or dlogits pointer is null");
  return distill(d, grad_loss, loss, lse, dlogits, dlogits_pitch, stream);
}
