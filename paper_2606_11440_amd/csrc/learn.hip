// C ABI of the learner's operators: checks of arguments, workspaces, launches.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <new>
#include <vector>

#include "learn_adamw.h"
#include "learn_host.h"

using namespace im::learn;

struct im_adamw {
  int device = 0;
  int bits = 32, grad_dtype = IM_F32;
  int64_t runs = 0, blocks = 1;
  AdamwRun* table = nullptr;
  im_adamw_tensor* tensors = nullptr;
  uint32_t* done = nullptr;
};

thread_local char im::learn::t_error[256] = "no error";

extern "C" {

const char* im_learn_last_error(void) { return t_error; }

im_status im_linear_workspace(const im_linear_desc* d, int32_t backward, int64_t* bytes) {
  LEARN_OK(check_linear(d));
  LEARN_CHECK(bytes, "bytes is NULL");
  LEARN_CHECK(backward == 0 || backward == 1, "backward is 0 or 1");
  *bytes = backward ? linear_backward(*d, nullptr).bytes : linear_forward(*d, nullptr).bytes;
  return IM_OK;
}

im_status im_linear_forward(const im_linear_desc* d, const int32_t* offsets, const void* x, const void* W,
                            const float* b, void* y, void* ws, int64_t ws_bytes, int32_t* error, void* stream) {
  LEARN_OK(check_linear(d));
  LEARN_OK(check_groups(d->n_groups, offsets));
  const int64_t e = size_of(d->dtype);
  LEARN_CHECK(stride_ok(d->ld_x, d->in_dim) && stride_ok(d->ld_y, d->out_dim), "ld_x or ld_y out of range");
  LEARN_CHECK(W && (d->n_rows == 0 || (x && y)), "x, W or y is NULL");
  LEARN_CHECK(aligned(x, e) && aligned(W, e) && aligned(y, e) && aligned(b, 4) && aligned(error, 4),
              "a pointer is not aligned to its elements");
  const RowWork w = linear_forward(*d, ws);
  const int64_t n = d->n_rows, G = d->n_groups, k = d->in_dim, m = d->out_dim;
  if (n > 0) {
    LEARN_OK(check_launch(w.plan));
    LEARN_OK(check_areas({flat("offsets", offsets, 4 * (G + 1), false), matrix("x", x, n, k, d->ld_x, e, false),
                          flat("W", W, G * m * k * e, false), flat("b", b, 4 * G * m, false),
                          matrix("y", y, n, m, d->ld_y, e, true), flat("workspace", ws, w.bytes, true),
                          flat("error", error, 4, true)}));
  }
  LEARN_OK(check_work(ws, ws_bytes, w.bytes));
  if (n == 0) return IM_OK;
  RowArgs a = row_args(offsets, d->n_groups, d->n_rows, w.plan, error);
  a.part = w.part;
  a.K = d->in_dim;
  a.N = d->out_dim;
  a.A = x;
  a.lda = d->ld_x;
  a.B = W;
  a.ldb = d->in_dim;
  a.b_group = (int64_t)d->in_dim * d->out_dim;
  a.bias = b;
  a.bias_group = d->out_dim;
  a.C = y;
  a.ldc = d->ld_y;
  a.relu = d->relu;
  LEARN_HIP(launch_rows_product(a, d->dtype, w.plan.shape, kStore, (hipStream_t)stream));
  return IM_OK;
}

im_status im_linear_backward(const im_linear_desc* d, const int32_t* offsets, const void* dy, const void* x,
                             const void* W, void* dx, void* dW, float* db, void* ws, int64_t ws_bytes, int32_t* error,
                             void* stream) {
  LEARN_OK(check_linear(d));
  LEARN_OK(check_groups(d->n_groups, offsets));
  const int64_t e = size_of(d->dtype);
  const bool some = d->n_rows > 0;
  LEARN_CHECK(!some || dy, "dy is NULL");
  LEARN_CHECK(stride_ok(d->ld_y, d->out_dim), "ld_y out of range");
  LEARN_CHECK(!dx || !some || (W && stride_ok(d->ld_dx, d->in_dim)), "dx needs W and a valid ld_dx");
  LEARN_CHECK(!some || !(dW || (dx && d->relu_in)) || (x && stride_ok(d->ld_x, d->in_dim)),
              "dW, and dx with relu_in, need x and a valid ld_x");
  LEARN_CHECK(aligned(dy, e) && aligned(x, e) && aligned(W, e) && aligned(dx, e) && aligned(dW, e) && aligned(db, 4) &&
                  aligned(error, 4),
              "a pointer is not aligned to its elements");
  const LinearBackward w = linear_backward(*d, ws);
  LEARN_OK(check_launch(w.input.plan));
  LEARN_OK(check_grid(w.sums.plan));
  const int64_t n = d->n_rows, G = d->n_groups, k = d->in_dim, m = d->out_dim;
  const bool reads_x = dW || (dx && d->relu_in);
  LEARN_OK(check_areas({flat("offsets", offsets, 4 * (G + 1), false), matrix("dy", dy, n, m, d->ld_y, e, false),
                        matrix("x", reads_x ? x : nullptr, n, k, d->ld_x, e, false),
                        flat("W", dx ? W : nullptr, G * m * k * e, false), matrix("dx", dx, n, k, d->ld_dx, e, true),
                        flat("dW", dW, G * m * k * e, true), flat("db", db, 4 * G * m, true),
                        flat("workspace", ws, w.bytes, true), flat("error", error, 4, true)}));
  LEARN_OK(check_work(ws, ws_bytes, w.bytes));
  if (dx && some) {
    RowArgs a = row_args(offsets, d->n_groups, d->n_rows, w.input.plan, error);
    a.part = w.input.part;
    a.K = d->out_dim;
    a.N = d->in_dim;
    a.A = dy;
    a.lda = d->ld_y;
    a.B = W;
    a.ldb = d->in_dim;
    a.b_group = (int64_t)d->in_dim * d->out_dim;
    a.C = dx;
    a.ldc = d->ld_dx;
    a.X = d->relu_in ? x : nullptr;
    a.ldx = d->ld_x;
    a.first = a.last = 1;
    LEARN_HIP(launch_rows_product(a, d->dtype, w.input.plan.shape, kStoreInput, (hipStream_t)stream));
  }
  if (dW || db) {
    SumArgs a = {};
    a.offsets = offsets;
    a.G = d->n_groups;
    a.n = d->n_rows;
    a.M = d->out_dim;
    a.N = dW ? d->in_dim : 1;   // db alone: a column of dy in place of x
    a.P = dy;
    a.ldp = d->ld_y;
    a.Q = dW ? x : dy;
    a.ldq = dW ? d->ld_x : d->ld_y;
    a.dW = dW;
    a.w_group = (int64_t)d->in_dim * d->out_dim;
    a.db = db;
    a.part = w.sums.part;
    a.cuts = w.sums.cuts;
    a.granule = (int32_t)w.sums.plan.granule;
    a.parts = (int32_t)w.sums.plan.parts;
    a.row_tiles = (int32_t)w.sums.plan.row_tiles;
    a.col_tiles = dW ? (int32_t)w.sums.plan.col_tiles : 1;
    a.error = error;
    LEARN_HIP(launch_sums(a, d->dtype, w.sums.plan.shape, (hipStream_t)stream));
  }
  return IM_OK;
}

// ---- softmax head ----------------------------------------------------------------

}  // extern "C"

namespace {

im_status check_head(const im_head_desc* d) {
  LEARN_CHECK(d, "desc is NULL");
  LEARN_CHECK(d->n_groups >= 1 && d->n_groups <= IM_MAX_GROUPS, "n_groups out of range");
  LEARN_CHECK(d->n_rows >= 0 && d->n_rows <= IM_MAX_ROWS, "n_rows out of range");
  LEARN_CHECK(d->dim >= 1 && d->dim <= IM_MAX_DIM, "dim out of range");
  LEARN_CHECK(d->n_classes >= 1 && d->n_classes <= IM_MAX_CLASSES, "n_classes out of range");
  LEARN_CHECK(d->dtype == IM_F32 || d->dtype == IM_BF16, "dtype out of range");
  LEARN_CHECK(d->relu_in == 0 || d->relu_in == 1, "relu_in is 0 or 1");
  return IM_OK;
}

struct HeadForward {
  RowPlan plan;
  float *stats, *taken;
  int64_t bytes;
};
HeadForward head_forward(const im_head_desc& d, void* ws) {
  HeadForward w;
  w.plan = plan_rows(d.dtype, d.n_rows, d.n_groups, d.n_classes, d.dim, compute_units(), false);
  Sections s(ws);
  const bool split = w.plan.col_tiles > 1;
  w.stats = s.take<float>(split ? w.plan.col_tiles * d.n_rows * 3 : 0);
  w.taken = s.take<float>(split ? d.n_rows : 0);
  w.bytes = s.used;
  return w;
}

// The gradient's pieces: dz of `width` classes at a time.
struct HeadBackward {
  int64_t width, pieces;
  RowPlan logits;
  RowWork input;
  SumWork sums;
  void* dz;
  float *sum, *db_part;
  uint8_t* live;
  int64_t bytes;
};
HeadBackward head_backward(const im_head_desc& d, void* ws) {
  HeadBackward w;
  const int64_t n = d.n_rows, G = d.n_groups, V = d.n_classes;
  const int cus = compute_units();
  // dz of a piece stays within 2^27 elements; pieces are alike and 1024 classes at least
  const int64_t most = n > 0 ? ((int64_t)1 << 27) / n : V;
  w.pieces = (V + (most < 1024 ? 1024 : most) - 1) / (most < 1024 ? 1024 : most);
  w.width = w.pieces > 1 ? ((V + w.pieces - 1) / w.pieces + 255) / 256 * 256 : (V + 7) / 8 * 8;
  w.pieces = (V + w.width - 1) / w.width;
  const int64_t classes = w.pieces > 1 ? w.width : V;
  w.logits = plan_rows(d.dtype, n, G, classes, d.dim, cus, false);
  Sections s(ws);
  w.dz = s.take<char>(n * w.width * size_of(d.dtype));
  w.sum = s.take<float>(w.pieces > 1 ? n * d.dim : 0);
  w.db_part = s.take<float>(w.logits.row_tiles * V);
  w.live = s.take<uint8_t>(n);
  w.input = row_work(d.dtype, n, G, d.dim, classes, true, s.base ? s.base + s.used : nullptr);
  s.used += w.input.bytes;
  w.sums = sum_work(d.dtype, n, G, classes, d.dim, s.base ? s.base + s.used : nullptr);
  w.bytes = s.used + w.sums.bytes;
  return w;
}

struct NarrowWork {
  NarrowPlan plan;
  float* pieces;
  int4* cuts;
  int64_t bytes;
};
NarrowWork narrow_work(const im_head_desc& d, void* ws) {
  NarrowWork w;
  w.plan = plan_narrow(d.n_rows, d.n_groups, d.dim, d.n_classes, compute_units());
  Sections s(ws);
  w.pieces = s.take<float>(2 * w.plan.parts * w.plan.piece);
  w.cuts = s.take<int4>(w.plan.parts > 0 ? d.n_groups : 0);
  if (w.plan.parts == 0) w.cuts = nullptr;
  w.bytes = s.used;
  return w;
}
bool narrow(const im_head_desc& d) { return narrow_supported(d.dtype, d.dim, d.n_classes); }
int64_t head_backward_bytes(const im_head_desc& d) {
  return narrow(d) ? narrow_work(d, nullptr).bytes : head_backward(d, nullptr).bytes;
}

}  // namespace

extern "C" {

im_status im_head_workspace(const im_head_desc* d, int32_t backward, int64_t* bytes) {
  LEARN_OK(check_head(d));
  LEARN_CHECK(bytes, "bytes is NULL");
  LEARN_CHECK(backward == 0 || backward == 1, "backward is 0 or 1");
  *bytes = d->n_rows == 0 && !backward ? 0 : (backward ? head_backward_bytes(*d) : head_forward(*d, nullptr).bytes);
  return IM_OK;
}

im_status im_head_forward(const im_head_desc* d, const int32_t* offsets, const void* h, const void* W, const float* b,
                          const uint32_t* valid, const int32_t* target, float* logp, float* entropy, float* lse,
                          void* ws, int64_t ws_bytes, int32_t* error, void* stream) {
  LEARN_OK(check_head(d));
  LEARN_OK(check_groups(d->n_groups, offsets));
  const int64_t e = size_of(d->dtype);
  LEARN_CHECK(stride_ok(d->ld_h, d->dim), "ld_h out of range");
  LEARN_CHECK(W && (d->n_rows == 0 || (h && target && logp)), "h, W, target or logp is NULL");
  LEARN_CHECK(aligned(h, e) && aligned(W, e) && aligned(b, 4) && aligned(valid, 4) && aligned(target, 4) &&
                  aligned(logp, 4) && aligned(entropy, 4) && aligned(lse, 4) && aligned(error, 4),
              "a pointer is not aligned to its elements");
  if (d->n_rows == 0) return IM_OK;
  const HeadForward w = head_forward(*d, ws);
  LEARN_OK(check_launch(w.plan));
  const int64_t n = d->n_rows, G = d->n_groups, k = d->dim, V = d->n_classes;
  LEARN_OK(check_areas({flat("offsets", offsets, 4 * (G + 1), false), matrix("h", h, n, k, d->ld_h, e, false),
                        flat("W", W, G * V * k * e, false), flat("b", b, 4 * G * V, false),
                        flat("valid", valid, 4 * n * ((V + 31) / 32), false), flat("target", target, 4 * n, false),
                        flat("logp", logp, 4 * n, true), flat("entropy", entropy, 4 * n, true),
                        flat("lse", lse, 4 * n, true), flat("workspace", ws, w.bytes, true),
                        flat("error", error, 4, true)}));
  LEARN_OK(check_work(ws, ws_bytes, w.bytes));
  RowArgs a = row_args(offsets, d->n_groups, d->n_rows, w.plan, error);
  a.K = d->dim;
  a.N = a.V = d->n_classes;
  a.words = (d->n_classes + 31) / 32;
  a.A = h;
  a.lda = d->ld_h;
  a.B = W;
  a.ldb = d->dim;
  a.b_group = (int64_t)d->dim * d->n_classes;
  a.bias = b;
  a.bias_group = d->n_classes;
  a.valid = valid;
  a.target = target;
  a.stats = w.stats;
  a.taken = w.taken;
  a.logp = logp;
  a.entropy = entropy;
  a.lse = lse;
  LEARN_HIP(launch_rows_product(a, d->dtype, w.plan.shape, kStats, (hipStream_t)stream));
  return IM_OK;
}

im_status im_head_backward(const im_head_desc* d, const int32_t* offsets, const void* h, const void* W, const float* b,
                           const uint32_t* valid, const int32_t* target, const float* lse, const float* entropy,
                           const float* dlogp, const float* dentropy, void* dh, void* dW, float* db, void* ws,
                           int64_t ws_bytes, int32_t* error, void* stream) {
  LEARN_OK(check_head(d));
  LEARN_OK(check_groups(d->n_groups, offsets));
  const int64_t e = size_of(d->dtype);
  const bool some = d->n_rows > 0;
  LEARN_CHECK(stride_ok(d->ld_h, d->dim) && (!dh || stride_ok(d->ld_dh, d->dim)), "ld_h or ld_dh out of range");
  LEARN_CHECK(!some || (h && W && target && lse && dlogp), "h, W, target, lse or dlogp is NULL");
  LEARN_CHECK(!some || !dentropy || entropy, "dentropy needs entropy");
  LEARN_CHECK(aligned(h, e) && aligned(W, e) && aligned(dh, e) && aligned(dW, e) && aligned(b, 4) && aligned(valid, 4) &&
                  aligned(target, 4) && aligned(lse, 4) && aligned(entropy, 4) && aligned(dlogp, 4) &&
                  aligned(dentropy, 4) && aligned(db, 4) && aligned(error, 4),
              "a pointer is not aligned to its elements");
  const int64_t V = d->n_classes;
  const auto check_outputs = [&](int64_t ws_need) {
    const int64_t n = d->n_rows, G = d->n_groups, k = d->dim;
    return check_areas({flat("offsets", offsets, 4 * (G + 1), false), matrix("h", h, n, k, d->ld_h, e, false),
                        flat("W", W, G * V * k * e, false), flat("b", b, 4 * G * V, false),
                        flat("valid", valid, 4 * n * ((V + 31) / 32), false), flat("target", target, 4 * n, false),
                        flat("lse", lse, 4 * n, false), flat("entropy", dentropy ? entropy : nullptr, 4 * n, false),
                        flat("dlogp", dlogp, 4 * n, false), flat("dentropy", dentropy, 4 * n, false),
                        matrix("dh", dh, n, k, d->ld_dh, e, true), flat("dW", dW, G * V * k * e, true),
                        flat("db", db, 4 * G * V, true), flat("workspace", ws, ws_need, true),
                        flat("error", error, 4, true)});
  };
  if (narrow(*d)) {
    const NarrowWork w = narrow_work(*d, ws);
    LEARN_OK(check_outputs(w.bytes));
    LEARN_OK(check_work(ws, ws_bytes, w.bytes));
    if (!dh && !dW && !db) return IM_OK;
    NarrowArgs a = {};
    a.offsets = offsets;
    a.G = d->n_groups;
    a.n = d->n_rows;
    a.d = d->dim;
    a.V = d->n_classes;
    a.words = (d->n_classes + 31) / 32;
    a.relu_in = d->relu_in;
    a.h = h;
    a.ld_h = d->ld_h;
    a.W = W;
    a.bias = b;
    a.valid = valid;
    a.target = target;
    a.lse = lse;
    a.entropy = entropy;
    a.dlogp = dlogp;
    a.dentropy = dentropy;
    a.dh = dh;
    a.ld_dh = d->ld_dh;
    a.dW = dW;
    a.db = db;
    a.pieces = w.pieces;
    a.cuts = w.cuts;
    a.piece = w.plan.piece;
    a.pitch = w.plan.pitch;
    a.granule = (int32_t)w.plan.granule;
    a.parts = (int32_t)w.plan.parts;
    a.error = error;
    LEARN_HIP(launch_narrow(a, (hipStream_t)stream));
    return IM_OK;
  }
  const HeadBackward w = head_backward(*d, ws);
  LEARN_OK(check_launch(w.logits));
  LEARN_OK(check_launch(w.input.plan));
  LEARN_OK(check_grid(w.sums.plan));
  LEARN_OK(check_outputs(w.bytes));
  LEARN_OK(check_work(ws, ws_bytes, w.bytes));
  if (!dh && !dW && !db) return IM_OK;
  const hipStream_t s = (hipStream_t)stream;
  for (int64_t piece = 0; piece < w.pieces; ++piece) {
    const int64_t c0 = piece * w.width, width = V - c0 < w.width ? V - c0 : w.width;
    const char* Wp = static_cast<const char*>(W) + c0 * d->dim * e;
    if (some) {
      RowArgs a = row_args(offsets, d->n_groups, d->n_rows, w.logits, error);
      a.col_tiles = (int32_t)((width + cols_per_tile(w.logits.shape) - 1) / cols_per_tile(w.logits.shape));
      a.K = d->dim;
      a.N = (int32_t)width;
      a.V = d->n_classes;
      a.col0 = (int32_t)c0;
      a.words = (d->n_classes + 31) / 32;
      a.A = h;
      a.lda = d->ld_h;
      a.B = Wp;
      a.ldb = d->dim;
      a.b_group = V * d->dim;
      a.bias = b;
      a.bias_group = V;
      a.C = w.dz;
      a.ldc = w.width;
      a.valid = valid;
      a.target = target;
      a.lse = const_cast<float*>(lse);
      a.entropy = const_cast<float*>(entropy);
      a.dlogp = dlogp;
      a.dentropy = dentropy;
      a.db_part = db ? w.db_part : nullptr;
      a.db_width = V;
      a.live = w.live;
      LEARN_HIP(launch_rows_product(a, d->dtype, w.logits.shape, kGradLogits, s));
    }
    if (dh && some) {
      RowArgs a = row_args(offsets, d->n_groups, d->n_rows, w.input.plan, error);
      a.part = w.input.part;
      if (a.split_k * (int64_t)(a.splits - 1) >= width) a.splits = (int32_t)((width + a.split_k - 1) / a.split_k);   // the last piece
      a.K = (int32_t)width;
      a.N = d->dim;
      a.A = w.dz;
      a.lda = w.width;
      a.B = Wp;
      a.ldb = d->dim;
      a.b_group = V * d->dim;
      a.C = dh;
      a.ldc = d->ld_dh;
      a.X = d->relu_in ? h : nullptr;
      a.ldx = d->ld_h;
      a.sum = w.pieces > 1 ? w.sum : nullptr;
      a.first = piece == 0;
      a.last = piece == w.pieces - 1;
      LEARN_HIP(launch_rows_product(a, d->dtype, w.input.plan.shape, kStoreInput, s));
    }
    if (dW) {
      SumArgs a = {};
      a.offsets = offsets;
      a.G = d->n_groups;
      a.n = d->n_rows;
      a.M = (int32_t)width;
      a.N = d->dim;
      a.P = w.dz;
      a.ldp = w.width;
      a.Q = h;
      a.ldq = d->ld_h;
      a.live = w.live;
      a.dW = static_cast<char*>(dW) + c0 * d->dim * e;
      a.w_group = V * d->dim;
      a.part = w.sums.part;
      a.cuts = w.sums.cuts;
      a.granule = (int32_t)w.sums.plan.granule;
      a.parts = (int32_t)w.sums.plan.parts;
      const int64_t tile = rows_per_sum(w.sums.plan.shape);
      a.row_tiles = (int32_t)((width + tile - 1) / tile);
      a.col_tiles = (int32_t)w.sums.plan.col_tiles;
      a.error = error;
      LEARN_HIP(launch_sums(a, d->dtype, w.sums.plan.shape, s));
    }
  }
  if (db)
    LEARN_HIP(launch_bias_sum(some ? offsets : nullptr, d->n_groups, d->n_rows, rows_per_tile(w.logits.shape), w.db_part, V, db, s));
  return IM_OK;
}

// ---- AdamW -------------------------------------------------------------------------

}  // extern "C"

namespace {

im_status check_tensor(const im_adamw_tensor& t, int bits, int grad_dtype, int i) {
  LEARN_CHECK(t.n >= 0, "tensor %d: n out of range", i);
  LEARN_CHECK(t.decay == 0 || t.decay == 1, "tensor %d: decay is 0 or 1", i);
  if (t.n == 0) return IM_OK;
  LEARN_CHECK(t.param && t.grad && t.m && t.v, "tensor %d: param, grad, m or v is NULL", i);
  LEARN_CHECK(bits == 32 || (t.m_scale && t.v_scale), "tensor %d: 8-bit states need m_scale and v_scale", i);
  LEARN_CHECK(bits == 8 || (!t.m_scale && !t.v_scale), "tensor %d: 32-bit states have no scales", i);
  LEARN_CHECK(aligned(t.param, 4) && aligned(t.grad, size_of(grad_dtype)) && aligned(t.copy, 2) &&
                  (bits == 8 || (aligned(t.m, 4) && aligned(t.v, 4))) && aligned(t.m_scale, 4) && aligned(t.v_scale, 4),
              "tensor %d: a pointer is not aligned to its elements", i);
  return IM_OK;
}

// Whether something that a step writes lies in another buffer of the step.
bool overlap(const std::vector<im_adamw_tensor>& list, int bits, int grad_dtype) {
  struct Span {
    uintptr_t at, end;
    bool written;
  };
  std::vector<Span> spans;
  const auto add = [&](const void* p, int64_t bytes, bool written) {
    if (p && bytes) spans.push_back(Span{(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written});
  };
  for (const im_adamw_tensor& t : list) {
    if (t.n == 0) continue;
    const int64_t state = bits == 32 ? 4 : 1, blocks = (t.n + IM_STATE_BLOCK - 1) / IM_STATE_BLOCK;
    add(t.param, 4 * t.n, true);
    add(t.grad, (int64_t)size_of(grad_dtype) * t.n, false);
    add(t.m, state * t.n, true);
    add(t.v, state * t.n, true);
    add(t.m_scale, 4 * blocks, true);
    add(t.v_scale, 4 * blocks, true);
    add(t.copy, 2 * t.n, true);
  }
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.at < b.at; });
  uintptr_t any = 0, written = 0;   // ends of what came before
  for (const Span& s : spans) {
    if (s.at < (s.written ? any : written)) return true;
    any = std::max(any, s.end);
    if (s.written) written = std::max(written, s.end);
  }
  return false;
}

template <typename T>
hipError_t upload(T** out, const std::vector<T>& from, hipStream_t s) {
  if (from.empty()) return hipSuccess;
  hipError_t e = hipMalloc(reinterpret_cast<void**>(out), from.size() * sizeof(T));
  if (e == hipSuccess) e = hipMemcpyAsync(*out, from.data(), from.size() * sizeof(T), hipMemcpyHostToDevice, s);
  return e;
}

void free_adamw(im_adamw* o) {
  (void)hipFree(o->table);
  (void)hipFree(o->tensors);
  (void)hipFree(o->done);
  delete o;
}

// The plan's device as the current one within a call.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    err = hipGetDevice(&was_);
    if (err == hipSuccess && was_ != device) {
      err = hipSetDevice(device);
      moved_ = err == hipSuccess;
    }
  }
  ~OnDevice() {
    if (moved_) (void)hipSetDevice(was_);
  }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
  hipError_t err;

 private:
  int was_ = 0;
  bool moved_ = false;
};

}  // namespace

extern "C" {

im_status im_adamw_create(const im_adamw_tensor* tensors, int32_t n_tensors, int32_t state_bits, int32_t grad_dtype,
                          void* stream, im_adamw** out) {
  LEARN_CHECK(out, "out is NULL");
  LEARN_CHECK(n_tensors >= 0 && n_tensors <= IM_MAX_TENSORS, "n_tensors out of range");
  LEARN_CHECK(n_tensors == 0 || tensors, "tensors is NULL");
  LEARN_CHECK(state_bits == 32 || state_bits == 8, "state_bits is 32 or 8");
  LEARN_CHECK(grad_dtype == IM_F32 || grad_dtype == IM_BF16, "grad_dtype out of range");
  int64_t all = 0;
  for (int i = 0; i < n_tensors; ++i) {
    LEARN_OK(check_tensor(tensors[i], state_bits, grad_dtype, i));
    LEARN_CHECK(tensors[i].n <= IM_MAX_ELEMENTS - all, "more than %lld elements", (long long)IM_MAX_ELEMENTS);
    all += tensors[i].n;
  }
  im_adamw* o = new (std::nothrow) im_adamw();
  if (!o) return fail(IM_ENOMEM, "out of host memory");
  hipError_t e = hipGetDevice(&o->device);
  try {
    std::vector<AdamwRun> runs;
    std::vector<im_adamw_tensor> list(tensors, tensors + n_tensors);
    if (overlap(list, state_bits, grad_dtype)) {
      free_adamw(o);
      return fail(IM_EINVAL, "tensors overlap");
    }
    for (int i = 0; i < n_tensors; ++i) {
      const im_adamw_tensor& t = list[i];
      const int64_t state = state_bits == 32 ? 16 : 4;
      const bool al = aligned(t.param, 16) && aligned(t.grad, grad_dtype == IM_BF16 ? 8 : 16) && aligned(t.m, state) &&
                      aligned(t.v, state) && aligned(t.copy, 8);
      for (int64_t at = 0; at < t.n; at += kRun) runs.push_back(AdamwRun{at, i, al ? 1 : 0});
    }
    o->bits = state_bits;
    o->grad_dtype = grad_dtype;
    o->runs = (int64_t)runs.size();
    // 2^26 elements, a block a run against blocks that share the runs, 8 a CU: 353 and 367 us
    // with 32-bit states, 224 and 220 us with 8-bit ones
    // (a launch has less than 2^32 threads)
    o->blocks = state_bits == 32 ? std::min<int64_t>(o->runs, 1 << 23) : 8 * (int64_t)compute_units();
    const hipStream_t s = (hipStream_t)stream;
    const std::vector<uint32_t> zero(1, 0);
    if (e == hipSuccess && o->runs > 0x7fffffff) e = hipErrorInvalidValue;
    if (e == hipSuccess) e = upload(&o->table, runs, s);
    if (e == hipSuccess) e = upload(&o->tensors, list, s);
    if (e == hipSuccess) e = upload(&o->done, zero, s);
    const hipError_t w = hipStreamSynchronize(s);   // the host arrays end with this scope
    if (e == hipSuccess) e = w;
  } catch (const std::bad_alloc&) {
    free_adamw(o);
    return fail(IM_ENOMEM, "out of host memory");
  }
  if (e != hipSuccess) {
    free_adamw(o);
    return fail(e == hipErrorOutOfMemory ? IM_ENOMEM : IM_EHIP, "im_adamw_create: %s", hipGetErrorString(e));
  }
  *out = o;
  return IM_OK;
}

im_status im_adamw_step(im_adamw* o, double lr, double beta1, double beta2, double eps, double weight_decay,
                        int64_t* step, const float* scale, void* stream) {
  LEARN_CHECK(o, "opt is NULL");
  LEARN_CHECK(step, "step is NULL");
  LEARN_CHECK(aligned(step, 8) && aligned(scale, 4), "a pointer is not aligned to its elements");
  LEARN_CHECK(lr >= 0 && eps >= 0 && weight_decay >= 0 && std::isfinite(lr) && std::isfinite(eps) && std::isfinite(weight_decay),
              "lr, eps and weight_decay must be finite and >= 0");
  LEARN_CHECK(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1, "betas must be in [0, 1)");
  AdamwArgs a = {};
  a.table = o->table;
  a.tensors = o->tensors;
  a.runs = o->runs;
  a.blocks = o->blocks;
  a.step = step;
  a.scale = scale;
  a.done = o->done;
  a.beta1 = beta1;
  a.beta2 = beta2;
  a.lr = (float)lr;
  a.beta1f = (float)beta1;
  a.omb1 = (float)(1.0 - beta1);
  a.beta2f = (float)beta2;
  a.omb2 = (float)(1.0 - beta2);
  a.eps = eps > 0 ? std::max((float)eps, FLT_MIN) : 0.f;   // subnormal: zero states would give 0 times infinity
  a.keep = (float)(1.0 - lr * weight_decay);
  const OnDevice on(o->device);
  LEARN_HIP(on.err);
  LEARN_HIP(launch_adamw(a, o->bits, o->grad_dtype, (hipStream_t)stream));
  return IM_OK;
}

void im_adamw_destroy(im_adamw* o) {
  if (!o) return;
  const OnDevice on(o->device);
  (void)hipDeviceSynchronize();
  free_adamw(o);
}

}  // extern "C"
