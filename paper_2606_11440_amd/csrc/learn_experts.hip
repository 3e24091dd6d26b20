// C ABI of the operators around experts and of rows in 8 bits: checks of arguments, launches.
#include <cmath>

#include "learn_host.h"

using namespace im::learn;

namespace {

// ---- routing -------------------------------------------------------------------

im_status check_router(const im_router_desc* d) {
  LEARN_CHECK(d, "desc is NULL");
  LEARN_CHECK(d->n_rows >= 0 && d->n_rows <= IM_MAX_ROWS, "n_rows out of range");
  LEARN_CHECK(d->n_experts >= 1 && d->n_experts <= IM_MAX_GROUPS, "n_experts out of range");
  LEARN_CHECK(d->dtype == IM_F32 || d->dtype == IM_BF16, "dtype out of range");
  LEARN_CHECK(d->score == IM_SOFTMAX || d->score == IM_SIGMOID, "score out of range");
  LEARN_CHECK(d->renorm == 0 || d->renorm == 1, "renorm is 0 or 1");
  LEARN_CHECK(std::isfinite(d->scale), "scale is not finite");
  LEARN_CHECK(d->top_k >= 1 && d->top_k <= IM_MAX_TOP_K && d->top_k <= d->n_experts, "top_k out of range");
  LEARN_CHECK(stride_ok(d->ld_z, d->n_experts), "ld_z out of range");
  return IM_OK;
}

RouterArgs router_args(const im_router_desc& d, const void* z, const uint32_t* valid) {
  RouterArgs a = {};
  a.n = d.n_rows;
  a.E = d.n_experts;
  a.k = d.top_k;
  a.sets = d.n_sets;
  a.top_sets = d.top_sets;
  a.best = d.set_best;
  a.renorm = d.renorm;
  a.scale = d.scale;
  a.z = z;
  a.ld_z = d.ld_z;
  a.valid = valid;
  a.words = (d.n_experts + 31) / 32;
  a.cus = compute_units();
  return a;
}

// ---- rows to experts and back -----------------------------------------------------

im_status check_pairs(const im_dispatch_desc* d) {
  LEARN_CHECK(d, "desc is NULL");
  LEARN_CHECK(d->n_rows >= 0 && d->n_rows <= IM_MAX_ROWS, "n_rows out of range");
  LEARN_CHECK(d->top_k >= 1 && d->top_k <= IM_MAX_TOP_K, "top_k out of range");
  LEARN_CHECK((int64_t)d->n_rows * d->top_k <= IM_MAX_ROWS, "n_rows top_k out of range");
  return IM_OK;
}
im_status check_plan(const im_dispatch_desc* d) {
  LEARN_OK(check_pairs(d));
  LEARN_CHECK(d->n_experts >= 1 && d->n_experts <= IM_MAX_GROUPS, "n_experts out of range");
  return IM_OK;
}
im_status check_exchange(const im_dispatch_desc* d, bool codes) {
  LEARN_OK(check_pairs(d));
  LEARN_CHECK(d->n_slots >= 0 && d->n_slots <= IM_MAX_ROWS, "n_slots out of range");
  LEARN_CHECK(d->dim >= 1 && d->dim <= IM_MAX_DIM, "dim out of range");
  LEARN_CHECK(d->dtype == IM_F32 || d->dtype == IM_BF16 || (codes && d->dtype == IM_CODES), "dtype out of range");
  LEARN_CHECK(stride_ok(d->ld_row, d->dim), "ld_row out of range");
  LEARN_CHECK(stride_ok(d->ld_slot, d->dim), "ld_slot out of range");
  return IM_OK;
}

struct PlanWork {
  PlanArgs args;
  int64_t bytes;
};
PlanWork plan_work(const im_dispatch_desc& d, void* ws) {
  PlanWork w = {};
  PlanArgs& a = w.args;
  a.pairs = (int64_t)d.n_rows * d.top_k;
  a.E = d.n_experts;
  a.blocks = (int32_t)plan_blocks(a.pairs, compute_units(), a.each);
  Sections s(ws);
  a.count = a.blocks > 1 ? s.take<int32_t>((int64_t)a.blocks * a.E) : nullptr;
  w.bytes = s.used;
  return w;
}

int64_t element(int dtype) { return dtype == IM_CODES ? 1 : size_of(dtype); }

ExchangeArgs exchange_args(const im_dispatch_desc& d, const int32_t* slot, int32_t* error) {
  ExchangeArgs a = {};
  a.n = d.n_rows;
  a.k = d.top_k;
  a.n_slots = d.n_slots;
  a.dim = d.dim;
  a.slot = slot;
  a.error = error;
  return a;
}

// Sums of slots' rows: of dispatch_backward and combine_forward.
im_status sum_slots(const im_dispatch_desc* d, const char* from_name, const void* from, const int32_t* slot,
                    const float* weight, const char* to_name, void* to, int32_t* error, void* stream) {
  const int64_t n = d->n_rows, k = d->dim, e = element(d->dtype);
  LEARN_CHECK(aligned(from, e) && aligned(to, e) && aligned(slot, 4) && aligned(weight, 4) && aligned(error, 4),
              "a pointer is not aligned to its elements");
  LEARN_CHECK(n == 0 || (slot && to && (from || d->n_slots == 0)), "slot, %s or %s is NULL", from_name, to_name);
  LEARN_OK(check_areas({matrix(from_name, from, d->n_slots, k, d->ld_slot, e, false),
                        flat("slot", slot, 4 * n * d->top_k, false), flat("weight", weight, 4 * n * d->top_k, false),
                        matrix(to_name, to, n, k, d->ld_row, e, true), flat("error", error, 4, true)}));
  if (n == 0) return IM_OK;
  ExchangeArgs a = exchange_args(*d, slot, error);
  a.weight = weight;
  a.from = from;
  a.ld_from = d->ld_slot;
  a.to = to;
  a.ld_to = d->ld_row;
  LEARN_HIP(launch_gather(a, d->dtype, (hipStream_t)stream));
  return IM_OK;
}

// ---- rows in 8 bits ------------------------------------------------------------------

im_status check_rows(const im_rows_desc* d) {
  LEARN_CHECK(d, "desc is NULL");
  LEARN_CHECK(d->n_rows >= 0 && d->n_rows <= IM_MAX_ROWS, "n_rows out of range");
  LEARN_CHECK(d->dim >= 1 && d->dim <= IM_MAX_DIM, "dim out of range");
  LEARN_CHECK(d->dtype == IM_F32 || d->dtype == IM_BF16, "dtype out of range");
  LEARN_CHECK(d->keep == 0 || d->keep == 1, "keep is 0 or 1");
  LEARN_CHECK(stride_ok(d->ld_x, d->dim) && stride_ok(d->ld_codes, d->dim), "ld_x or ld_codes out of range");
  return IM_OK;
}
im_status check_packed(const im_rows_desc* d, const void* x, const int8_t* codes, const float* scale, bool pack) {
  LEARN_OK(check_rows(d));
  const int64_t n = d->n_rows, e = size_of(d->dtype);
  LEARN_CHECK(n == 0 || (x && codes && scale), "x, codes or scale is NULL");
  LEARN_CHECK(aligned(x, e) && aligned(scale, 4), "a pointer is not aligned to its elements");
  return check_areas({matrix("x", x, n, d->dim, d->ld_x, e, !pack), matrix("codes", codes, n, d->dim, d->ld_codes, 1, pack),
                      flat("scale", scale, 4 * n, pack)});
}

RowWork packed_forward(const im_linear_desc& d, void* ws) {
  RowWork w;
  w.plan = plan_packed(d.n_rows, d.n_groups, d.out_dim, d.in_dim, compute_units());
  Sections s(ws);
  w.part = s.take<float>(w.plan.splits > 1 ? w.plan.splits * d.n_rows * d.out_dim : 0);
  w.bytes = s.used;
  return w;
}

}  // namespace

extern "C" {

im_status im_router_forward(const im_router_desc* d, const void* z, const float* bias, const uint32_t* valid,
                            int32_t* expert, float* weight, void* stream) {
  LEARN_OK(check_router(d));
  LEARN_CHECK(d->n_sets >= 1 && d->n_sets <= d->n_experts && d->n_experts % d->n_sets == 0, "n_sets does not divide n_experts");
  LEARN_CHECK(d->top_sets >= 1 && d->top_sets <= d->n_sets, "top_sets out of range");
  LEARN_CHECK(d->set_best == 1 || d->set_best == 2, "set_best is 1 or 2");
  LEARN_CHECK(d->top_k <= d->n_experts / d->n_sets * d->top_sets, "top_k is more than top_sets sets have");
  const int64_t n = d->n_rows, E = d->n_experts, e = size_of(d->dtype);
  LEARN_CHECK(n == 0 || (z && expert && weight), "z, expert or weight is NULL");
  LEARN_CHECK(aligned(z, e) && aligned(bias, 4) && aligned(valid, 4) && aligned(expert, 4) && aligned(weight, 4),
              "a pointer is not aligned to its elements");
  LEARN_OK(check_areas({matrix("z", z, n, E, d->ld_z, e, false), flat("bias", bias, 4 * E, false),
                        flat("valid", valid, 4 * n * ((E + 31) / 32), false),
                        flat("expert", expert, 4 * n * d->top_k, true), flat("weight", weight, 4 * n * d->top_k, true)}));
  if (n == 0) return IM_OK;
  RouterArgs a = router_args(*d, z, valid);
  a.bias = bias;
  a.expert = expert;
  a.weight = weight;
  LEARN_HIP(launch_router_forward(a, d->dtype, d->score, (hipStream_t)stream));
  return IM_OK;
}

im_status im_router_backward(const im_router_desc* d, const void* z, const uint32_t* valid, const int32_t* expert,
                             const float* dweight, void* dz, int32_t* error, void* stream) {
  LEARN_OK(check_router(d));
  LEARN_CHECK(stride_ok(d->ld_dz, d->n_experts), "ld_dz out of range");
  const int64_t n = d->n_rows, E = d->n_experts, e = size_of(d->dtype);
  LEARN_CHECK(n == 0 || (z && expert && dweight && dz), "z, expert, dweight or dz is NULL");
  LEARN_CHECK(aligned(z, e) && aligned(dz, e) && aligned(valid, 4) && aligned(expert, 4) && aligned(dweight, 4) &&
                  aligned(error, 4),
              "a pointer is not aligned to its elements");
  LEARN_OK(check_areas({matrix("z", z, n, E, d->ld_z, e, false), flat("valid", valid, 4 * n * ((E + 31) / 32), false),
                        flat("expert", expert, 4 * n * d->top_k, false),
                        flat("dweight", dweight, 4 * n * d->top_k, false), matrix("dz", dz, n, E, d->ld_dz, e, true),
                        flat("error", error, 4, true)}));
  if (n == 0) return IM_OK;
  RouterArgs a = router_args(*d, z, valid);
  a.expert = const_cast<int32_t*>(expert);   // read only
  a.dweight = dweight;
  a.dz = dz;
  a.ld_dz = d->ld_dz;
  a.error = error;
  LEARN_HIP(launch_router_backward(a, d->dtype, d->score, (hipStream_t)stream));
  return IM_OK;
}

im_status im_dispatch_workspace(const im_dispatch_desc* d, int64_t* bytes) {
  LEARN_OK(check_plan(d));
  LEARN_CHECK(bytes, "bytes is NULL");
  *bytes = plan_work(*d, nullptr).bytes;
  return IM_OK;
}

im_status im_dispatch_plan(const im_dispatch_desc* d, const int32_t* expert, int32_t* offsets, int32_t* slot, void* ws,
                           int64_t ws_bytes, int32_t* error, void* stream) {
  LEARN_OK(check_plan(d));
  LEARN_CHECK(offsets && (d->n_rows == 0 || (expert && slot)), "expert, offsets or slot is NULL");
  LEARN_CHECK(aligned(expert, 4) && aligned(offsets, 4) && aligned(slot, 4) && aligned(error, 4),
              "a pointer is not aligned to its elements");
  PlanWork w = plan_work(*d, ws);
  LEARN_OK(check_areas({flat("expert", expert, 4 * w.args.pairs, false),
                        flat("offsets", offsets, 4 * ((int64_t)d->n_experts + 1), true),
                        flat("slot", slot, 4 * w.args.pairs, true), flat("workspace", ws, w.bytes, true),
                        flat("error", error, 4, true)}));
  LEARN_OK(check_work(ws, ws_bytes, w.bytes));
  w.args.expert = expert;
  w.args.offsets = offsets;
  w.args.slot = slot;
  w.args.error = error;
  LEARN_HIP(launch_dispatch_plan(w.args, (hipStream_t)stream));
  return IM_OK;
}

im_status im_dispatch_forward(const im_dispatch_desc* d, const void* x, const int32_t* slot, void* xs, int32_t* error,
                              void* stream) {
  LEARN_OK(check_exchange(d, true));
  const int64_t n = d->n_rows, k = d->dim, e = element(d->dtype);
  LEARN_CHECK(n == 0 || (x && slot && (xs || d->n_slots == 0)), "x, slot or xs is NULL");
  LEARN_CHECK(aligned(x, e) && aligned(xs, e) && aligned(slot, 4) && aligned(error, 4),
              "a pointer is not aligned to its elements");
  LEARN_OK(check_areas({matrix("x", x, n, k, d->ld_row, e, false), flat("slot", slot, 4 * n * d->top_k, false),
                        matrix("xs", xs, d->n_slots, k, d->ld_slot, e, true), flat("error", error, 4, true)}));
  if (n == 0) return IM_OK;
  ExchangeArgs a = exchange_args(*d, slot, error);
  a.from = x;
  a.ld_from = d->ld_row;
  a.to = xs;
  a.ld_to = d->ld_slot;
  LEARN_HIP(launch_send(a, d->dtype, (hipStream_t)stream));
  return IM_OK;
}

im_status im_dispatch_backward(const im_dispatch_desc* d, const void* dxs, const int32_t* slot, void* dx, int32_t* error,
                               void* stream) {
  LEARN_OK(check_exchange(d, false));
  return sum_slots(d, "dxs", dxs, slot, nullptr, "dx", dx, error, stream);
}

im_status im_combine_forward(const im_dispatch_desc* d, const void* ys, const int32_t* slot, const float* weight, void* y,
                             int32_t* error, void* stream) {
  LEARN_OK(check_exchange(d, false));
  LEARN_CHECK(d->n_rows == 0 || weight, "weight is NULL");
  return sum_slots(d, "ys", ys, slot, weight, "y", y, error, stream);
}

im_status im_combine_backward(const im_dispatch_desc* d, const void* dy, const void* ys, const int32_t* slot,
                              const float* weight, void* dys, float* dweight, int32_t* error, void* stream) {
  LEARN_OK(check_exchange(d, false));
  const int64_t n = d->n_rows, k = d->dim, e = element(d->dtype), m = d->n_slots;
  LEARN_CHECK(!dys || stride_ok(d->ld_dslot, d->dim), "ld_dslot out of range");
  LEARN_CHECK(n == 0 || (dy && slot), "dy or slot is NULL");
  LEARN_CHECK(n == 0 || !dys || weight, "dys needs weight");
  LEARN_CHECK(n == 0 || !dweight || ys || m == 0, "dweight needs ys");
  LEARN_CHECK(aligned(dy, e) && aligned(ys, e) && aligned(dys, e) && aligned(slot, 4) && aligned(weight, 4) &&
                  aligned(dweight, 4) && aligned(error, 4),
              "a pointer is not aligned to its elements");
  LEARN_OK(check_areas({matrix("dy", dy, n, k, d->ld_row, e, false),
                        matrix("ys", dweight ? ys : nullptr, m, k, d->ld_slot, e, false),
                        flat("slot", slot, 4 * n * d->top_k, false),
                        flat("weight", dys ? weight : nullptr, 4 * n * d->top_k, false),
                        matrix("dys", dys, m, k, d->ld_dslot, e, true), flat("dweight", dweight, 4 * n * d->top_k, true),
                        flat("error", error, 4, true)}));
  if (n == 0 || (!dys && !dweight)) return IM_OK;
  ExchangeArgs a = exchange_args(*d, slot, error);
  a.weight = weight;
  a.from = dy;
  a.ld_from = d->ld_row;
  a.to = dys;
  a.ld_to = d->ld_dslot;
  a.ys = ys;
  a.ld_ys = d->ld_slot;
  a.dweight = dweight;
  LEARN_HIP(launch_combine_backward(a, d->dtype, (hipStream_t)stream));
  return IM_OK;
}

im_status im_rows_pack(const im_rows_desc* d, const void* x, int8_t* codes, float* scale, void* stream) {
  LEARN_OK(check_packed(d, x, codes, scale, true));
  if (d->n_rows == 0) return IM_OK;
  PackArgs a = {};
  a.n = d->n_rows;
  a.dim = d->dim;
  a.keep = d->keep;
  a.x = x;
  a.ld_x = d->ld_x;
  a.codes = codes;
  a.ld_codes = d->ld_codes;
  a.scale = scale;
  LEARN_HIP(launch_pack(a, d->dtype, (hipStream_t)stream));
  return IM_OK;
}

im_status im_rows_unpack(const im_rows_desc* d, const int8_t* codes, const float* scale, void* x, void* stream) {
  LEARN_OK(check_packed(d, x, codes, scale, false));
  if (d->n_rows == 0) return IM_OK;
  PackArgs a = {};
  a.n = d->n_rows;
  a.dim = d->dim;
  a.codes = const_cast<int8_t*>(codes);   // read only
  a.ld_codes = d->ld_codes;
  a.scale = const_cast<float*>(scale);
  a.out = x;
  a.ld_x = d->ld_x;
  LEARN_HIP(launch_unpack(a, d->dtype, (hipStream_t)stream));
  return IM_OK;
}

im_status im_linear_workspace_packed(const im_linear_desc* d, int32_t backward, int64_t* bytes) {
  LEARN_OK(check_linear(d));
  LEARN_CHECK(bytes, "bytes is NULL");
  LEARN_CHECK(backward == 0 || backward == 1, "backward is 0 or 1");
  *bytes = backward ? linear_backward(*d, nullptr).bytes : packed_forward(*d, nullptr).bytes;
  return IM_OK;
}

im_status im_linear_forward_packed(const im_linear_desc* d, const int32_t* offsets, const int8_t* x, const float* x_scale,
                                   const int8_t* W, const float* W_scale, const float* b, void* y, void* ws,
                                   int64_t ws_bytes, int32_t* error, void* stream) {
  LEARN_OK(check_linear(d));
  LEARN_OK(check_groups(d->n_groups, offsets));
  const int64_t e = size_of(d->dtype);
  LEARN_CHECK(stride_ok(d->ld_x, d->in_dim) && stride_ok(d->ld_y, d->out_dim), "ld_x or ld_y out of range");
  LEARN_CHECK(W && W_scale && (d->n_rows == 0 || (x && x_scale && y)), "x, x_scale, W, W_scale or y is NULL");
  LEARN_CHECK(aligned(x_scale, 4) && aligned(W_scale, 4) && aligned(y, e) && aligned(b, 4) && aligned(error, 4),
              "a pointer is not aligned to its elements");
  const RowWork w = packed_forward(*d, ws);
  const int64_t n = d->n_rows, G = d->n_groups, k = d->in_dim, m = d->out_dim;
  if (n > 0) {
    LEARN_OK(check_launch(w.plan));
    LEARN_OK(check_areas({flat("offsets", offsets, 4 * (G + 1), false), matrix("x", x, n, k, d->ld_x, 1, false),
                          flat("x_scale", x_scale, 4 * n, false), flat("W", W, G * m * k, false),
                          flat("W_scale", W_scale, 4 * G * m, false), flat("b", b, 4 * G * m, false),
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
  LEARN_HIP(launch_packed_product(a, PackedScales{x_scale, W_scale}, d->dtype, w.plan.shape, (hipStream_t)stream));
  return IM_OK;
}

im_status im_linear_backward_packed(const im_linear_desc* d, const int32_t* offsets, const void* dy, const int8_t* x,
                                    const float* x_scale, const void* W, void* dx, void* dW, float* db, void* ws,
                                    int64_t ws_bytes, int32_t* error, void* stream) {
  LEARN_OK(check_linear(d));
  LEARN_OK(check_groups(d->n_groups, offsets));
  const int64_t e = size_of(d->dtype);
  const bool some = d->n_rows > 0, mask = dx && d->relu_in;
  LEARN_CHECK(!some || dy, "dy is NULL");
  LEARN_CHECK(stride_ok(d->ld_y, d->out_dim), "ld_y out of range");
  LEARN_CHECK(!dx || !some || (W && stride_ok(d->ld_dx, d->in_dim)), "dx needs W and a valid ld_dx");
  LEARN_CHECK(!some || !(dW || mask) || (x && stride_ok(d->ld_x, d->in_dim)),
              "dW, and dx with relu_in, need x and a valid ld_x");
  LEARN_CHECK(!some || !dW || x_scale, "dW needs x_scale");
  LEARN_CHECK(aligned(dy, e) && aligned(x_scale, 4) && aligned(W, e) && aligned(dx, e) && aligned(dW, e) &&
                  aligned(db, 4) && aligned(error, 4),
              "a pointer is not aligned to its elements");
  const LinearBackward w = linear_backward(*d, ws);
  LEARN_OK(check_launch(w.input.plan));
  LEARN_OK(check_grid(w.sums.plan));
  const int64_t n = d->n_rows, G = d->n_groups, k = d->in_dim, m = d->out_dim;
  LEARN_OK(check_areas({flat("offsets", offsets, 4 * (G + 1), false), matrix("dy", dy, n, m, d->ld_y, e, false),
                        matrix("x", dW || mask ? x : nullptr, n, k, d->ld_x, 1, false),
                        flat("x_scale", dW ? x_scale : nullptr, 4 * n, false),
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
    a.X = mask ? x : nullptr;
    a.ldx = d->ld_x;
    a.first = a.last = 1;
    LEARN_HIP(launch_rows_product(a, d->dtype, w.input.plan.shape, mask ? kStoreInputCodes : kStoreInput, (hipStream_t)stream));
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
    a.Q = dW ? static_cast<const void*>(x) : dy;
    a.ldq = dW ? d->ld_x : d->ld_y;
    a.scale = dW ? x_scale : nullptr;
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

}  // extern "C"
