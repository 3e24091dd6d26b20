// Host side of the learner's calls: errors, checks of arguments and areas, workspaces and
// the launch arguments that several operators share.
#pragma once
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <utility>

#include "learn_internal.h"

namespace im {
namespace learn {

extern thread_local char t_error[256];   // the calling thread's last failed call

__attribute__((format(printf, 2, 3))) inline im_status fail(im_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(t_error, sizeof(t_error), fmt, ap);
  va_end(ap);
  return s;
}

#define LEARN_HIP(call)                                                                              \
  do {                                                                                               \
    const hipError_t _e = (call);                                                                    \
    if (_e != hipSuccess)                                                                            \
      return fail(_e == hipErrorOutOfMemory ? IM_ENOMEM : IM_EHIP, "%s: %s", #call, hipGetErrorString(_e)); \
  } while (0)

#define LEARN_CHECK(cond, ...)                       \
  do {                                               \
    if (!(cond)) return fail(IM_EINVAL, __VA_ARGS__); \
  } while (0)

// Compute units of the current device (256 where the query fails).
inline int compute_units() {
  static int known[64];   // each device's is written once it is known, always with the same value
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 256;
  if (dev >= 0 && dev < 64 && __atomic_load_n(&known[dev], __ATOMIC_RELAXED) > 0)
    return __atomic_load_n(&known[dev], __ATOMIC_RELAXED);
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) return 256;
  if (dev >= 0 && dev < 64) __atomic_store_n(&known[dev], n, __ATOMIC_RELAXED);
  return n;
}

// Sections of a workspace, each 256-byte aligned.
struct Sections {
  char* base;
  int64_t used = 0;
  explicit Sections(void* p) : base(static_cast<char*>(p)) {}
  template <typename T>
  T* take(int64_t count) {
    T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
    used += (count * (int64_t)sizeof(T) + 255) & ~(int64_t)255;
    return p;
  }
};

inline int64_t size_of(int dtype) { return dtype == IM_BF16 ? 2 : 4; }
inline bool aligned(const void* p, int64_t a) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(a - 1)) == 0; }

inline bool stride_ok(int64_t ld, int64_t width) { return ld >= width && ld <= IM_MAX_LD; }

inline im_status check_groups(int32_t G, const int32_t* offsets) {
  LEARN_CHECK(offsets || G == 1, "offsets NULL needs n_groups = 1");
  LEARN_CHECK(aligned(offsets, 4), "offsets is not 4-byte aligned");
  return IM_OK;
}
inline im_status check_work(const void* ws, int64_t have, int64_t need) {
  LEARN_CHECK(have >= need && (need == 0 || ws), "workspace of %lld bytes, %lld needed", (long long)have, (long long)need);
  LEARN_CHECK(need == 0 || aligned(ws, 256), "workspace is not 256-byte aligned");
  return IM_OK;
}
inline im_status check_launch(const RowPlan& p) {
  if (p.row_tiles * p.col_tiles * p.splits >= 1 << 30) return fail(IM_EUNSUPPORTED, "2^30 tiles or more");
  return IM_OK;
}
inline im_status check_grid(const SumPlan& p) {
  // a launch has less than 2^32 threads in a dimension
  if (p.parts * p.row_tiles * p.col_tiles * threads_per_sum(p.shape) >= (int64_t)1 << 32)
    return fail(IM_EUNSUPPORTED, "2^32 threads or more");
  return IM_OK;
}
// Memory that a call reads or writes: rows of `width` bytes, `stride` bytes apart.
struct Area {
  const char* name;
  const void* at;
  int64_t rows, width, stride;
  bool written;
};
inline Area flat(const char* name, const void* p, int64_t bytes, bool written) { return Area{name, p, 1, bytes, bytes, written}; }
inline Area matrix(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t e, bool written) {
  if (rows > 1 && ld > cols) return Area{name, p, rows, cols * e, ld * e, written};
  return flat(name, p, rows * cols * e, written);
}

// Whether two areas share a byte. Views of the same rows that take different
// columns do not.
inline bool meet(const Area* a, const Area* b) {
  if (reinterpret_cast<uintptr_t>(a->at) > reinterpret_cast<uintptr_t>(b->at)) std::swap(a, b);
  if (!a->at || !b->at || a->rows * a->width == 0 || b->rows * b->width == 0) return false;
  const int64_t by = (int64_t)(reinterpret_cast<uintptr_t>(b->at) - reinterpret_cast<uintptr_t>(a->at));
  if (by >= (a->rows - 1) * a->stride + a->width) return false;
  if (a->rows == 1) return true;   // b begins in it
  if (b->rows == 1 || b->stride == a->stride) {   // b's first row: in a row of a, or behind it and into the next
    const int64_t row = by / a->stride, column = by % a->stride;
    return column < a->width || (column + b->width > a->stride && row + 1 < a->rows);
  }
  for (int64_t i = 0, j = 0; i < a->rows && j < b->rows;) {   // rows of both in their order
    const int64_t x = i * a->stride, y = by + j * b->stride;
    if (x + a->width <= y) ++i;
    else if (y + b->width <= x) ++j;
    else return true;
  }
  return false;
}

// Nothing that a call writes lies in anything else of the call: its blocks run side by side.
template <size_t N>
im_status check_areas(const Area (&areas)[N]) {
  for (size_t i = 0; i < N; ++i)
    for (size_t j = areas[i].written && areas[i].at ? 0 : N; j < N; ++j)
      if (i != j && meet(&areas[i], &areas[j])) return fail(IM_EINVAL, "%s overlaps %s", areas[i].name, areas[j].name);
  return IM_OK;
}

#define LEARN_OK(call)                       \
  do {                                       \
    const im_status _s = (call);             \
    if (_s != IM_OK) return _s;              \
  } while (0)

// ---- layers ------------------------------------------------------------------

inline im_status check_linear(const im_linear_desc* d) {
  LEARN_CHECK(d, "desc is NULL");
  LEARN_CHECK(d->n_groups >= 1 && d->n_groups <= IM_MAX_GROUPS, "n_groups out of range");
  LEARN_CHECK(d->n_rows >= 0 && d->n_rows <= IM_MAX_ROWS, "n_rows out of range");
  LEARN_CHECK(d->in_dim >= 1 && d->in_dim <= IM_MAX_DIM, "in_dim out of range");
  LEARN_CHECK(d->out_dim >= 1 && d->out_dim <= IM_MAX_DIM, "out_dim out of range");
  LEARN_CHECK(d->dtype == IM_F32 || d->dtype == IM_BF16, "dtype out of range");
  LEARN_CHECK((d->relu | d->relu_in) == 0 || (d->relu | d->relu_in) == 1, "relu and relu_in are 0 or 1");
  return IM_OK;
}

struct SumWork {
  SumPlan plan;
  float* part;
  int4* cuts;
  int64_t bytes;
};
// Plan and workspace of the sums over rows.
inline SumWork sum_work(int dtype, int64_t n, int64_t G, int64_t M, int64_t N, void* ws) {
  SumWork w;
  w.plan = plan_sums(dtype, n, G, M, N, compute_units());
  Sections s(ws);
  // one part cuts no group: it leaves no pieces, only which groups are empty
  const bool joined = w.plan.parts > 1 || (w.plan.parts == 1 && G > 1);
  w.part = s.take<float>(w.plan.parts > 1 ? 2 * w.plan.parts * w.plan.row_tiles * w.plan.col_tiles * w.plan.piece : 0);
  w.cuts = s.take<int4>(joined ? G : 0);
  if (!joined) w.cuts = nullptr;
  w.bytes = s.used;
  return w;
}

inline RowArgs row_args(const int32_t* offsets, int32_t G, int32_t n, const RowPlan& p, int32_t* error) {
  RowArgs a = {};
  a.offsets = offsets;
  a.G = G;
  a.n = n;
  a.row_tiles = (int32_t)p.row_tiles;
  a.col_tiles = (int32_t)p.col_tiles;
  a.error = error;
  a.cus = compute_units();
  a.splits = (int32_t)p.splits;
  a.split_k = (int32_t)p.split_k;
  return a;
}

// A row product with the workspace of its runs of k.
struct RowWork {
  RowPlan plan;
  float* part;
  int64_t bytes;
};
inline RowWork row_work(int dtype, int64_t n, int64_t G, int64_t N, int64_t K, bool may_split, void* ws) {
  RowWork w;
  w.plan = plan_rows(dtype, n, G, N, K, compute_units(), may_split);
  Sections s(ws);
  w.part = s.take<float>(w.plan.splits > 1 ? w.plan.splits * n * N : 0);
  w.bytes = s.used;
  return w;
}
inline RowWork linear_forward(const im_linear_desc& d, void* ws) {
  return row_work(d.dtype, d.n_rows, d.n_groups, d.out_dim, d.in_dim, true, ws);
}
struct LinearBackward {
  RowWork input;
  SumWork sums;
  int64_t bytes;
};
inline LinearBackward linear_backward(const im_linear_desc& d, void* ws) {
  LinearBackward w;
  w.input = row_work(d.dtype, d.n_rows, d.n_groups, d.in_dim, d.out_dim, true, ws);
  w.sums = sum_work(d.dtype, d.n_rows, d.n_groups, d.out_dim, d.in_dim,
                    ws ? static_cast<char*>(ws) + w.input.bytes : nullptr);
  w.bytes = w.input.bytes + w.sums.bytes;
  return w;
}

}  // namespace learn
}  // namespace im
