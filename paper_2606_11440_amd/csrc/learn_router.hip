// Routing to experts: scores of a row's logits, the choice of its best experts, their
// weights, and the gradient of the logits.
#include "learn_internal.h"
#include "learn_softmax.h"
#include "wave.h"

namespace im {
namespace learn {
namespace {

constexpr int kMostChoices = 4;   // choices of a lane: top_k is at most 32, and 8 lanes at least hold them

// e^x, off by less than 2 units: the product with log2 e is taken in two floats. x <= 0.
__device__ __forceinline__ float exp_near(float x) {
  constexpr float kLow = 1.925963033500e-8f;   // log2 e less its float
  const float y = fmaxf(x, -104.f);            // e^-104 is 0
  const float t = y * kLog2e, r = fmaf(y, kLow, fmaf(y, kLog2e, -t));
  return exp2_(t) * fmaf(r, kLn2, 1.f);
}

// Sum and largest of v over L neighbouring lanes (a power of two), the same in all of them.
template <int L, class F>
__device__ __forceinline__ float across(float v, F f) {
  if constexpr (L > 1) v = f(v, __builtin_bit_cast(float, xshfl<1>(__builtin_bit_cast(int32_t, v))));
  if constexpr (L > 2) v = f(v, __builtin_bit_cast(float, xshfl<2>(__builtin_bit_cast(int32_t, v))));
  if constexpr (L > 4) v = f(v, __builtin_bit_cast(float, xshfl<4>(__builtin_bit_cast(int32_t, v))));
  if constexpr (L > 8) v = f(v, __builtin_bit_cast(float, xshfl<8>(__builtin_bit_cast(int32_t, v))));
  if constexpr (L > 16) v = f(v, __builtin_bit_cast(float, xshfl<16>(__builtin_bit_cast(int32_t, v))));
  if constexpr (L > 32) v = f(v, __builtin_bit_cast(float, xshfl<32>(__builtin_bit_cast(int32_t, v))));
  return v;
}
template <int L>
__device__ __forceinline__ float sum_of(float v) {
  return across<L>(v, [](float a, float b) { return a + b; });
}
template <int L>
__device__ __forceinline__ float most_of(float v) {
  return across<L>(v, [](float a, float b) { return fmaxf(a, b); });
}

// The logit of expert j as it counts: -infinity where the expert is not valid (NaN too).
template <typename T>
__device__ __forceinline__ float logit(const RouterArgs& a, int64_t row, int j) {
  const float z = (float)static_cast<const T*>(a.z)[row * a.ld_z + j];
  const bool ok = !a.valid || ((a.valid[row * a.words + (j >> 5)] >> (j & 31)) & 1u);
  return ok && z > -INFINITY ? fminf(z, 3.4028234663852886e38f) : -INFINITY;
}

// Weights of a row's chosen experts, which L lanes hold: choice t L + l is lane l's t-th.
// top, total: largest logit of the row and its sum of exponentials (softmax without renorm).
// Sigmoids are divided by a common e^m where all are small, so that their shares do not
// depend on how small.
template <int L>
__device__ __forceinline__ void weigh(const RouterArgs& a, int score, const float (&z)[kMostChoices], float top,
                                      float total, float (&w)[kMostChoices]) {
  float m = -INFINITY;
#pragma unroll
  for (int t = 0; t < kMostChoices; ++t) m = fmaxf(m, z[t]);
  m = most_of<L>(m);
  const float ref = m == -INFINITY ? 0.f : m, below = fminf(ref, 0.f);
  float sum = 0.f;
#pragma unroll
  for (int t = 0; t < kMostChoices; ++t) {
    float v = 0.f;
    if (z[t] > -INFINITY) {
      if (score == IM_SIGMOID) {
        const float e = exp_near(-fabsf(z[t]));
        v = (z[t] < 0.f ? (a.renorm ? exp_near(z[t] - below) : e) : 1.f) / (1.f + e);
      } else {
        v = exp_near(z[t] - (a.renorm ? ref : top));
      }
    }
    w[t] = v;
    sum += v;
  }
  if (a.renorm) total = sum_of<L>(sum);
  else if (score == IM_SIGMOID) total = 1.f;
#pragma unroll
  for (int t = 0; t < kMostChoices; ++t) w[t] = z[t] > -INFINITY ? a.scale * (w[t] / total) : 0.f;
}

// ---- the choice in 64 bits ---------------------------------------------------

// What the wave's lanes wrote to LDS before, they read after (LDS serves a wave in order).
__device__ __forceinline__ void lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ double shfl_xor_f64(double v, int m) {
  return __builtin_bit_cast(double, shfl_xor(__builtin_bit_cast(int64_t, v), m));
}

// A row's choice by a whole wave, every c as it is defined. Lane l has experts 64 v + l; `keys` is LDS
// of the wave. choice[t]: the 64 t + l-th chosen expert (t < 1: top_k is at most 32), or -1.
template <typename T, int V>
__device__ int choose_exact(const RouterArgs& a, int score, int64_t row, double* keys) {
  const int lane = (int)threadIdx.x % 64;
  float z[V];
  double key[V], share[V];
  float top = -INFINITY;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int j = v * 64 + lane;
    z[v] = j < a.E ? logit<T>(a, row, j) : -INFINITY;
    top = fmaxf(top, z[v]);
  }
  const bool bias = a.bias != nullptr, sums = a.sets > 1 && a.best == 2;
#pragma unroll
  for (int v = 0; v < V; ++v) share[v] = 0.;
  if (bias || sums) {
    if (score == IM_SIGMOID) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const double e = exp(-fabs((double)z[v]));
        share[v] = (z[v] < 0.f ? e : 1.) / (1. + e);
      }
    } else {
      top = most_of<64>(top);
      const double ref = top == -INFINITY ? 0. : (double)top;
      double total = 0.;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        share[v] = exp((double)z[v] - ref);
        total += share[v];
      }
#pragma unroll
      for (int d = 1; d < 64; d *= 2) total += shfl_xor_f64(total, d);
#pragma unroll
      for (int v = 0; v < V; ++v) share[v] /= total;   // a row without a valid expert has none to choose
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int j = v * 64 + lane;
    key[v] = bias && j < a.E ? share[v] + (double)a.bias[j] : (double)z[v];
    if (!(z[v] > -INFINITY) || !(key[v] > -INFINITY)) key[v] = -INFINITY;   // NaN too
  }
  if (a.top_sets < a.sets) {
    const int each = a.E / a.sets;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int j = v * 64 + lane;
      if (j < a.E) keys[j] = !sums || bias || key[v] == -INFINITY ? key[v] : share[v];
    }
    lds_order();
    double value[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int s = v * 64 + lane;
      value[v] = -INFINITY;
      if (s >= a.sets) continue;
      double first = -INFINITY, second = -INFINITY;
      for (int i = 0; i < each; ++i) {
        const double x = keys[s * each + i];
        second = fmax(second, fmin(first, x));
        first = fmax(first, x);
      }
      value[v] = first;
      if (a.best == 2 && second > -INFINITY) value[v] += second;
    }
    lds_order();
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v * 64 + lane < a.sets) keys[v * 64 + lane] = value[v];
    lds_order();
    int rank[V];   // sets that come before the lane's
#pragma unroll
    for (int v = 0; v < V; ++v) rank[v] = 0;
    for (int s = 0; s < a.sets; ++s) {
      const double x = keys[s];
#pragma unroll
      for (int v = 0; v < V; ++v) rank[v] += x > value[v] || (x == value[v] && s < v * 64 + lane);
    }
    lds_order();
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v * 64 + lane < a.sets) keys[v * 64 + lane] = rank[v] < a.top_sets ? 1. : 0.;
    lds_order();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int j = v * 64 + lane;
      if (j < a.E && keys[j / each] == 0.) key[v] = -INFINITY;
    }
    lds_order();
  }
  int mine = -1;
  for (int c = 0; c < a.k; ++c) {
    double best = -INFINITY;
    int at = 1 << 30;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (key[v] > best) {
        best = key[v];
        at = v * 64 + lane;
      }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double x = shfl_xor_f64(best, d);
      const int i = shfl_xor(at, d);
      if (x > best || (x == best && i < at)) {
        best = x;
        at = i;
      }
    }
    if (!(best > -INFINITY)) break;   // nothing is left, in any lane
    if (lane == c) mine = at;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v * 64 + lane == at) key[v] = -INFINITY;
  }
  return mine;
}

template <typename T, int V>
__global__ __launch_bounds__(256) void router_kernel(const RouterArgs a, int score) {
  __shared__ double lds[4][V * 64];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  for (int64_t row = (int64_t)blockIdx.x * 4 + wave; row < a.n; row += (int64_t)gridDim.x * 4) {
  const int mine = choose_exact<T, V>(a, score, row, lds[wave]);
  float z[kMostChoices], w[kMostChoices], top = 0.f, total = 1.f;
#pragma unroll
  for (int t = 0; t < kMostChoices; ++t) z[t] = -INFINITY;
  if (lane < a.k && mine >= 0) z[0] = logit<T>(a, row, mine);
  if (score == IM_SOFTMAX && !a.renorm) {
    top = -INFINITY;
    for (int j = lane; j < a.E; j += 64) top = fmaxf(top, logit<T>(a, row, j));
    top = most_of<64>(top);
    top = top == -INFINITY ? 0.f : top;
    total = 0.f;
    for (int j = lane; j < a.E; j += 64) total += exp_near(logit<T>(a, row, j) - top);
    total = sum_of<64>(total);
  }
  weigh<64>(a, score, z, top, total, w);
  if (lane < a.k) {
    a.expert[row * a.k + lane] = mine;
    a.weight[row * a.k + lane] = w[0];
  }
  }
}

// ---- the gradient ---------------------------------------------------------------

// A row is L lanes' (64 / L rows a wave); lane l has experts 4 L (v / 4) + 4 l + v % 4.
template <typename T, int L, int V>
__global__ __launch_bounds__(256) void router_backward_kernel(const RouterArgs a, int score) {
  const int l = (int)threadIdx.x % L;
  constexpr int kRows = 256 / L;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.n; first += (int64_t)gridDim.x * kRows) {
  const int64_t at = first + (int)threadIdx.x / L, row = at < a.n ? at : a.n - 1;
  const bool in = at < a.n;   // the last block's other lanes follow the last row, and store nothing
  int e[kMostChoices];
  float z[kMostChoices], dw[kMostChoices], w[kMostChoices], d[kMostChoices], q[V];
  bool wrong = false;
#pragma unroll
  for (int t = 0; t < kMostChoices; ++t) {
    const int c = t * L + l;
    e[t] = -1;
    z[t] = -INFINITY;
    dw[t] = 0.f;
    if (c < a.k) {
      e[t] = a.expert[row * a.k + c];
      if (e[t] >= 0 && e[t] < a.E) z[t] = logit<T>(a, row, e[t]);
      wrong |= e[t] != -1 && z[t] == -INFINITY;
      if (z[t] > -INFINITY) dw[t] = a.dweight[row * a.k + c];
      else e[t] = -1;
    }
  }
  if (wrong && in && a.error) atomicOr(a.error, IM_ERR_ACTION);
  const bool dense = score == IM_SOFTMAX && !a.renorm;
  float top = 0.f, total = 1.f;
#pragma unroll
  for (int v = 0; v < V; ++v) q[v] = 0.f;
  if (dense) {
    top = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int j = v / 4 * 4 * L + 4 * l + v % 4;
      q[v] = j < a.E ? logit<T>(a, row, j) : -INFINITY;
      top = fmaxf(top, q[v]);
    }
    top = most_of<L>(top);
    top = top == -INFINITY ? 0.f : top;
    total = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      q[v] = exp_near(q[v] - top);
      total += q[v];
    }
    total = sum_of<L>(total);
    total = total > 0.f ? total : 1.f;
  }
  weigh<L>(a, score, z, top, total, w);
  float dot = 0.f;   // of weights and their gradients
#pragma unroll
  for (int t = 0; t < kMostChoices; ++t) dot += w[t] * dw[t];
  dot = sum_of<L>(dot);
  // scale q (dw - sum q dw) with w = scale q
  const float mean = a.renorm ? (a.scale != 0.f ? dot / a.scale : 0.f) : 0.f;
#pragma unroll
  for (int t = 0; t < kMostChoices; ++t) {
    d[t] = w[t] * (dw[t] - mean);
    if (score == IM_SIGMOID && z[t] > -INFINITY) {
      const float x = exp_near(-fabsf(z[t]));   // 1 - sigmoid
      d[t] *= (z[t] < 0.f ? 1.f : x) / (1.f + x);
    }
  }
  const float each = dense ? -dot / total : 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) q[v] *= each;
  for (int c = 0; c < a.k; ++c) {
    const int i = __shfl(c < L ? e[0] : (c < 2 * L ? e[1] : (c < 3 * L ? e[2] : e[3])), c % L, L);
    const float x = __shfl(c < L ? d[0] : (c < 2 * L ? d[1] : (c < 3 * L ? d[2] : d[3])), c % L, L);
#pragma unroll
    for (int v = 0; v < V; ++v) q[v] += v / 4 * 4 * L + 4 * l + v % 4 == i ? x : 0.f;
  }
  if (!in) continue;
  T* const to = static_cast<T*>(a.dz) + row * a.ld_dz;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int j = v / 4 * 4 * L + 4 * l + v % 4;
    if (j < a.E) to[j] = (T)q[v];
  }
  }
}

// a launch has less than 2^32 threads in a dimension: past this many blocks they take more rows each
unsigned blocks_of(int64_t n, int rows) {
  const int64_t blocks = (n + rows - 1) / rows, most = 1 << 20;
  return (unsigned)(blocks < most ? blocks : most);
}

template <typename T>
hipError_t forward(const RouterArgs& a, int score, hipStream_t s) {
  const dim3 grid(blocks_of(a.n, 4)), block(256);
  if (a.E <= 64) hipLaunchKernelGGL((router_kernel<T, 1>), grid, block, 0, s, a, score);
  else if (a.E <= 256) hipLaunchKernelGGL((router_kernel<T, 4>), grid, block, 0, s, a, score);
  else hipLaunchKernelGGL((router_kernel<T, 16>), grid, block, 0, s, a, score);
  return hipGetLastError();
}

template <typename T, int L, int V>
hipError_t backward_rows(const RouterArgs& a, int score, hipStream_t s) {
  hipLaunchKernelGGL((router_backward_kernel<T, L, V>), dim3(blocks_of(a.n, 256 / L)), dim3(256), 0, s, a, score);
  return hipGetLastError();
}
template <typename T>
hipError_t backward(const RouterArgs& a, int score, hipStream_t s) {
  if (a.E <= 32) return backward_rows<T, 8, 4>(a, score, s);
  if (a.E <= 64) return backward_rows<T, 8, 8>(a, score, s);
  if (a.E <= 128) return backward_rows<T, 8, 16>(a, score, s);
  if (a.E <= 256) return backward_rows<T, 16, 16>(a, score, s);
  if (a.E <= 512) return backward_rows<T, 32, 16>(a, score, s);
  return backward_rows<T, 64, 16>(a, score, s);
}

}  // namespace

hipError_t launch_router_forward(const RouterArgs& a, int dtype, int score, hipStream_t s) {
  return dtype == IM_BF16 ? forward<__bf16>(a, score, s) : forward<float>(a, score, s);
}
hipError_t launch_router_backward(const RouterArgs& a, int dtype, int score, hipStream_t s) {
  return dtype == IM_BF16 ? backward<__bf16>(a, score, s) : backward<float>(a, score, s);
}

}  // namespace learn
}  // namespace im
