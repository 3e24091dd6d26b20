// Routing to experts: scores of a row's logits, the choice of its best experts, their
// weights, and the gradient of the logits.
//
// A row's experts are spread over few lanes (16 a lane where there are as many), so that most of the
// work is within lanes and a wave has several rows. What bounds it is the number of operations: 262144 rows of
// 64 experts in 8 sets, fp32, sigmoid and bias, 46 us (75 MB: 14 us at the rate of a copy), of some 1170
// instructions for 16 rows; 8 lanes of 8 experts took 61 us, a wave a row in 64 bits throughout 332. The gradient
// of 100003 rows of 193 experts, bf16, dense softmax: 30 us (85 MB: 16 us); adding the choices' parts
// to every lane's experts in registers took 39.
#include "learn_internal.h"
#include "learn_softmax.h"
#include "learn_tile.h"
#include "wave.h"

namespace im {
namespace learn {
namespace {

constexpr float kLargest = 3.4028234663852886e38f;

// Choices of a lane where a row is L lanes': top_k is at most 32.
template <int L>
constexpr int kMostChoices = L >= 32 ? 1 : 32 / L;

// e^x, off by less than 2 units: the product with log2 e is taken in two floats. x <= 0.
__device__ __forceinline__ float exp_near(float x) {
  constexpr float kLow = 1.925963033500e-8f;   // log2 e less its float
  const float y = fmaxf(x, -104.f);            // e^-104 is 0
  const float t = y * kLog2e, r = fmaf(y, kLow, fmaf(y, kLog2e, -t));
  return exp2_(t) * fmaf(r, kLn2, 1.f);
}

// f over L neighbouring lanes (a power of two), the same in all of them. A step's partners already
// hold the same within their half, so a mirror of the lanes serves as well as an exchange.
template <int L, class F>
__device__ __forceinline__ int32_t across(int32_t v, F f) {
  if constexpr (L > 1) v = f(v, dpp<0xB1>(v));     // quad_perm [1,0,3,2]
  if constexpr (L > 2) v = f(v, dpp<0x4E>(v));     // quad_perm [2,3,0,1]
  if constexpr (L > 4) v = f(v, dpp<0x141>(v));    // half-row mirror
  if constexpr (L > 8) v = f(v, dpp<0x140>(v));    // row mirror
  if constexpr (L > 16) v = f(v, xshfl<16>(v));
  if constexpr (L > 32) v = f(v, xshfl<32>(v));
  return v;
}
template <int L>
__device__ __forceinline__ int32_t most_of(int32_t v) {
  return across<L>(v, [](int32_t a, int32_t b) { return max(a, b); });
}
template <int L>
__device__ __forceinline__ int32_t least_of(int32_t v) {
  return across<L>(v, [](int32_t a, int32_t b) { return min(a, b); });
}
template <int L>
__device__ __forceinline__ float sum_of(float v) {
  return __builtin_bit_cast(float, across<L>(__builtin_bit_cast(int32_t, v), [](int32_t a, int32_t b) {
    return __builtin_bit_cast(int32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
  }));
}

// Floats as integers that order as they do (no NaN; -0 is not +0), and back.
__device__ __forceinline__ int32_t ordered(float x) {
  const int32_t b = __builtin_bit_cast(int32_t, x);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float from_ordered(int32_t b) {
  return __builtin_bit_cast(float, b ^ ((b >> 31) & 0x7fffffff));
}
constexpr int32_t kNone = (int32_t)0x807fffff;   // of -infinity
template <int L>
__device__ __forceinline__ float most_of(float v) {
  return from_ordered(most_of<L>(ordered(v)));
}

// The logit of expert j as it counts: -infinity where the expert is not valid (NaN too).
template <typename T>
__device__ __forceinline__ float logit(const RouterArgs& a, int64_t row, int j) {
  const float z = (float)static_cast<const T*>(a.z)[row * a.ld_z + j];
  const bool ok = !a.valid || ((a.valid[row * a.words + (j >> 5)] >> (j & 31)) & 1u);
  return ok ? fminf(fmaxf(z, -INFINITY), kLargest) : -INFINITY;   // NaN: -infinity
}

// Weights of a row's chosen experts, which L lanes hold: choice t L + l is lane l's t-th.
// top, total: largest logit of the row and its sum of exponentials (softmax without renorm).
// Sigmoids are divided by a common e^m where all are small, so that their shares do not
// depend on how small.
template <int L, int C>
__device__ __forceinline__ void weigh(const RouterArgs& a, int score, const float (&z)[C], float top, float total,
                                      float (&w)[C]) {
  float m = -INFINITY;
#pragma unroll
  for (int t = 0; t < C; ++t) m = fmaxf(m, z[t]);
  m = most_of<L>(m);
  const float ref = m == -INFINITY ? 0.f : m, below = fminf(ref, 0.f);
  float sum = 0.f;
#pragma unroll
  for (int t = 0; t < C; ++t) {
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
  for (int t = 0; t < C; ++t) w[t] = z[t] > -INFINITY ? a.scale * (w[t] / total) : 0.f;
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
// of the wave, 64 V doubles. Lane l gets the row's l-th chosen expert, or -1.
template <typename T, int V>
__device__ __forceinline__ int choose_exact(const RouterArgs& a, int score, int64_t row, double* keys) {
  const int lane = fresh_thread() % 64;   // nothing of this is worked out ahead, in registers of the rows that need none
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

// A row by a whole wave: choice in 64 bits, weights, stores.
template <typename T, int V>
__device__ __forceinline__ void route_exact(const RouterArgs& a, int score, int64_t row, double* keys) {
  const int lane = fresh_thread() % 64;
  const int mine = choose_exact<T, V>(a, score, row, keys);
  float z[1] = {mine >= 0 ? logit<T>(a, row, mine) : -INFINITY}, w[1], top = 0.f, total = 1.f;
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

// ---- the choice in 32 bits --------------------------------------------------------

// Four neighbouring logits from expert j on, as `logit` takes them.
template <typename T>
__device__ __forceinline__ void logits4(const RouterArgs& a, int64_t row, int j, float (&z)[4]) {
  const T* from = static_cast<const T*>(a.z) + row * a.ld_z + j;
  uint32_t ok = ~0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) z[i] = -INFINITY;
  if (j >= a.E) return;
  if (a.valid) ok = a.valid[row * a.words + (j >> 5)] >> (j & 31);
  if (j + 4 <= a.E) {
    typedef T four __attribute__((ext_vector_type(4)));
    typedef four any __attribute__((aligned(sizeof(T))));
    const four v = *reinterpret_cast<const any*>(from);
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = (float)v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (j + i < a.E) z[i] = (float)from[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    z[i] = fminf(fmaxf(z[i], -INFINITY), kLargest);   // NaN: -infinity
  if (a.valid) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {   // its bit as a mask of all: a bit select
      const uint32_t m = (uint32_t)((int32_t)(ok << (31 - i)) >> 31);
      z[i] = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, z[i]) & m) | (0xff800000u & ~m));
    }
  }
}

// The number of element v of lane l is place(v) + 4 l.
template <int L>
__device__ __forceinline__ constexpr int place(int v) {
  return v / 4 * 4 * L + v % 4;
}

// The largest first: Batcher's network of compare-exchanges, two integer operations each.
template <int V>
struct Network {
  int count, low[V * 8], high[V * 8];
  constexpr Network() : count(0), low{}, high{} {
    for (int p = 1; p < V; p *= 2)
      for (int k = p; k >= 1; k /= 2)
        for (int j = k % p; j + k < V; j += 2 * k)
          for (int i = 0; i < k && i + j + k < V; ++i)
            if ((i + j) / (2 * p) == (i + j + k) / (2 * p)) {
              low[count] = i + j;
              high[count++] = i + j + k;
            }
  }
};
template <int V, int I = 0>
__device__ __forceinline__ void sort_down(int32_t (&x)[V]) {
  constexpr Network<V> net;
  if constexpr (I < net.count) {
    constexpr int i = net.low[I], j = net.high[I];
    const int32_t a = x[i], b = x[j];
    x[i] = max(a, b);
    x[j] = min(a, b);
    sort_down<V, I + 1>(x);
  }
}

// Drops the first of a lane's sorted keys where it was taken (a bit select a key).
template <int V>
__device__ __forceinline__ void take_front(int32_t (&x)[V], bool taken, int32_t none) {
  const int32_t m = taken ? -1 : 0;
#pragma unroll
  for (int u = 0; u < V; ++u) x[u] = (x[u] & ~m) | ((u + 1 < V ? x[u + 1] : none) & m);
}

// Best and second of four.
__device__ __forceinline__ void two_best(const float (&x)[4], float& first, float& second) {
  const float a = fmaxf(x[0], x[1]), b = fminf(x[0], x[1]), c = fmaxf(x[2], x[3]), d = fminf(x[2], x[3]);
  first = fmaxf(a, c);
  second = fmaxf(fminf(a, c), fmaxf(b, d));
}
template <int CTRL>
__device__ __forceinline__ void two_best_with(float& first, float& second, bool both) {
  const float f = __builtin_bit_cast(float, dpp<CTRL>(__builtin_bit_cast(int32_t, first)));
  if (both) {
    const float s = __builtin_bit_cast(float, dpp<CTRL>(__builtin_bit_cast(int32_t, second)));
    second = fmaxf(fminf(first, f), fmaxf(second, s));
  }
  first = fmaxf(first, f);
}

// A row is L lanes' (64 / L rows a wave); lane l has V experts, four neighbours at a time, and C choices.
// SCORES: the choice goes by scores (a bias, or sets by the sum of their best), which fp32 knows
// up to `near` only. Where two that decide something (neighbours in the order of the chosen and the
// first that is not, or the last set taken and the first left) are no further apart, the
// row is done again in 64 bits: one row of some thousand, and every row with scores that are equal there. The
// order is then found on integers whose low bits are the number within the lane. Otherwise the choice goes by the logits themselves, exactly.
// SETS: 0 none, 1 sets of 4, 8, .. experts within the lanes' fours, 2 any.
template <typename T, int L, int V, int C, bool SCORES, int SETS>
__global__ __launch_bounds__(256) void router_kernel(const RouterArgs a, int score) {
  constexpr int kRows = 64 / L, kWide = L * V < 64 ? 1 : L * V / 64;
  constexpr int kPitch = L * V + 4;   // floats of a row
  constexpr int kLds = kRows * kPitch * 4 > kWide * 512 ? kRows * kPitch * 4 : kWide * 512;
  __shared__ __attribute__((aligned(16))) char lds[4][kLds];
  const int wave = threadIdx.x / 64, l0 = threadIdx.x % L;
  const int each = a.E / a.sets;
  const bool pairs = a.best == 2;
  float bias[SCORES ? V : 1];
  if constexpr (SCORES) {
#pragma unroll
    for (int v = 0; v < V; ++v) bias[v] = a.bias && place<L>(v) + 4 * l0 < a.E ? a.bias[place<L>(v) + 4 * l0] : 0.f;
  }
  for (int64_t first = ((int64_t)blockIdx.x * 4 + wave) * kRows; first < a.n; first += (int64_t)gridDim.x * 4 * kRows) {
    const int lane = fresh_thread() % 64, l = lane % L, r = lane / L;
    float* const mine = reinterpret_cast<float*>(lds[wave]) + r * kPitch;   // the row's LDS
    const bool in = first + r < a.n;   // the last wave's other lanes follow the last row, and store nothing
    const int64_t row = in ? first + r : a.n - 1;
    float key[V];
#pragma unroll
    for (int v = 0; v < V; v += 4) {
      float z[4];
      logits4<T>(a, row, place<L>(v) + 4 * l, z);
#pragma unroll
      for (int i = 0; i < 4; ++i) key[v + i] = z[i];
    }
    float top = 0.f, total = 1.f, near = 0.f;
    const bool softmax_sum = score == IM_SOFTMAX && (SCORES || !a.renorm);
    if (SCORES || softmax_sum) {
      top = key[0];
#pragma unroll
      for (int v = 1; v < V; ++v) top = fmaxf(top, key[v]);
      top = most_of<L>(top);
      top = top == -INFINITY ? 0.f : top;
    }
    if constexpr (!SCORES) {
      if (softmax_sum) {
        total = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) total += exp_near(key[v] - top);
        total = sum_of<L>(total);
      }
    } else {
      float most;   // the largest score
      if (score == IM_SOFTMAX) {
        total = 0.f;
        float e[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          e[v] = exp_near(key[v] - top);
          total += e[v];
        }
        total = sum_of<L>(total);
        most = 1.f / fmaxf(total, 1.f);
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = key[v] > -INFINITY ? e[v] * most : -INFINITY;
        // the sum of the exponentials by lanes is off by 24 2^-24 of itself (which counts by the shares'
        // difference), each of two shares by 5 units and |z - top| 2^-24 e^(z - top) of the largest
        near = most * 0x1p-17f;
      } else {
        most = __builtin_amdgcn_rcpf(1.f + exp_(-top));
        float least = key[0];
#pragma unroll
        for (int v = 1; v < V; ++v) least = fminf(least, key[v]);
        uint32_t out = 0;   // experts that are not valid, where there are any
        if (ballot(least == -INFINITY) != 0) {
#pragma unroll
          for (int v = 0; v < V; ++v) out |= key[v] == -INFINITY ? 1u << v : 0u;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = __builtin_amdgcn_rcpf(1.f + exp_(-key[v]));
        if (ballot(out != 0) != 0) {
#pragma unroll
          for (int v = 0; v < V; ++v) key[v] = (out >> v) & 1u ? -INFINITY : key[v];
        }
        // the exponential is off by (1.25 |z| + 2) 2^-24 of itself, which counts by the score times
        // (1 - score); the sum and the reciprocal add 3 2^-24 of the score; both for two scores. Below the normal
        // floats the reciprocal gives 0: 2^-126 more of each.
        near = most * (0x1p-20f + 0x1p-21f * fmaxf(-top, 0.f)) + 0x1p-124f;
      }
      if (a.bias) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          key[v] = fmaxf(key[v] + bias[v], -INFINITY);   // NaN: -infinity
        }
      }
    }
    bool unsure = false;   // the row's, the same in its lanes
    if constexpr (SETS != 0) {
      const bool sums = SCORES && pairs;
      float taken = INFINITY, left = -INFINITY, large = 0.f;   // large: of what was added up, for its rounding
      lds_order();
      if constexpr (SETS == 1) {   // a set is `span` neighbouring lanes' four
        const int shift = __builtin_ctz(each / 4), span = 1 << shift, rows4 = L >> shift;   // sets of a four of all lanes
        float value[V / 4];
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
          const float x[4] = {key[4 * q], key[4 * q + 1], key[4 * q + 2], key[4 * q + 3]};
          float best, second;
          two_best(x, best, second);
          if (span > 1) two_best_with<0xB1>(best, second, sums);
          if (span > 2) two_best_with<0x4E>(best, second, sums);
          if (L > 4 && span > 4) two_best_with<0x141>(best, second, sums);
          if (L > 8 && span > 8) two_best_with<0x140>(best, second, sums);
          value[q] = sums && second > -INFINITY ? best + second : best;
          if (best > -INFINITY) large = fmaxf(large, fabsf(best) + fabsf(value[q] - best));
          const int s = q * rows4 + (l >> shift);
          if (s < a.sets) mine[s] = value[q];
          else value[q] = -INFINITY;
        }
        if (l < 4) mine[a.sets + l] = -INFINITY;   // the last four are read whole
        lds_order();
        // sets that come before the lane's; by scores those of a larger value, and of equal ones all are taken: where
        // they are too many then, the row is unsure
        int rank[V / 4], count = 0;
#pragma unroll
        for (int q = 0; q < V / 4; ++q) rank[q] = 0;
#pragma unroll 2
        for (int s = 0; s < a.sets; s += 4) {
          const f32x4 o = *reinterpret_cast<const f32x4*>(mine + s);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < V / 4; ++q) {
              rank[q] += o[i] > value[q];
              if constexpr (!SCORES) rank[q] += o[i] == value[q] && s + i < q * rows4 + (l >> shift);
            }
        }
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
          const bool chosen = rank[q] < a.top_sets;
          taken = chosen ? fminf(taken, value[q]) : taken;
          left = chosen ? left : fmaxf(left, value[q]);
          if constexpr (SCORES) count += chosen && value[q] > -INFINITY;
#pragma unroll
          for (int i = 0; i < 4; ++i) key[4 * q + i] = chosen ? key[4 * q + i] : -INFINITY;
        }
        if constexpr (SCORES)   // each set counts in its lanes
          unsure = across<L>(count, [](int32_t a, int32_t b) { return a + b; }) > a.top_sets << shift;
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (place<L>(v) + 4 * l < a.E) mine[place<L>(v) + 4 * l] = key[v];
        lds_order();
        float value[V];
        for (int i = 0; i * L < a.sets; ++i) {
          const int s = i * L + l;
          float best = -INFINITY, second = -INFINITY;
          if (s < a.sets)
            for (int j = 0; j < each; ++j) {
              const float x = mine[s * each + j];
              second = fmaxf(second, fminf(best, x));
              best = fmaxf(best, x);
            }
          const float x = sums && second > -INFINITY ? best + second : best;
          if (best > -INFINITY) large = fmaxf(large, fabsf(best) + fabsf(x - best));
#pragma unroll
          for (int v = 0; v < V; ++v) value[v] = v == i ? x : value[v];
        }
        lds_order();
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (v * L + l < a.sets) mine[v * L + l] = value[v];
        lds_order();
        uint32_t chosen = 0;
        for (int i = 0; i * L < a.sets; ++i) {
          float x = 0.f;
#pragma unroll
          for (int v = 0; v < V; ++v) x = v == i ? value[v] : x;
          int rank = 0;
          for (int s = 0; s < a.sets; ++s) {
            const float o = mine[s];
            rank += o > x || (o == x && s < i * L + l);
          }
          if (i * L + l < a.sets) {
            chosen |= rank < a.top_sets ? 1u << i : 0u;
            if (rank < a.top_sets) taken = fminf(taken, x);
            else left = fmaxf(left, x);
          }
        }
        lds_order();
        for (int i = 0; i * L < a.sets; ++i)
          if (i * L + l < a.sets) mine[i * L + l] = (chosen >> i) & 1u ? 1.f : 0.f;
        lds_order();
        const float inverse = 1.f / (float)each;
#pragma unroll
        for (int v = 0; v < V; ++v) {   // numbers below 1024: the product of a half more is exact enough
          const int s = (int)(((float)(place<L>(v) + 4 * l) + 0.5f) * inverse);
          key[v] = mine[s < a.sets ? s : a.sets - 1] == 0.f ? -INFINITY : key[v];
        }
      }
      if constexpr (SCORES) {   // a sum of two is off by twice as much
        taken = -most_of<L>(-taken);
        left = most_of<L>(left);
        unsure |= left > -INFINITY && !(taken - left > 3.f * near + most_of<L>(large) * 0x1p-21f);
      }
    }
    // The keys as integers in their order. Scores' low bits become the number within the lane, and the
    // lower half of a bf16 logit what tells the lower index: such keys are sorted within the lane,
    // and each choice takes one from a lane's front. An infinite one counts as the largest float, which no bf16 number
    // is: the factor of 1 + 2^-23 takes that to infinity, and of others changes the lower half only. fp32 logits are
    // looked through.
    constexpr bool kSorted = SCORES || sizeof(T) == 2;
    int32_t at[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (SCORES) at[v] = (ordered(key[v]) & ~(V - 1)) | (V - 1 - v);   // of -infinity: kNone at most
      else if constexpr (kSorted) at[v] = (ordered(fmaf(key[v], 1.f + 0x1p-23f, 0.f)) & ~0xffff) | (0xffff - place<L>(v) - 4 * l);
      else at[v] = ordered(key[v] + 0.f);   // -0 as +0
    }
    if constexpr (kSorted) sort_down<V>(at);
    int choice[C];
    float before = INFINITY, apart = INFINITY, size = 0.f;   // least distance, largest magnitude
#pragma unroll
    for (int t = 0; t < C; ++t) choice[t] = -1;
    for (int c = 0; c <= a.k; ++c) {
      if (!SCORES && c == a.k) break;
      int32_t best = at[0];
      if constexpr (!kSorted) {
#pragma unroll
        for (int v = 1; v < V; ++v) best = max(best, at[v]);
      }
      const int32_t mine_best = best;
      best = most_of<L>(best);
      int j;
      if constexpr (SCORES) {
        // without the place, whose bits would count as up to V - 1 units more: a lower bound, so that what lies between
        // two is too large by as much at most. NaN where none is left, which counts in neither; a key of infinity
        // makes the size infinite and the row unsure.
        const float value = from_ordered(best & ~(V - 1));
        if (c > 0) apart = fminf(apart, before - value);
        size = fmaxf(size, fabsf(value));
        before = value;
        if (c == a.k) break;
        const int v = V - 1 - (best & (V - 1));
        const int own = mine_best == best ? (v >> 2) * 4 * L + (v & 3) + 4 * l : 1 << 30;
        j = least_of<L>(own);   // an equal one of another lane stays: the row is unsure then
        take_front<V>(at, own == j, kNone);
        j = best > kNone ? j : -1;
      } else if constexpr (kSorted) {
        j = best >= (kNone & ~0xffff) + 0x10000 ? 0xffff - (best & 0xffff) : -1;
        take_front<V>(at, mine_best == best, kNone & ~0xffff);   // no two are equal
      } else {
        j = 1 << 30;   // the lowest that has it
#pragma unroll
        for (int v = V - 1; v >= 0; --v) j = at[v] == best ? place<L>(v) : j;
        j = least_of<L>(j + 4 * l);
#pragma unroll
        for (int v = 0; v < V; ++v) at[v] = j - 4 * l == place<L>(v) ? kNone : at[v];
        j = best != kNone ? j : -1;
      }
#pragma unroll
      for (int t = 0; t < C; ++t) choice[t] = c == t * L + l ? j : choice[t];
    }
    // a sum with a bias is rounded to 2^-24 of itself, and its low bits are taken as zeros
    if constexpr (SCORES) unsure |= !(apart > near + (0x1p-22f + V * 0x1p-23f) * size);
    float z[C], w[C];
#pragma unroll
    for (int t = 0; t < C; ++t)
      z[t] = choice[t] >= 0 ? fminf((float)static_cast<const T*>(a.z)[row * a.ld_z + choice[t]], kLargest) : -INFINITY;
    weigh<L>(a, score, z, top, total, w);
#pragma unroll
    for (int t = 0; t < C; ++t)
      if (in && t * L + l < a.k && !unsure) {
        a.expert[row * a.k + t * L + l] = choice[t];
        a.weight[row * a.k + t * L + l] = w[t];
      }
    if constexpr (SCORES) {
      uint64_t again = ballot(unsure && in);
      while (again) {   // row by row, by the whole wave
        const int g = __builtin_ctzll(again) / L;
        lds_order();
        route_exact<T, kWide>(a, score, first + g, reinterpret_cast<double*>(lds[wave]));
        lds_order();
        again &= ~((L == 64 ? ~0ull : (1ull << (L % 64)) - 1) << (g * L));
      }
    }
  }
}

// ---- the gradient ---------------------------------------------------------------

// A row is L lanes' (64 / L rows a wave); lane l has experts 4 L (v / 4) + 4 l + v % 4.
// C choices a lane.
template <typename T, int L, int V, int C>
__global__ __launch_bounds__(256) void router_backward_kernel(const RouterArgs a, int score) {
  __shared__ __attribute__((aligned(16))) float lds[4][64 * V];
  const int l = (int)threadIdx.x % L;
  constexpr int kRows = 256 / L;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.n; first += (int64_t)gridDim.x * kRows) {
    const int64_t at = first + (int)threadIdx.x / L, row = at < a.n ? at : a.n - 1;
    const bool in = at < a.n;   // the last block's other lanes follow the last row, and store nothing
    int e[C];
    float z[C], dw[C], w[C], d[C], q[V];
    bool wrong = false;
#pragma unroll
    for (int t = 0; t < C; ++t) {
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
      for (int v = 0; v < V; v += 4) {
        float x[4];
        logits4<T>(a, row, place<L>(v) + 4 * l, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          q[v + i] = x[i];
          top = fmaxf(top, x[i]);
        }
      }
      top = most_of<L>(top);
      top = top == -INFINITY ? 0.f : top;
      total = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        // of bf16 logits the gradient is rounded to 2^-8: an exponential off by |z - top| 2^-23 will do
        q[v] = sizeof(T) == 2 ? exp_(q[v] - top) : exp_near(q[v] - top);
        total += q[v];
      }
      total = sum_of<L>(total);
      total = total > 0.f ? total : 1.f;
    }
    weigh<L>(a, score, z, top, total, w);
    float dot = 0.f;   // of weights and their gradients
#pragma unroll
    for (int t = 0; t < C; ++t) dot += w[t] * dw[t];
    dot = sum_of<L>(dot);
    // scale q (dw - sum q dw) with w = scale q
    const float mean = a.renorm ? (a.scale != 0.f ? dot / a.scale : 0.f) : 0.f;
#pragma unroll
    for (int t = 0; t < C; ++t) {
      d[t] = w[t] * (dw[t] - mean);
      if (score == IM_SIGMOID && z[t] > -INFINITY) {
        const float x = exp_near(-fabsf(z[t]));   // 1 - sigmoid
        d[t] *= (z[t] < 0.f ? 1.f : x) / (1.f + x);
      }
    }
    const float each = dense ? -dot / total : 0.f;
    // no zero times NaN or infinity where the expert is not valid
    const bool odd = !(fabsf(each) <= kLargest);
    if (ballot(odd) != 0) {
#pragma unroll
      for (int v = 0; v < V; ++v) q[v] = q[v] == 0.f ? 0.f : q[v] * each;
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) q[v] *= each;
    }
    // The choices' parts are added in LDS: a row's listed experts are as a rule no two the same, which
    // each place's last writer tells. Where they are, they are added in their order, one by one.
    float* const mine = lds[threadIdx.x / 64] + ((int)threadIdx.x % 64) / L * (L * V);
    lds_order();
#pragma unroll
    for (int t = 0; t < C; ++t)
      if (e[t] >= 0) mine[e[t]] = __builtin_bit_cast(float, t * L + l);
    lds_order();
    bool twice = false;
#pragma unroll
    for (int t = 0; t < C; ++t) twice |= e[t] >= 0 && __builtin_bit_cast(int, mine[e[t]]) != t * L + l;
    lds_order();
    if (ballot(twice) != 0) {
      for (int c = 0; c < a.k; ++c) {
        int ec = e[0];
        float dc = d[0];
#pragma unroll
        for (int t = 1; t < C; ++t) {
          ec = c / L == t ? e[t] : ec;
          dc = c / L == t ? d[t] : dc;
        }
        const int i = __shfl(ec, c % L, L);
        const float x = __shfl(dc, c % L, L);
#pragma unroll
        for (int v = 0; v < V; ++v) q[v] += i - 4 * l == place<L>(v) ? x : 0.f;
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; v += 4)
        *reinterpret_cast<f32x4*>(mine + place<L>(v) + 4 * l) = f32x4{q[v], q[v + 1], q[v + 2], q[v + 3]};
      lds_order();
#pragma unroll
      for (int t = 0; t < C; ++t)
        if (e[t] >= 0) mine[e[t]] += d[t];
      lds_order();
#pragma unroll
      for (int v = 0; v < V; v += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(mine + place<L>(v) + 4 * l);
#pragma unroll
        for (int i = 0; i < 4; ++i) q[v + i] = x[i];
      }
    }
    if (!in) continue;
    T* const to = static_cast<T*>(a.dz) + row * a.ld_dz;
#pragma unroll
    for (int v = 0; v < V; v += 4) {
      const int j = place<L>(v) + 4 * l;
      typedef T four __attribute__((ext_vector_type(4)));
      typedef four any __attribute__((aligned(sizeof(T))));
      four o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = (T)q[v + i];
      if (j + 4 <= a.E) {
        *reinterpret_cast<any*>(to + j) = o;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (j + i < a.E) to[j + i] = o[i];
      }
    }
  }
}

// a launch has less than 2^32 threads in a dimension: past this many blocks they take more rows each
unsigned blocks_of(int64_t n, int rows) {
  const int64_t blocks = (n + rows - 1) / rows, most = 1 << 20;
  return (unsigned)(blocks < most ? blocks : most);
}

template <typename T, int L, int V, int C, bool SCORES>
void forward_sets(const RouterArgs& a, int score, const dim3& grid, hipStream_t s) {
  const int each = a.E / a.sets;
  const dim3 block(256);
  if (a.top_sets == a.sets)
    hipLaunchKernelGGL((router_kernel<T, L, V, C, SCORES, 0>), grid, block, 0, s, a, score);
  else if (L <= 16 && (each & (each - 1)) == 0 && each >= 4 && each <= 4 * L)
    hipLaunchKernelGGL((router_kernel<T, L, V, C, SCORES, 1>), grid, block, 0, s, a, score);
  else   // of one kernel for any number of choices
    hipLaunchKernelGGL((router_kernel<T, L, V, kMostChoices<L>, SCORES, 2>), grid, block, 0, s, a, score);
}
template <typename T, int L, int V>
hipError_t forward_rows(const RouterArgs& a, int score, hipStream_t s) {
  const bool scores = a.bias || (a.top_sets < a.sets && a.best == 2);
  // blocks that share the rows: what a wave works out of the sets and biases serves several rows
  const int64_t blocks = ((int64_t)a.n + 256 / L - 1) / (256 / L), most = (int64_t)a.cus * 8;
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
  if (a.k <= L) {
    if (scores) forward_sets<T, L, V, 1, true>(a, score, grid, s);
    else forward_sets<T, L, V, 1, false>(a, score, grid, s);
  } else {
    if (scores) forward_sets<T, L, V, kMostChoices<L>, true>(a, score, grid, s);
    else forward_sets<T, L, V, kMostChoices<L>, false>(a, score, grid, s);
  }
  return hipGetLastError();
}
template <typename T>
hipError_t forward(const RouterArgs& a, int score, hipStream_t s) {
  if (a.E <= 16) return forward_rows<T, 4, 4>(a, score, s);
  if (a.E <= 32) return forward_rows<T, 4, 8>(a, score, s);
  if (a.E <= 64) return forward_rows<T, 4, 16>(a, score, s);
  if (a.E <= 128) return forward_rows<T, 8, 16>(a, score, s);
  if (a.E <= 256) return forward_rows<T, 16, 16>(a, score, s);
  if (a.E <= 512) return forward_rows<T, 32, 16>(a, score, s);
  return forward_rows<T, 64, 16>(a, score, s);
}

template <typename T, int L, int V>
hipError_t backward_rows(const RouterArgs& a, int score, hipStream_t s) {
  const dim3 grid(blocks_of(a.n, 256 / L)), block(256);
  if (a.k <= L) hipLaunchKernelGGL((router_backward_kernel<T, L, V, 1>), grid, block, 0, s, a, score);
  else hipLaunchKernelGGL((router_backward_kernel<T, L, V, kMostChoices<L>>), grid, block, 0, s, a, score);
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
