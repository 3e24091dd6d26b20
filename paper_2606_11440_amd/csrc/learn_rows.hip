// Products of grouped rows with their group's weights, and what follows them
// in registers: the layers (bias, ReLU), the gradient of a layer's input (the
// ReLU before it) and the softmax head (statistics, gradient of the logits).
#include <type_traits>

#include "learn_internal.h"
#include "learn_tile.h"

namespace im {
namespace learn {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float exp_(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// kVec neighbouring values of a row, of which `left` exist (kVec or more: all).
template <typename T>
struct Run {
  static constexpr int N = kVec<T>;
  float v[N];
  __device__ __forceinline__ void load(const T* p, int left) {
    if (left >= N) {
      const u32x4 x = load16(p);
      T e[N];
      __builtin_memcpy(e, &x, 16);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = (float)e[i];
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = i < left ? (float)p[i] : 0.f;
    }
  }
  __device__ __forceinline__ void store(T* p, int left) const {
    T e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = (T)v[i];
    if (left >= N) {
      u32x4 x;
      __builtin_memcpy(&x, e, 16);
      *reinterpret_cast<u32x4_any*>(p) = x;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < left) p[i] = e[i];
    }
  }
};
__device__ __forceinline__ f32x4 load4(const float* p, int left) {
  typedef f32x4 any __attribute__((aligned(4)));
  if (left >= 4) return *reinterpret_cast<const any*>(p);
  f32x4 v;
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = r < left ? p[r] : 0.f;
  return v;
}
__device__ __forceinline__ void store4(float* p, f32x4 v, int left) {
  typedef f32x4 any __attribute__((aligned(4)));
  if (left >= 4) {
    *reinterpret_cast<any*>(p) = v;
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r < left) p[r] = v[r];
  }
}

// Passes a block's results through LDS to runs of a row: f(row of the tile,
// column of the tile, run). A fragment's own layout would store 32 bytes of 16
// rows at a time; here a wave stores whole lines. 16 WM rows at a time, through
// two buffers in turn, so that one barrier does for each. A thread keeps its column.
template <typename T, class S, class F>
__device__ __forceinline__ void by_rows(const f32x4 (&acc)[S::MI][S::NJ], char* lds, F f) {
  constexpr int kPitch = S::BN * 4 + 16, kRows = S::WM * 16, kAcross = S::BN / kVec<T>;
  static_assert(S::NT % kAcross == 0 && kRows * kAcross % S::NT == 0, "a thread keeps its column");
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, wm = wave / S::WN, wn = wave % S::WN;
  const int c = ((int)threadIdx.x % kAcross) * kVec<T>;
#pragma unroll
  for (int i = 0; i < S::MI; ++i) {
    char* buf = lds + (i & 1) * kRows * kPitch;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
      *reinterpret_cast<f32x4*>(buf + (wm * 16 + lane % 16) * kPitch + ((wn * S::NJ + j) * 16 + (lane / 16) * 4) * 4) =
          acc[i][j];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kRows * kAcross / S::NT; ++k) {
      const int r = (int)threadIdx.x / kAcross + k * (S::NT / kAcross);
      Run<T> run;
#pragma unroll
      for (int e = 0; e < kVec<T>; e += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(buf + r * kPitch + (c + e) * 4);
#pragma unroll
        for (int q = 0; q < 4; ++q) run.v[e + q] = v[q];
      }
      f((r / 16) * S::MI * 16 + i * 16 + r % 16, c, run);
    }
  }
}

// Softmax statistics of some classes of a row: the largest logit, and with it
// subtracted sum exp and sum exp z. Nothing seen: {-inf, 0, 0}.
struct Stats {
  float top, sum, zsum;
};
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b) {
  Stats o;
  o.top = fmaxf(a.top, b.top);
  const float da = a.top == -INFINITY ? 0.f : a.top - o.top, db = b.top == -INFINITY ? 0.f : b.top - o.top;
  const float ea = exp_(da), eb = exp_(db);   // a side that saw nothing has sums of zero (NaN sums stay)
  o.sum = a.sum * ea + b.sum * eb;
  o.zsum = (a.zsum + da * a.sum) * ea + (b.zsum + db * b.sum) * eb;
  return o;
}

// Whether class j of a row is valid; the target counts as none where it is not.
__device__ __forceinline__ bool class_valid(const RowArgs& a, int64_t row, int j) {
  return !a.valid || ((a.valid[row * a.words + (j >> 5)] >> (j & 31)) & 1u);
}
__device__ __forceinline__ int target_of(const RowArgs& a, int64_t row, bool& wrong) {
  const int y = a.target[row];
  wrong = y < -1 || y >= a.V || (y >= 0 && !class_valid(a, row, y));
  return wrong ? -1 : y;
}
// What a head's epilogue reads of a row.
struct Row {
  int y;
  float lse, up, ent, H;
  __device__ __forceinline__ void load(const RowArgs& a, int64_t row, int hi, bool gradient) {
    y = -1;
    if (row >= hi) return;
    y = a.target[row];
    if (!gradient) return;
    lse = a.lse[row];
    up = a.dlogp[row];
    ent = a.dentropy ? a.dentropy[row] : 0.f;
    H = a.dentropy ? a.entropy[row] : 0.f;
  }
  // the target is a valid class of the row, or none; true where it was neither
  __device__ __forceinline__ bool check(const RowArgs& a, int64_t row, int hi) {
    if (row >= hi) return false;
    const bool wrong = y < -1 || y >= a.V || (y >= 0 && !class_valid(a, row, y));
    if (wrong) y = -1;
    if (y < 0) up = 0.f;
    return wrong;
  }
};
__device__ __forceinline__ void put_row(const RowArgs& a, int64_t row, const Stats& s, int y, float zy) {
  const bool some = !(s.sum == 0.f);
  const float ln = some ? __logf(s.sum) : 0.f;
  a.logp[row] = some && y >= 0 ? zy - s.top - ln : 0.f;
  if (a.entropy) a.entropy[row] = some ? ln - s.zsum / s.sum : 0.f;
  if (a.lse) a.lse[row] = some ? s.top + ln : -INFINITY;
}

template <typename T, class S, bool COLUMNS, int EPI>
__global__ __launch_bounds__(S::NT, S::kWaves) void rows_kernel(const RowArgs a) {
  using P = RowTile<T, S::BM, S::NT, S::D, S::SB>;
  using Q = typename std::conditional<COLUMNS, ColTile<T, S::BN, S::NT, S::D, S::SB>, RowTile<T, S::BN, S::NT, S::D, S::SB>>::type;
  using Product = Sum<T, S, P, Q, false>;
  __shared__ __attribute__((aligned(16))) char lds[2 * Product::kBuf];
  __shared__ Row rows[EPI == kStats || EPI == kGradLogits ? S::BM : 1];

  int rt, ct;
  tile_of(blockIdx.x, a.row_tiles, a.col_tiles, rt, ct);
  Part part;
  bool bad;
  const bool found = find_part(a.offsets, a.G, a.n, S::BM, rt, part, bad);
  if (bad && blockIdx.x == 0 && threadIdx.x == 0 && a.error) atomicOr(a.error, IM_ERR_COUNT);
  if (!found) return;

  const T* A = static_cast<const T*>(a.A);
  const T* B = static_cast<const T*>(a.B) + part.g * a.b_group;
  const int n_first = ct * S::BN;   // < N: the launch has no column tiles past the operand
  Product x;
  x.lds = lds;
  x.steps = (a.K + P::kStage - 1) / P::kStage;
  x.p.init(A, a.lda, part.lo, part.hi - 1, a.K);
  if constexpr (COLUMNS) x.q.init(B, a.ldb, n_first, a.N, 0, a.K);
  else x.q.init(B, a.ldb, n_first, a.N - 1, a.K);
  // a head's row: loaded before the sums, needed after them
  Row mine{};
  if constexpr (EPI == kStats || EPI == kGradLogits) mine.load(a, part.lo + (int)threadIdx.x, part.hi, EPI == kGradLogits);
  x.run();
  auto& acc = x.acc;
  if constexpr (EPI == kStats || EPI == kGradLogits) {
    const bool wrong = mine.check(a, part.lo + (int)threadIdx.x, part.hi);
    if (wrong && a.col0 == 0 && ct == 0 && a.error) atomicOr(a.error, IM_ERR_ACTION);
    static_assert(S::NT >= S::BM, "a thread a row");
    if ((int)threadIdx.x < S::BM) rows[threadIdx.x] = mine;
    __syncthreads();
  }

  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, g4 = (lane / 16) * 4;
  const int wm = wave / S::WN, wn = wave % S::WN;
  const int m_at = wm * S::MI * 16 + lane % 16, n_at = n_first + wn * S::NJ * 16 + g4;
  const float* bias = a.bias ? a.bias + part.g * a.bias_group + a.col0 : nullptr;

  static_assert(2 * S::WM * 16 * (S::BN * 4 + 16) <= (int)sizeof(lds), "the results pass through the stages' LDS");
  if constexpr (EPI == kStore) {
    Run<T> plus;
    const int c = n_first + ((int)threadIdx.x % (S::BN / kVec<T>)) * kVec<T>;
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) plus.v[e] = bias && c + e < a.N ? bias[c + e] : 0.f;
    by_rows<T, S>(acc, lds, [&](int m, int n, Run<T>& run) {
      const int64_t row = part.lo + m;
      if (row >= part.hi || n_first + n >= a.N) return;
#pragma unroll
      for (int e = 0; e < kVec<T>; ++e) {
        run.v[e] += plus.v[e];
        if (a.relu) run.v[e] = run.v[e] < 0.f ? 0.f : run.v[e];   // NaN stays
      }
      run.store(static_cast<T*>(a.C) + row * a.ldc + n_first + n, a.N - n_first - n);
    });
  }
  if constexpr (EPI == kStoreInput) {
    by_rows<T, S>(acc, lds, [&](int m, int n0, Run<T>& run) {
      const int64_t row = part.lo + m;
      const int n = n_first + n0, left = a.N - n;
      if (row >= part.hi || left <= 0) return;
      if (a.sum) {
        float* sum = a.sum + row * a.N + n;
#pragma unroll
        for (int e = 0; e < kVec<T>; e += 4) {
          f32x4 v = {run.v[e], run.v[e + 1], run.v[e + 2], run.v[e + 3]};
          if (!a.first && left > e) v += load4(sum + e, left - e);
          if (!a.last && left > e) store4(sum + e, v, left - e);
#pragma unroll
          for (int q = 0; q < 4; ++q) run.v[e + q] = v[q];
        }
        if (!a.last) return;
      }
      if (a.X) {
        Run<T> x;
        x.load(static_cast<const T*>(a.X) + row * a.ldx + n, left);
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) run.v[e] = x.v[e] > 0.f ? run.v[e] : 0.f;
      }
      run.store(static_cast<T*>(a.C) + row * a.ldc + n, left);
    });
  }

  if constexpr (EPI == kStats) {
    // each row's classes lie in four lanes of WN waves
    float* taken = reinterpret_cast<float*>(lds);                    // [BM]
    Stats* across = reinterpret_cast<Stats*>(lds + S::BM * 4);       // [WN][BM]
    static_assert(S::BM * 4 + S::WN * S::BM * sizeof(Stats) <= sizeof(lds), "fits");
    const bool whole = a.col_tiles == 1;
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
      const int m = m_at + i * 16;
      const int64_t row = part.lo + m;
      const bool in = row < part.hi;
      const int y = rows[m].y;
      Stats s{-INFINITY, 0.f, 0.f};
      uint32_t ok = 0;
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) {
        const int n = n_at + j * 16, left = a.N - n;
        if (left <= 0 || !in) continue;
        if (bias) acc[i][j] += load4(bias + n, left);
        uint32_t bits = left >= 4 ? 15u : (1u << left) - 1u;
        // four classes from a multiple of 4: one word
        if (a.valid) bits &= a.valid[row * a.words + (n >> 5)] >> (n & 31);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float z = acc[i][j][r];
          if (n + r == y) (whole ? taken[m] : a.taken[row]) = z;
          if (!((bits >> r) & 1u) || z == -INFINITY) continue;
          ok |= 1u << (j * 4 + r);
          s.top = fmaxf(s.top, z);
        }
      }
      const float ref = s.top == -INFINITY ? 0.f : s.top;
#pragma unroll
      for (int j = 0; j < S::NJ; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float d = acc[i][j][r] - ref, e = exp_(d);
          const bool take = (ok >> (j * 4 + r)) & 1u;
          s.sum += take ? e : 0.f;
          s.zsum += take ? e * d : 0.f;
        }
#pragma unroll
      for (int d = 16; d < 64; d *= 2) {
        const Stats o{__shfl_xor(s.top, d), __shfl_xor(s.sum, d), __shfl_xor(s.zsum, d)};
        s = join(s, o);
      }
      if (g4 == 0) across[wn * S::BM + m] = s;
    }
    __syncthreads();
    for (int m = threadIdx.x; m < S::BM; m += S::NT) {
      const int64_t row = part.lo + m;
      if (row >= part.hi) continue;
      Stats s = across[m];
#pragma unroll
      for (int w = 1; w < S::WN; ++w) s = join(s, across[w * S::BM + m]);
      if (whole) {
        put_row(a, row, s, rows[m].y, taken[m]);
      } else {
        float* to = a.stats + ((int64_t)ct * a.n + row) * 3;
        to[0] = s.top, to[1] = s.sum, to[2] = s.zsum;
      }
    }
  }

  if constexpr (EPI == kGradLogits) {
    float colsum[S::NJ][4];
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) colsum[j][r] = 0.f;
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
      const int64_t row = part.lo + m_at + i * 16;
      if (row >= part.hi) continue;
      const Row& of = rows[m_at + i * 16];
      const int y = of.y;
      const float lse = of.lse, up = of.up, ent = of.ent, H = of.H;
      const bool live = (up != 0.f || ent != 0.f) && lse != -INFINITY;
      // a row that adds nothing is kept from the sums over rows where its h is not finite (its
      // logits then are not either); elsewhere its zeros do
      if (a.live && a.col0 == 0 && ct == 0 && wn == 0 && g4 == 0)
        a.live[row] = live || fabsf(acc[i][0][0]) < INFINITY;
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) {
        const int n = n_at + j * 16, left = a.N - n;
        if (left <= 0) continue;
        f32x4 z = acc[i][j], dz;   // dz takes the logits' place
        if (bias) z += load4(bias + n, left);
        const int c = a.col0 + n;   // pieces begin at multiples of 32 classes
        uint32_t bits = live ? (left >= 4 ? 15u : (1u << left) - 1u) : 0u;
        if (a.valid) bits &= a.valid[row * a.words + (c >> 5)] >> (c & 31);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float lp = z[r] - lse, pr = exp_(lp);
          const bool ok = ((bits >> r) & 1u) && z[r] != -INFINITY;
          float d = up * ((c + r == y ? 1.f : 0.f) - pr);
          if (a.dentropy && pr != 0.f) d -= ent * pr * (lp + H);
          dz[r] = ok ? d : 0.f;
          colsum[j][r] += dz[r];
        }
        acc[i][j] = dz;
      }
    }
    by_rows<T, S>(acc, lds, [&](int m, int n, Run<T>& run) {
      const int64_t row = part.lo + m;
      if (row < part.hi && n_first + n < a.N)
        run.store(static_cast<T*>(a.C) + row * a.ldc + n_first + n, a.N - n_first - n);
    });
    if (a.db_part) {
      __syncthreads();
      float* across = reinterpret_cast<float*>(lds);   // [WM][BN]
      static_assert(S::WM * S::BN * 4 <= sizeof(lds), "fits");
#pragma unroll
      for (int j = 0; j < S::NJ; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v = colsum[j][r];
#pragma unroll
          for (int d = 1; d < 16; d *= 2) v += __shfl_xor(v, d);
          if (lane % 16 == 0) across[wm * S::BN + n_at - n_first + j * 16 + r] = v;
        }
      __syncthreads();
      for (int c = threadIdx.x; c < S::BN; c += S::NT) {
        if (n_first + c >= a.N) continue;
        float v = across[c];
#pragma unroll
        for (int w = 1; w < S::WM; ++w) v += across[w * S::BN + c];
        a.db_part[(int64_t)rt * a.db_width + a.col0 + n_first + c] = v;
      }
    }
  }
}

// Joins the column tiles' statistics of 16 rows a block: 16 threads a row.
__global__ __launch_bounds__(256) void join_kernel(const RowArgs a) {
  __shared__ Stats across[4][16];
  const int r = threadIdx.x % 16, part = threadIdx.x / 16;
  const int64_t row = (int64_t)blockIdx.x * 16 + r;
  int end = a.n;
  if (a.offsets) {
    Part run;
    bool bad;
    find_part(a.offsets, a.G, a.n, 1, 0, run, bad);
    if (bad) return;
    end = a.offsets[a.G];
  }
  Stats s{-INFINITY, 0.f, 0.f};
  if (row < end)
    for (int c = part; c < a.col_tiles; c += 16) {
      const float* p = a.stats + ((int64_t)c * a.n + row) * 3;
      s = join(s, Stats{p[0], p[1], p[2]});
    }
#pragma unroll
  for (int d = 16; d < 64; d *= 2) s = join(s, Stats{__shfl_xor(s.top, d), __shfl_xor(s.sum, d), __shfl_xor(s.zsum, d)});
  if (threadIdx.x % 64 < 16) across[threadIdx.x / 64][r] = s;
  __syncthreads();
  if (threadIdx.x >= 16 || row >= end) return;
  for (int w = 1; w < 4; ++w) s = join(s, across[w][r]);
  bool wrong;
  const int y = target_of(a, row, wrong);
  put_row(a, row, s, y, y >= 0 ? a.taken[row] : 0.f);
}

using Large = Shape<2, 4, 8, 4, 1, 128>;    // 256 x 256, 512 threads
using Middle = Shape<2, 2, 4, 4, 1, 128>;   // 128 x 128
using Narrow = Shape<4, 1, 2, 4, 1, 128>;   // 128 x 64
using Small = Shape<2, 2, 2, 2, 2, 128>;    // 64 x 64

template <typename T, class S, bool COLUMNS, int EPI>
hipError_t launch(const RowArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((rows_kernel<T, S, COLUMNS, EPI>), dim3((unsigned)(a.row_tiles * a.col_tiles)), dim3(S::NT), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && EPI == kStats && a.col_tiles > 1) {
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)((a.n + 15) / 16)), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}
template <typename T, bool COLUMNS, int EPI>
hipError_t launch_shape(const RowArgs& a, int shape, hipStream_t s) {
  switch (shape) {
    case 0: return launch<T, Large, COLUMNS, EPI>(a, s);
    case 1: return launch<T, Middle, COLUMNS, EPI>(a, s);
    case 2: return launch<T, Narrow, COLUMNS, EPI>(a, s);
    default: return launch<T, Small, COLUMNS, EPI>(a, s);
  }
}
template <typename T>
hipError_t launch_type(const RowArgs& a, int shape, int epilogue, hipStream_t s) {
  switch (epilogue) {
    case kStore: return launch_shape<T, false, kStore>(a, shape, s);
    case kStoreInput: return launch_shape<T, true, kStoreInput>(a, shape, s);
    case kStats: return launch_shape<T, false, kStats>(a, shape, s);
    default: return launch_shape<T, false, kGradLogits>(a, shape, s);
  }
}

}  // namespace

RowPlan plan_rows(int dtype, int64_t n, int64_t G, int64_t N, int cus) {
  static const int bm[] = {Large::BM, Middle::BM, Narrow::BM, Small::BM};
  static const int bn[] = {Large::BN, Middle::BN, Narrow::BN, Small::BN};
  auto tiles = [&](int s) { return (n / bm[s] + G) * ((N + bn[s] - 1) / bn[s]); };
  int s = 3;
  if (N <= Narrow::BN && n >= 64 * cus) s = 2;
  else if (N > Narrow::BN && tiles(0) >= cus && n >= 256 * G) s = 0;
  else if (N > Narrow::BN && tiles(1) >= cus && n >= 128 * G) s = 1;
  (void)dtype;
  RowPlan p;
  p.shape = s;
  p.row_tiles = (n + bm[s] - 1) / bm[s] + (G > 1 ? G - 1 : 0);
  p.col_tiles = (N + bn[s] - 1) / bn[s];
  return p;
}

int rows_per_tile(int shape) {
  return shape == 0 ? Large::BM : (shape == 1 ? Middle::BM : (shape == 2 ? Narrow::BM : Small::BM));
}

int cols_per_tile(int shape) {
  return shape == 0 ? Large::BN : (shape == 1 ? Middle::BN : (shape == 2 ? Narrow::BN : Small::BN));
}

hipError_t launch_rows_product(const RowArgs& a, int dtype, int shape, int epilogue, hipStream_t s) {
  return dtype == IM_BF16 ? launch_type<__bf16>(a, shape, epilogue, s) : launch_type<float>(a, shape, epilogue, s);
}

}  // namespace learn
}  // namespace im
