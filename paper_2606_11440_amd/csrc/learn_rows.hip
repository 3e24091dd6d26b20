// Products of grouped rows with their group's weights, and what follows them
// in registers: the layers (bias, ReLU), the gradient of a layer's input (the
// ReLU before it) and the softmax head (statistics, gradient of the logits).
//
// A stage of k is 128 bytes (64 bf16, 32 fp32): one barrier a stage, a line of
// memory a row. The large tile, 256 x 256 with 32 fragments a wave, is what the
// matrix cores ask for: a wave reads 12 fragments of LDS for 32 products,
// one of a 128 x 128 tile 8 for 16. Its accumulators leave one block a CU, so a
// block keeps taking tiles, and the loads of the next one's first stage pass
// under the epilogue. Measured, bf16 (kernel alone): 8192 x 8192 x 8192 0.94 to
// 1.01 ms (1.09 to 1.17 PFLOP/s; a library product of the size 1.28), 8192 x 4096 x
// 4096 258 us (286 with rows of 4095), 262144 x 256 x 256 74 us (3.6 TB/s: 50 us at the
// rate of a copy), 16 x 4096 x 4096 14 us (6.3 us of W at the rate of a copy).
// What bounds it: at large k the LDS and its barriers (the matrix cores are busy
// 50 to 60 % of the time); at k of 4 stages or fewer the epilogue, which the one
// block of a CU does not overlap with products. Tried, and slower or equal: two
// stages in flight in registers, 256 x 128 tiles, and leaving out the fragments
// of rows that a ragged tile lacks (8192^3 0.95 to 1.03 ms).
#include <type_traits>

#include "learn_internal.h"
#include "learn_softmax.h"
#include "learn_tile.h"

namespace im {
namespace learn {
namespace {


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

// Softmax statistics of some classes of a row: the largest logit, and with it
// subtracted sum e^z and sum e^z z. Nothing seen: {-inf, 0, 0}. Logits are scaled
// by log2 e once the largest is taken from them, on the way into the exponential
// only: a finite one stays finite down to the lowest float.
struct Stats {
  float top, sum, zsum;
};
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b) {
  Stats o;
  o.top = fmaxf(a.top, b.top);
  // at kLeastE the exponential is 0; further down the distance times the sum would overflow (0 times infinity)
  const float da = a.top == -INFINITY ? 0.f : fmaxf(a.top - o.top, kLeastE);
  const float db = b.top == -INFINITY ? 0.f : fmaxf(b.top - o.top, kLeastE);
  const float ea = exp_(da), eb = exp_(db);   // a side that saw nothing has sums of zero (NaN sums stay)
  o.sum = a.sum * ea + b.sum * eb;
  o.zsum = (a.zsum + da * a.sum) * ea + (b.zsum + db * b.sum) * eb;
  return o;
}

// Whether class j of a row is valid; the target counts as none where it is not.
__device__ __forceinline__ bool class_valid(const RowArgs& a, int64_t row, int j) {
  return !a.valid || ((a.valid[row * a.words + (j >> 5)] >> (j & 31)) & 1u);
}
__device__ __forceinline__ bool target_wrong(const RowArgs& a, int64_t row, int y) {
  return y < -1 || y >= a.V || (y >= 0 && !class_valid(a, row, y));
}
// zy: logit of the target
__device__ __forceinline__ void put_row(const RowArgs& a, int64_t row, const Stats& s, int y, float zy) {
  const bool some = !(s.sum == 0.f);
  const float lg = some ? __builtin_amdgcn_logf(s.sum) * kLn2 : 0.f;   // logf: log2
  a.logp[row] = some && y >= 0 ? zy - s.top - lg : 0.f;
  if (a.entropy) a.entropy[row] = some ? lg - s.zsum / s.sum : 0.f;
  if (a.lse) a.lse[row] = some ? s.top + lg : -INFINITY;
}

// What a head's epilogue reads of a row. For the gradient, with t = log2 pi:
//   dz = 2^t (A + B t), and `up` more at the target;
//   A = -up - ent H, B = -ent ln 2, t = (z - lse) log2 e
// A row that adds nothing has A = B = up = 0 and lse = +inf, so that t is the
// least there is and every dz is 0, whatever its logits are.
struct Row {
  int y;
  float lse, A, B, up;
  bool live;
  __device__ __forceinline__ void load(const RowArgs& a, int64_t row, int hi, bool gradient) {
    y = -1;
    A = B = up = 0.f;
    lse = INFINITY;
    live = false;
    if (row >= hi) return;
    y = a.target[row];
    if (!gradient) return;
    lse = a.lse[row];
    up = a.dlogp[row];
    A = a.dentropy ? a.entropy[row] : 0.f;
    B = a.dentropy ? a.dentropy[row] : 0.f;
  }
  // the target is a valid class of the row, or none; true where it was neither
  __device__ __forceinline__ bool check(const RowArgs& a, int64_t row, int hi, bool gradient) {
    if (row >= hi) return false;
    const bool wrong = target_wrong(a, row, y);
    if (wrong) y = -1;
    if (!gradient) return wrong;
    if (y < 0) up = 0.f;
    const float H = A, ent = B;
    live = (up != 0.f || ent != 0.f) && !(lse <= kMasked);
    up = live ? up : 0.f;
    A = live ? -up - ent * H + (lse - lse) : 0.f;   // an lse that is not finite makes the row NaN
    B = live ? -ent * kLn2 : 0.f;
    lse = live ? lse : INFINITY;
    return wrong;
  }
};

template <typename T, class S, bool COLUMNS, int EPI>
__global__ __launch_bounds__(S::NT, S::kWaves) void rows_kernel(const RowArgs a) {
  using P = RowTile<T, S::BM, S::NT, S::D, S::SB>;
  using Q = typename std::conditional<COLUMNS, ColTile<T, S::BN, S::NT, S::D, S::SB>,
                                      RowTile<T, S::BN, S::NT, S::D, S::SB>>::type;
  using Product = Sum<T, S, P, Q, false>;
  constexpr bool kHead = EPI == kStats || EPI == kGradLogits;
  __shared__ __attribute__((aligned(16))) char lds[2 * Product::kBuf];
  __shared__ Groups groups;
  __shared__ float column_sums[EPI == kGradLogits ? S::WM * S::BN : 1];
  static_assert(S::NT >= S::BM, "a thread a row");
  static_assert(EPI != kGradLogits || S::NT >= S::BN, "a thread a column");

  groups.init(a.offsets, a.G, a.n, S::BM);
  __syncthreads();
  if (groups.total < 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.error) atomicOr(a.error, IM_ERR_COUNT);
    return;
  }
  // with several runs of k a tile is as many units of work, one after the other
  const int row_tiles = groups.total, splits = EPI == kPartial ? a.splits : 1, total = row_tiles * a.col_tiles * splits;
  int tile = blockIdx.x;
  if (tile >= total) return;

  Product x;
  x.lds = lds;
  x.steps = (a.K + P::kStage - 1) / P::kStage;
  Row mine;
  int rt, ct, g, lo, hi, split = 0;
  auto enter = [&](int t) {   // takes tile t: its first loads are on their way
    const int tid = fresh_thread();
    int k0 = 0, K = a.K;
    if constexpr (EPI == kPartial) {
      split = t % splits;
      t /= splits;
      k0 = split * a.split_k;
      K = a.K - k0 < a.split_k ? a.K - k0 : a.split_k;
      x.steps = (K + P::kStage - 1) / P::kStage;
    }
    tile_of(t, row_tiles, a.col_tiles, rt, ct);
    groups.find(a.offsets, a.G, a.n, S::BM, rt, g, lo, hi);
    const T* B = static_cast<const T*>(a.B) + g * a.b_group;
    x.p.init(static_cast<const T*>(a.A) + k0, a.lda, lo, hi - 1, K, tid);
    // ct * BN < N: the launch has no column tiles past the operand
    if constexpr (COLUMNS) x.q.init(B, a.ldb, ct * S::BN, a.N, k0, k0 + K, tid);
    else x.q.init(B + k0, a.ldb, ct * S::BN, a.N - 1, K, tid);
    x.begin();
    if constexpr (kHead) mine.load(a, (int64_t)lo + tid, hi, EPI == kGradLogits);
  };
  enter(tile);
  x.first_stage();
  while (true) {
    x.run();
    auto& acc = x.acc;
    const int tid = fresh_thread(), lane = tid % 64, wave = tid / 64, g4 = (lane / 16) * 4;
    const int wm = wave / S::WN, wn = wave % S::WN, m_at = wm * S::MI * 16 + lane % 16;
    // the tile at hand; the next one's loads run through its epilogue
    const int at_lo = lo, at_hi = hi, at_rt = rt, at_ct = ct, at_g = g, at_split = split, n_first = ct * S::BN;
    // a head's rows, behind what the statistics take of the stages' LDS
    Row* const rows = reinterpret_cast<Row*>(lds + S::BM * 4 + S::WN * S::BM * (int)sizeof(Stats));
    static_assert(S::BM * (4 + S::WN * (int)sizeof(Stats) + (int)sizeof(Row)) <= (int)sizeof(lds), "fits");
    if constexpr (kHead) {
      const bool wrong = mine.check(a, (int64_t)lo + tid, hi, EPI == kGradLogits);
      if (wrong && a.col0 == 0 && ct == 0 && a.error) atomicOr(a.error, IM_ERR_ACTION);
      if (tid < S::BM) rows[tid] = mine;
      __syncthreads();
    }
    tile += gridDim.x;
    const bool more = tile < total;
    auto next = [&] {
      if (more) enter(tile);
    };
    auto last = [&](bool on) {   // the next tile's first stage takes the LDS that the epilogue has read
      if (!on) return;
      __syncthreads();
      x.first_stage();
    };
    const int n_at = n_first + wn * S::NJ * 16 + g4;
    const float* bias = a.bias ? a.bias + at_g * a.bias_group + a.col0 : nullptr;
    // A tile without an edge takes no branch on its way out: the next tile's loads,
    // issued before its stores, are then waited for without them.
    const bool full = at_hi - at_lo == S::BM && n_first + S::BN <= a.N;
    using O = Out<T, S, (int)sizeof(lds)>;
    char* const C = reinterpret_cast<char*>(static_cast<T*>(a.C) + (int64_t)at_lo * a.ldc + n_first);
    auto place = [&](int m, int c) { return ((uint32_t)m * (uint32_t)a.ldc + (uint32_t)c) * (uint32_t)sizeof(T); };
    auto put = [&](int, int m, int c, u32x4 v) { *reinterpret_cast<u32x4_any*>(C + place(m, c)) = v; };
    auto put_some = [&](int, int m, int c, u32x4 v) {
      const int left = a.N - n_first - c;
      if (at_lo + m >= at_hi || left <= 0) return;
      T* const to = reinterpret_cast<T*>(C + place(m, c));
      if (left >= kVec<T>) *reinterpret_cast<u32x4_any*>(to) = v;
      else store_few(to, v, left);
    };

    if constexpr (EPI == kPartial) {
      using F = Out<float, S, (int)sizeof(lds)>;
      float* const part = a.part + (int64_t)at_split * a.n * a.N;
      F::run(lds, tid, [&](int i, int j) { return acc[i][j]; }, next, [&](int, int m, int c, u32x4 v) {
        const int64_t row = (int64_t)at_lo + m;
        const int n = n_first + c;
        if (row < at_hi && n < a.N) store4(part + row * a.N + n, __builtin_bit_cast(f32x4, v), a.N - n);
      });
      last(more);
    }

    if constexpr (EPI == kStore) {
      f32x4 plus[S::NJ];
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) {
        plus[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (bias && n_at + j * 16 < a.N) plus[j] = load4(bias + n_at + j * 16, a.N - n_at - j * 16);
      }
      const float least = a.relu ? 0.f : -INFINITY;
      auto value = [&](int i, int j) {
        f32x4 v = acc[i][j] + plus[j];
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = v[r] < least ? least : v[r];   // NaN stays
        return v;
      };
      if (full) {
        O::run(lds, tid, value, next, put);
        last(more);
      } else {
        O::run(lds, tid, value, next, put_some);
        last(more);
      }
    }

    if constexpr (EPI == kStoreInput) {
      auto value = [&](int i, int j) { return acc[i][j]; };
      if (a.sum) {   // a piece of a head's classes
        using F = Out<float, S, (int)sizeof(lds)>;
        F::run(lds, tid, value, [] {}, [&](int, int m, int c, u32x4 x) {
          const int64_t row = (int64_t)at_lo + m;
          const int n = n_first + c, left = a.N - n;
          if (row >= at_hi || left <= 0) return;
          f32x4 v = __builtin_bit_cast(f32x4, x);
          float* sum = a.sum + row * a.N + n;
          if (!a.first) v += load4(sum, left);
          if (!a.last) {
            store4(sum, v, left);
            return;
          }
          for (int q = 0; q < 4 && q < left; ++q) {
            const float y = v[q];
            const bool keep = !a.X || (float)static_cast<const T*>(a.X)[row * a.ldx + n + q] > 0.f;
            static_cast<T*>(a.C)[row * a.ldc + n + q] = (T)(keep ? y : 0.f);
          }
        });
        next();
        last(more);
      } else if (!a.X) {
        if (full) {
          O::run(lds, tid, value, next, put);
          last(more);
        } else {
          O::run(lds, tid, value, next, put_some);
          last(more);
        }
      } else {
        // the layer's input, loaded before the results that it lets through are read
        const char* const X = reinterpret_cast<const char*>(static_cast<const T*>(a.X) + (int64_t)at_lo * a.ldx + n_first);
        auto x_at = [&](int k) {
          const int m = O::row_of(k / O::kUnits, k % O::kUnits, tid), c = O::column_of(tid);
          return ((uint32_t)m * (uint32_t)a.ldx + (uint32_t)c) * (uint32_t)sizeof(T);
        };
        constexpr int kAll = O::kUnits * O::kPasses, kAhead = kAll < 8 ? kAll : 8;
        u32x4 xs[kAhead];
        if (full) {
          O::run(lds, tid, value,
                 [&] {
                   if (O::kPasses == 1) next();
#pragma unroll
                   for (int k = 0; k < kAhead; ++k) xs[k] = *reinterpret_cast<const u32x4_any*>(X + x_at(k));
                 },
                 [&](int k, int m, int c, u32x4 v) {
                   put(k, m, c, where_positive<T>(v, xs[k % kAhead]));
                   if (k + kAhead < kAll) xs[k % kAhead] = *reinterpret_cast<const u32x4_any*>(X + x_at(k + kAhead));
                 });
          if (O::kPasses > 1) next();
          last(more);
        } else {
          O::run(lds, tid, value, next, [&](int k, int m, int c, u32x4 v) {
            const int left = a.N - n_first - c;
            if (at_lo + m >= at_hi || left <= 0) return;
            const T* const from = reinterpret_cast<const T*>(X + x_at(k));
            put_some(k, m, c, where_positive<T>(v, left >= kVec<T> ? load16(from) : load_few(from, left)));
          });
          last(more);
        }
      }
    }

    if constexpr (kHead) {
      // A wave's columns begin at a multiple of 32 classes (as pieces do): their mask words
      constexpr int kWords = (S::NJ * 16 + 31) / 32;
      uint32_t words[S::MI][kWords];
      if (a.valid) {
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
          const int64_t row = at_lo + m_at + i * 16 < at_hi ? at_lo + m_at + i * 16 : at_hi - 1;
#pragma unroll
          for (int w = 0; w < kWords; ++w) {
            const int at = (a.col0 + n_first + wn * S::NJ * 16) / 32 + w;
            words[i][w] = a.valid[row * a.words + (at < a.words ? at : a.words - 1)];
          }
        }
      }
      const int n_wave = n_first + wn * S::NJ * 16;
      auto near = [&](int y) { return (unsigned)(y - n_wave) < (unsigned)(S::NJ * 16); };
      auto bits_of = [&](int i, int j) { return words[i][j / 2] >> ((j & 1) * 16 + g4); };
      f32x4 plus[S::NJ];   // the classes' biases
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) {
        plus[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (bias && n_at + j * 16 < a.N) plus[j] = load4(bias + n_at + j * 16, a.N - n_at - j * 16);
      }

      if constexpr (EPI == kStats) {
        // each row's classes lie in four lanes of WN waves
        float* taken = reinterpret_cast<float*>(lds);                    // [BM]
        Stats* across = reinterpret_cast<Stats*>(lds + S::BM * 4);       // [WN][BM]
        const bool whole = a.col_tiles == 1, edge = n_first + S::BN > a.N;
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
          const int m = m_at + i * 16, y = rows[m].y;
          Stats s{-INFINITY, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < S::NJ; ++j) acc[i][j] += plus[j];
          if (__any(near(y))) {   // the target is in the wave's columns for some rows
#pragma unroll
            for (int j = 0; j < S::NJ; ++j) {
              const int at = y - n_at - j * 16;
              const f32x4 z = acc[i][j];
              if ((unsigned)at < 4u)
                (whole ? taken[m] : a.taken[(int64_t)at_lo + m]) = at == 0 ? z[0] : (at == 1 ? z[1] : (at == 2 ? z[2] : z[3]));
            }
          }
          if (a.valid) {
#pragma unroll
            for (int j = 0; j < S::NJ; ++j) {
              const uint32_t bits = bits_of(i, j);
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[i][j][r] = (bits >> r) & 1u ? acc[i][j][r] : -INFINITY;
            }
          }
          if (edge) {
#pragma unroll
            for (int j = 0; j < S::NJ; ++j)
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[i][j][r] = n_at + j * 16 + r < a.N ? acc[i][j][r] : -INFINITY;
          }
#pragma unroll
          for (int j = 0; j < S::NJ; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) s.top = fmaxf(s.top, acc[i][j][r]);
          const float ref = s.top == -INFINITY ? 0.f : s.top;
          if (a.entropy) {
#pragma unroll
            for (int j = 0; j < S::NJ; ++j)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float d = acc[i][j][r] - ref, e = exp_(d);
                s.sum += e;                                    // NaN goes this way
                s.zsum = fmaf(e, fmaxf(d, kLeastE), s.zsum);   // no 0 times infinity
              }
          } else {
#pragma unroll
            for (int j = 0; j < S::NJ; ++j)
#pragma unroll
              for (int r = 0; r < 4; ++r) s.sum += exp_(acc[i][j][r] - ref);
          }
#pragma unroll
          for (int d = 16; d < 64; d *= 2) {
            const Stats o{__shfl_xor(s.top, d), __shfl_xor(s.sum, d), __shfl_xor(s.zsum, d)};
            s = join(s, o);
          }
          if (g4 == 0) across[wn * S::BM + m] = s;
        }
        next();
        __syncthreads();
        for (int m = tid; m < S::BM; m += S::NT) {
          const int64_t row = (int64_t)at_lo + m;
          if (row >= at_hi) continue;
          Stats s = across[m];
#pragma unroll
          for (int w = 1; w < S::WN; ++w) s = join(s, across[w * S::BM + m]);
          if (whole) {
            put_row(a, row, s, rows[m].y, taken[m]);
          } else {
            float* to = a.stats + ((int64_t)at_ct * a.n + row) * 3;
            to[0] = s.top, to[1] = s.sum, to[2] = s.zsum;
          }
        }
        last(more);
      }

      if constexpr (EPI == kGradLogits) {
        f32x4 colsum[S::NJ];
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) colsum[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
          const int m = m_at + i * 16;
          const Row of = rows[m];
          // a row that adds nothing is kept from the sums over rows where its h is not finite
          // (its logits then are not either); elsewhere its zeros do
          if (a.live && a.col0 == 0 && at_ct == 0 && wn == 0 && g4 == 0 && at_lo + m < at_hi)
            a.live[(int64_t)at_lo + m] = of.live || fabsf(acc[i][0][0]) < INFINITY;
          const int y = of.y - a.col0;
          const bool target = __any(near(y));   // in the wave's columns for some rows
#pragma unroll
          for (int j = 0; j < S::NJ; ++j) {
            const int n = n_at + j * 16;
            f32x4 dz;   // takes the logits' place
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              // the logit is rounded as the statistics' is, before lse is taken from it: where a bias
              // outweighs the products by far, lse holds nothing of them either
              const float t = log2_share(acc[i][j][r] + plus[j][r] - of.lse);
              dz[r] = exp2_(t) * fmaf(of.B, t, of.A);
            }
            if (target && (unsigned)(y - n) < 4u) {
#pragma unroll
              for (int r = 0; r < 4; ++r)
                dz[r] += y - n == r && acc[i][j][r] + plus[j][r] != -INFINITY ? of.up : 0.f;
            }
            if (a.valid) {
              const uint32_t bits = bits_of(i, j);
#pragma unroll
              for (int r = 0; r < 4; ++r) dz[r] = (bits >> r) & 1u ? dz[r] : 0.f;
            }
            colsum[j] += dz;   // rows past the tile's last have A = B = up = 0: nothing
            acc[i][j] = dz;
          }
        }
        if (a.db_part) {
          float* across = column_sums;   // [WM][BN]
#pragma unroll
          for (int j = 0; j < S::NJ; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float v = colsum[j][r];
#pragma unroll
              for (int d = 1; d < 16; d *= 2) v += __shfl_xor(v, d);
              if (lane % 16 == 0) across[wm * S::BN + n_at - n_first + j * 16 + r] = v;
            }
        }
        // dz leaves rounded once to the products' type, half a step of dh's and dW's own: measured on
        // a head with entropy, errors of 0.0024 of the norm against 0.0017. Two bf16 numbers, as
        // narrow heads keep on the chip, would write and read twice as much here.
        __syncthreads();   // the rows are read: the results take the LDS
        auto value = [&](int i, int j) { return acc[i][j]; };
        auto sums = [&] {   // behind the barrier of the pass through LDS
          if (a.db_part && tid < S::BN && n_first + tid < a.N) {
            float v = column_sums[tid];
#pragma unroll
            for (int w = 1; w < S::WM; ++w) v += column_sums[w * S::BN + tid];
            a.db_part[(int64_t)at_rt * a.db_width + a.col0 + n_first + tid] = v;
          }
          next();
        };
        if (full) {
          O::run(lds, tid, value, sums, put);
          last(more);
        } else {
          O::run(lds, tid, value, sums, put_some);
          last(more);
        }
      }
    }
    if (!more) break;
  }
}

// Joins the column tiles' statistics, a block 16 rows at a time: 16 threads a row.
__global__ __launch_bounds__(256) void join_kernel(const RowArgs a) {
  __shared__ Stats across[4][16];
  const int r = threadIdx.x % 16, part = threadIdx.x / 16;
  int end = a.n;
  if (a.offsets) {
    if (!csr_holds(a.offsets, a.G, a.n)) return;
    end = a.offsets[a.G];
  }
  for (int64_t first = (int64_t)blockIdx.x * 16; first < end; first += (int64_t)gridDim.x * 16) {
    const int64_t row = first + r;
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
    if (threadIdx.x < 16 && row < end) {
      for (int w = 1; w < 4; ++w) s = join(s, across[w][r]);
      const int y = a.target[row];
      const bool none = y < 0 || target_wrong(a, row, y);
      put_row(a, row, s, none ? -1 : y, none ? 0.f : a.taken[row]);
    }
    __syncthreads();   // the next rows take the LDS
  }
}

// Joins the runs of k and finishes as kStore (STORE) or kStoreInput do: four
// columns of a row a thread.
template <typename T, bool STORE>
__global__ __launch_bounds__(256) void join_k_kernel(const RowArgs a) {
  const int across = (a.N + 3) / 4;
  int end = a.n;
  if (a.offsets) {
    if (!csr_holds(a.offsets, a.G, a.n)) return;
    end = a.offsets[a.G];
  }
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x, row = idx / across;
  if (row >= end) return;
  const int n = (int)(idx % across) * 4, left = a.N - n;
  const int64_t step = (int64_t)a.n * a.N;
  const float* part = a.part + row * a.N + n;
  f32x4 v = load4(part, left);
#pragma unroll 4
  for (int s = 1; s < a.splits; ++s) v += load4(part + s * step, left);
  if constexpr (STORE) {
    if (a.bias) {
      int g = 0, over = a.offsets ? a.G : 1;   // the last group that begins at or before the row
      while (over - g > 1) {
        const int mid = (g + over) / 2;
        if (a.offsets[mid] <= row) g = mid;
        else over = mid;
      }
      v += load4(a.bias + g * a.bias_group + n, left);
    }
    if (a.relu) {
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = v[r] < 0.f ? 0.f : v[r];   // NaN stays
    }
  } else if (a.sum) {
    float* sum = a.sum + row * a.N + n;
    if (!a.first) v += load4(sum, left);
    if (!a.last) {
      store4(sum, v, left);
      return;
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (r >= left) break;
    const float y = v[r];
    const bool keep = STORE || !a.X || (float)static_cast<const T*>(a.X)[row * a.ldx + n + r] > 0.f;
    static_cast<T*>(a.C)[row * a.ldc + n + r] = (T)(keep ? y : 0.f);
  }
}

using Large = Shape<2, 4, 8, 4, 1, 128>;    // 256 x 256, 512 threads
using Middle = Shape<2, 2, 4, 4, 1, 128>;   // 128 x 128
using Narrow = Shape<4, 1, 2, 4, 1, 128>;   // 128 x 64
using Small = Shape<2, 2, 2, 2, 2, 128>;    // 64 x 64

template <typename T, class S, bool COLUMNS, int EPI>
hipError_t launch(const RowArgs& a, hipStream_t s) {
  // blocks that share the tiles: as many as run at once
  const int tiles = a.row_tiles * a.col_tiles * (EPI == kPartial ? a.splits : 1), most = a.cus * S::kBlocks;
  hipLaunchKernelGGL((rows_kernel<T, S, COLUMNS, EPI>), dim3((unsigned)(tiles < most ? tiles : most)), dim3(S::NT), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && EPI == kStats && a.col_tiles > 1) {
    // a launch has less than 2^32 threads in a dimension: past 2^24 rows the blocks take more of them each
    const int blocks = (a.n + 15) / 16, at_most = 1 << 20;
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)(blocks < at_most ? blocks : at_most)), dim3(256), 0, s, a);
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
template <typename T, bool COLUMNS>
hipError_t launch_split(const RowArgs& a, int shape, hipStream_t s) {
  hipError_t e = shape == 1 ? launch<T, Middle, COLUMNS, kPartial>(a, s) : launch<T, Small, COLUMNS, kPartial>(a, s);
  if (e != hipSuccess) return e;
  // k is cut only where the results are two rounds of tiles at most: some millions of them
  const int64_t quads = (int64_t)a.n * ((a.N + 3) / 4);
  hipLaunchKernelGGL((join_k_kernel<T, !COLUMNS>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_type(const RowArgs& a, int shape, int epilogue, hipStream_t s) {
  switch (epilogue) {
    case kStore: return a.splits > 1 ? launch_split<T, false>(a, shape, s) : launch_shape<T, false, kStore>(a, shape, s);
    case kStoreInput:
      return a.splits > 1 ? launch_split<T, true>(a, shape, s) : launch_shape<T, true, kStoreInput>(a, shape, s);
    case kStats: return launch_shape<T, false, kStats>(a, shape, s);
    default: return launch_shape<T, false, kGradLogits>(a, shape, s);
  }
}

}  // namespace

// The shape with the least time: the rounds that its tiles take, each of as many
// stages as k has and of an epilogue. A stage takes kStageUs where the card is
// full of such blocks (measured: 8192 rows, 4096 x 4096), its share of that with
// fewer blocks on a CU, and kAlone at least (a block by itself waits for its
// loads). Several runs of k, joined by a second kernel (kJoin: its launch and
// latency), where few tiles would leave the card empty.
// Both sides, bf16, us with large / middle / narrow tiles: 193 to 512 of 64
// ragged groups 199 / 224 / 255; ragged experts 327 / 364 / 455; 256 to 256 of
// 262144 rows 74 / 79 / 86; statistics of 50021 classes 530 / 632 / 732, but those
// of 15 classes 93 / 59 / 37 (43 with small ones). Runs of k: 16 x 4096 x 4096 22
// -> 14, while 256 x 1024 x 1024 goes from 9 to 11 with 4 runs, 13 with 8.
RowPlan plan_rows(int dtype, int64_t n, int64_t G, int64_t N, int64_t K, int cus, bool may_split) {
  static const int bm[] = {Large::BM, Middle::BM, Narrow::BM, Small::BM};
  static const int bn[] = {Large::BN, Middle::BN, Narrow::BN, Small::BN};
  static const int per_cu[] = {Large::kBlocks, Middle::kBlocks, Narrow::kBlocks, Small::kBlocks};
  static const double kStageUs[2][4] = {{10.0, 5.0, 4.2, 2.5}, {2.0, 1.35, 1.2, 0.9}};
  static const double kEpilogueUs[4] = {6.0, 4.0, 3.0, 2.5};
  constexpr double kAlone = 0.7, kJoin = 8.0;
  const bool half = dtype == IM_BF16;
  const int64_t stage = 128 / (half ? 2 : 4);
  RowPlan best = {};
  double least = 0;
  for (int s = 0; s < 4; ++s) {
    RowPlan p;
    p.shape = s;
    p.row_tiles = (n + bm[s] - 1) / bm[s] + (G > 1 ? G - 1 : 0);
    p.col_tiles = (N + bn[s] - 1) / bn[s];
    const int64_t steps = (K + stage - 1) / stage, slots = (int64_t)cus * per_cu[s];
    // ragged groups: about half of the tiles that there may be at most
    const double tiles = (G > 1 ? (double)n / bm[s] + 0.5 * (double)(G < n ? G : n) + 0.5 : (double)p.row_tiles) * p.col_tiles;
    for (int64_t splits = 1; splits <= 64; splits *= 2) {
      if (splits > 1 && (!may_split || s == 0 || s == 2 || steps < 4 * splits || tiles * splits > 2 * slots)) break;
      const int64_t each = (steps + splits - 1) / splits;
      p.splits = (steps + each - 1) / each;
      p.split_k = each * stage;
      const double fill = tiles * splits / slots, rounds = fill < 1 ? 1 : (fill < 8 ? (double)(int64_t)(fill + 0.999) : fill);
      // blocks that share a CU
      const double beside = fill < 1 ? (double)(int64_t)(fill * per_cu[s] + 0.999) / per_cu[s] : 1;
      const double full = kStageUs[half][s] * beside, us = rounds * (each * (full > kAlone ? full : kAlone) + kEpilogueUs[s]) +
                        (p.splits > 1 ? kJoin + (double)p.splits * n * N * 8 / 3e6 : 0.0);
      if ((s == 0 && splits == 1) || us < least) {
        best = p;
        least = us;
      }
    }
  }
  return best;
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
