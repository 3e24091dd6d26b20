// Tiles of the learner's products: operands from memory through LDS to the
// matrix cores.
//
// A product sums over k of P[m][k] Q[n][k]. Either operand is stored with k
// contiguous ("rows": P[m] is a row of memory) or with k across the rows
// ("columns": memory row k holds P[.][k]); the three products of a layer need
// both: y = x W^T has rows and rows, dx = dy W rows and columns, dW = dy^T x
// columns and columns. Nothing is transposed in memory: a column tile goes to
// LDS as it lies there and is transposed on the way to registers.
//
// A stage is 128 bytes of k (64 bf16 or 32 fp32). Fragments are those of
// v_mfma_f32_16x16x32_bf16: lane l holds row l % 16, 8 values of k from
// 8 (l / 16). For fp32 a fragment is 4 values of k from 4 (l / 16), used by
// four v_mfma_f32_16x16x4_f32 in turn (the sum runs over the same k in another
// order). Products go in with the operands swapped, so that a lane's four
// results are four neighbouring n of one m.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace im {
namespace learn {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));   // gfx950 loads 16 bytes from any address
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int kStageBytes = 128;
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);             // elements of a 16-byte unit
template <typename T> constexpr int kStage = kStageBytes / (int)sizeof(T);  // k of a stage

template <typename T>
__device__ __forceinline__ u32x4 load16(const T* p) {
  return *reinterpret_cast<const u32x4_any*>(p);
}

// The last `n` elements of a unit, moved to its front; zeros behind them.
template <typename T>
__device__ __forceinline__ u32x4 keep_last(u32x4 v, int n) {
  unsigned __int128 x = __builtin_bit_cast(unsigned __int128, v);
  x = n > 0 ? x >> (8 * (int)sizeof(T) * (kVec<T> - n)) : 0;
  return __builtin_bit_cast(u32x4, x);
}

// n (1..kVec - 1) elements from p, one by one; zeros behind them.
template <typename T>
__device__ __forceinline__ u32x4 load_few(const T* p, int n) {
  T e[kVec<T>];
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) e[i] = i < n ? p[i] : T(0.f);
  u32x4 v;
  __builtin_memcpy(&v, e, 16);
  return v;
}

// A tile of ROWS memory rows with k contiguous, staged by NT threads. Rows past
// the operand's last are read from its last row: they reach results that are
// not stored only. In LDS a row is 8 units of 16 bytes; unit u of row r lies at
// u ^ (r / 2 % 8), so that the 16 lanes of a fragment read touch all 64 banks
// once (128-byte rows: two rows span the banks).
template <typename T, int ROWS, int NT>
struct RowTile {
  static constexpr int kUnits = ROWS * 8 / NT;
  static constexpr int kBytes = ROWS * kStageBytes;
  static_assert(ROWS * 8 % NT == 0 && NT % 8 == 0, "whole units per thread");
  const T* p[kUnits];
  u32x4 r[kUnits];
  int K;

  // rows [first, last] of the operand are the tile's (last - first may be less than ROWS - 1)
  __device__ __forceinline__ void init(const T* base, int64_t ld, int64_t first, int64_t last, int K_) {
    K = K_;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int64_t row = first + ((int)threadIdx.x + i * NT) / 8;
      p[i] = base + (row < last ? row : last) * ld + ((int)threadIdx.x % 8) * kVec<T>;
    }
  }
  __device__ __forceinline__ void load(int kt) {
    const int k0 = kt * kStage<T>;
    if (k0 + kStage<T> <= K) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) r[i] = load16(p[i] + k0);
    } else {   // the row ends inside the stage: its last unit is read so that it ends with the row
      const int n = K - k0 - ((int)threadIdx.x % 8) * kVec<T>;
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        if (n >= kVec<T>) r[i] = load16(p[i] + k0);
        else if (n <= 0) r[i] = u32x4{0, 0, 0, 0};
        else if (K >= kVec<T>) r[i] = keep_last<T>(load16(p[i] + k0 + n - kVec<T>), n);
        else r[i] = load_few(p[i] + k0, n);
      }
    }
  }
  __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int idx = (int)threadIdx.x + i * NT, row = idx / 8, u = idx % 8;
      *reinterpret_cast<u32x4*>(lds + row * kStageBytes + ((u ^ ((row >> 1) & 7)) << 4)) = r[i];
    }
  }
  // fragment of rows [m0, m0 + 16), half s of the stage
  static __device__ __forceinline__ u32x4 frag(const char* lds, int m0, int s) {
    const int lane = (int)threadIdx.x % 64, row = m0 + lane % 16;
    return *reinterpret_cast<const u32x4*>(lds + row * kStageBytes + (((s * 4 + lane / 16) ^ ((row >> 1) & 7)) << 4));
  }
};

// A tile of COLS columns with k across the rows. Columns past the operand's
// last reach results that are not stored only; rows of k past the end are zero.
// In LDS a row of k is COLS elements and a pad that spreads the rows of a
// fragment read over the banks: bf16 fragments take the rows of k in fours
// (ds_read_b64_tr_b16: lane i of 16 gives the address of 4 columns of row i / 4
// and receives the 4 rows of column i), fp32 ones a word per row.
template <typename T, int COLS, int NT>
struct ColTile {
  static constexpr int kRowUnits = COLS * (int)sizeof(T) / 16;
  static constexpr int kUnits = kStage<T> * kRowUnits / NT;
  static constexpr int kPitch = COLS * (int)sizeof(T) + (sizeof(T) == 2 ? 32 : 16);
  static constexpr int kBytes = kStage<T> * kPitch + (sizeof(T) == 2 ? 8 * 128 : 0);
  static_assert(kStage<T> * kRowUnits % NT == 0 && NT % kRowUnits == 0, "whole units per thread");
  const T* p;       // the thread's column in row 0 of k
  int64_t ld;
  int n;            // columns of the thread's unit that exist (kVec: all; 0: none)
  bool narrow;      // fewer columns than a unit holds
  int k_end;
  const uint8_t* live;   // rows of k to take (others are zero, whatever they hold), or NULL: all
  u32x4 r[kUnits];

  static __device__ __forceinline__ int at(int k) {
    return k * kPitch + (sizeof(T) == 2 ? (k >> 3) * 128 : 0);
  }
  // columns [first, C) of the operand, rows of k [.., k_end_) (k_end_ >= 1)
  __device__ __forceinline__ void init(const T* base, int64_t ld_, int first, int C, int k_end_,
                                       const uint8_t* live_ = nullptr) {
    ld = ld_;
    k_end = k_end_;
    live = live_;
    const int c = first + ((int)threadIdx.x % kRowUnits) * kVec<T>;
    n = C - c;
    n = n > kVec<T> ? kVec<T> : (n < 0 ? 0 : n);
    narrow = C < kVec<T>;
    // a unit that the operand's columns end in (or before) is read so that it ends with them
    p = base + (n == kVec<T> ? c : (narrow ? 0 : C - kVec<T>));
  }
  // rows of k [k0, k0 + stage)
  __device__ __forceinline__ void load(int64_t k0) {
    const bool whole = k0 + kStage<T> <= k_end;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int64_t k = k0 + ((int)threadIdx.x + i * NT) / kRowUnits;
      if ((!whole && k >= k_end) || (live && !live[k])) {
        r[i] = u32x4{0, 0, 0, 0};
        continue;
      }
      const T* q = p + k * ld;
      if (n == kVec<T>) r[i] = load16(q);
      else if (!narrow) r[i] = keep_last<T>(load16(q), n);
      else r[i] = n > 0 ? load_few(q, n) : u32x4{0, 0, 0, 0};
    }
  }
  __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int idx = (int)threadIdx.x + i * NT;
      *reinterpret_cast<u32x4*>(lds + at(idx / kRowUnits) + (idx % kRowUnits) * 16) = r[i];
    }
  }
  static __device__ __forceinline__ u32x4 frag(const char* lds, int m0, int s) {
    const int lane = (int)threadIdx.x % 64, i = lane % 16, g = lane / 16;
    if constexpr (sizeof(T) == 2) {
      const char* q = lds + at(s * 32 + g * 8 + i / 4) + (m0 + (i % 4) * 4) * 2;
      typedef __attribute__((address_space(3))) s16x4 lds4;
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(q));
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(q + 4 * kPitch));
      return __builtin_bit_cast(u32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      u32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = *reinterpret_cast<const uint32_t*>(lds + at(s * 16 + g * 4 + j) + (m0 + i) * 4);
      return v;
    }
  }
};

// acc[r] += sum over the fragment's k of Q[4 (lane / 16) + r] P[lane % 16]
template <typename T>
__device__ __forceinline__ f32x4 mma(u32x4 q, u32x4 p, f32x4 acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, q), __builtin_bit_cast(bf16x8, p), acc, 0,
                                                   0, 0);
  } else {
    const f32x4 a = __builtin_bit_cast(f32x4, q), b = __builtin_bit_cast(f32x4, p);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], acc, 0, 0, 0);
    return acc;
  }
}

// Block shape: WM x WN waves, each MI x NJ fragments of 16 x 16.
template <int WM_, int WN_, int MI_, int NJ_>
struct Shape {
  static constexpr int WM = WM_, WN = WN_, MI = MI_, NJ = NJ_;
  static constexpr int NT = WM * WN * 64, BM = WM * MI * 16, BN = WN * NJ * 16;
};

// The sum over stages [0, steps) of P and Q. Two LDS buffers: a stage is loaded
// into registers while the one before it is multiplied, then written to the
// other buffer. `first`: row of k of the column tiles' stage 0.
// ONES: also sums P alone over k, into sum[i] (lanes of one m hold the same value).
template <typename T, class S, class P, class Q, bool ONES>
__device__ __forceinline__ void sum_stages(P& p, Q& q, char* lds, int steps, f32x4 (&acc)[S::MI][S::NJ],
                                           f32x4 (&sum)[S::MI], bool ones, int64_t p0, int64_t p_step, int64_t q0,
                                           int64_t q_step) {
  constexpr int kBuf = P::kBytes + Q::kBytes;
  const int wave = (int)threadIdx.x / 64, m0 = (wave / S::WN) * S::MI * 16, n0 = (wave % S::WN) * S::NJ * 16;
  if (steps <= 0) return;
  const uint32_t one = sizeof(T) == 2 ? 0x3f803f80u : 0x3f800000u;
  const u32x4 all_one = {one, one, one, one};
  p.load(p0);
  q.load(q0);
  p.store(lds);
  q.store(lds + P::kBytes);
  __syncthreads();
  for (int kt = 0; kt < steps; ++kt) {
    const char* at = lds + (kt & 1) * kBuf;
    const bool more = kt + 1 < steps;
    if (more) {
      p.load(p0 + (kt + 1) * p_step);
      q.load(q0 + (kt + 1) * q_step);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 a[S::MI], b[S::NJ];
#pragma unroll
      for (int i = 0; i < S::MI; ++i) a[i] = P::frag(at, m0 + i * 16, s);
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) b[j] = Q::frag(at + P::kBytes, n0 + j * 16, s);
#pragma unroll
      for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) acc[i][j] = mma<T>(b[j], a[i], acc[i][j]);
      if constexpr (ONES) {
        if (ones) {
#pragma unroll
          for (int i = 0; i < S::MI; ++i) sum[i] = mma<T>(all_one, a[i], sum[i]);
        }
      }
    }
    if (more) {
      char* to = lds + ((kt + 1) & 1) * kBuf;
      p.store(to);
      q.store(to + P::kBytes);
    }
    __syncthreads();
  }
}

// ---- groups ----------------------------------------------------------------

struct Part {          // a run of `step` rows of a group
  int g, index, count;   // its group; its place among the group's runs, and how many those are
  int before;            // runs of the groups before it
  int lo, hi;            // its rows
};

// Run `want` of the groups' rows cut into runs of `step`, counted through the
// groups in order; also looks the whole CSR over. False: there is no such run,
// or the CSR is broken (`bad`). Every wave finds it for itself, 64 groups at a
// time; the answer is the same in all lanes.
__device__ __forceinline__ bool find_part(const int32_t* off, int G, int n, int step, int want, Part& part, bool& bad) {
  bad = false;
  if (!off) {
    part = Part{0, want, (int)(((int64_t)n + step - 1) / step), 0, 0, 0};
    if (want >= part.count) return false;
    part.lo = want * step;
    part.hi = n - part.lo > step ? part.lo + step : n;
    return true;
  }
  const int lane = (int)threadIdx.x % 64;
  int total = 0;
  bool found = false;
  for (int base = 0; base < G; base += 64) {
    const int g = base + lane;
    const int a = g < G ? off[g] : 0, b = g < G ? off[g + 1] : 0;
    const bool wrong = a < 0 || b < a || b > n || (g == 0 && a != 0);
    bad |= __ballot(wrong) != 0;
    if (bad) return false;
    const int t = (int)(((int64_t)(b - a) + step - 1) / step);
    int s = t;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(s, d);
      if (lane >= d) s += o;
    }
    const uint64_t hit = __ballot(want < total + s);
    if (!found && hit) {
      found = true;
      const int l = (int)__builtin_ctzll(hit);
      const int lo = __builtin_amdgcn_readlane(a, l), hi = __builtin_amdgcn_readlane(b, l);
      part.g = base + l;
      part.count = __builtin_amdgcn_readlane(t, l);
      part.before = total + __builtin_amdgcn_readlane(s, l) - part.count;
      part.index = want - part.before;
      part.lo = lo + part.index * step;
      part.hi = hi - part.lo > step ? part.lo + step : hi;
    }
    total += __builtin_amdgcn_readlane(s, 63);
  }
  return found;
}

// Runs of group g (part.before, part.count); false where the CSR is broken.
__device__ __forceinline__ bool find_group(const int32_t* off, int G, int n, int step, int g, Part& part) {
  if (!off) {
    part = Part{0, 0, (int)(((int64_t)n + step - 1) / step), 0, 0, n};
    return true;
  }
  const int lane = (int)threadIdx.x % 64;
  int before = 0;
  for (int base = 0; base < G; base += 64) {
    const int h = base + lane;
    const int a = h < G ? off[h] : 0, b = h < G ? off[h + 1] : 0;
    const bool wrong = a < 0 || b < a || b > n || (h == 0 && a != 0);
    if (__ballot(wrong) != 0) return false;
    const int t = (int)(((int64_t)(b - a) + step - 1) / step);
    int s = h < g ? t : 0;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
    before += s;
    if (g >= base && g < base + 64) part.count = __builtin_amdgcn_readlane(t, g - base);
  }
  part.g = g;
  part.before = before;
  return true;
}

// Tile (row, column) of block `b` of rows x cols tiles: the blocks of an XCD
// (b % 8) take neighbouring tiles, eight rows of tiles at a time, so that those
// running together share operands in its L2.
__device__ __forceinline__ void tile_of(int b, int rows, int cols, int& row, int& col) {
  const int total = rows * cols, each = total / 8, more = total % 8, x = b % 8;
  const int at = x * each + (x < more ? x : more) + b / 8;
  const int band = at / (8 * cols), first = band * 8, high = rows - first < 8 ? rows - first : 8;
  const int in = at - band * 8 * cols;
  row = first + in % high;
  col = in / high;
}

}  // namespace learn
}  // namespace im
