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
// A stage is SB = 64 or 128 bytes of k. Fragments are those of
// v_mfma_f32_16x16x32_bf16: lane l holds row l % 16, 8 values of k from
// 8 (l / 16). For fp32 a fragment is 4 values of k from 4 (l / 16), used by
// four v_mfma_f32_16x16x4_f32 in turn (the sum runs over the same k in another
// order). Products go in with the operands swapped, so that a lane's four
// results are four neighbouring n of one m.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "inframind_learn.h"

namespace im {
namespace learn {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));   // gfx950 loads 16 bytes from any address
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

template <typename T> constexpr int kVec = 16 / (int)sizeof(T);   // elements of a 16-byte unit
constexpr int kHalf = 64;                                          // bytes of k that a fragment covers

// A unit of results where x is above zero (neither NaN), else zeros. bf16: the
// numbers above zero are the 16-bit integers 1 .. 0x7f80 (infinity), so five
// packed integer operations make a factor of 1 or 0 for the bits of two results.
template <typename T>
__device__ __forceinline__ u32x4 where_positive(u32x4 v, u32x4 x) {
  if constexpr (sizeof(T) == 2) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    typedef short i16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t xi = x[i], vi = v[i];
      const u16x2 m = __builtin_bit_cast(u16x2, __builtin_elementwise_max(__builtin_bit_cast(i16x2, xi), i16x2{0, 0}));
      const u16x2 number = __builtin_elementwise_sub_sat(u16x2{0x7f81, 0x7f81}, m);   // 0: NaN
      const u16x2 one = __builtin_elementwise_min(__builtin_elementwise_min(m, number), u16x2{1, 1});
      const u16x2 out = __builtin_bit_cast(u16x2, vi) * one;
      v[i] = __builtin_bit_cast(uint32_t, out);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t xi = x[i];
      v[i] = __builtin_bit_cast(float, xi) > 0.f ? v[i] : 0u;
    }
  }
  return v;
}

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

// The thread's number, as a value the compiler takes for new each time: what
// follows from it is worked out where it is used, not kept in registers through
// a block's loop over its tiles.
__device__ __forceinline__ int fresh_thread() {
  int t = (int)threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

__device__ __forceinline__ int clamp_units(int n, int most) { return n < 0 ? 0 : (n > most ? most : n); }

// A tile of ROWS memory rows with k contiguous, staged by NT threads, D stages
// in flight in registers. Rows past the operand's last are read from its last
// row: they reach results that are not stored only. A unit that the row ends in
// is read so that it ends with the row, and moved into place on the way to LDS
// (no load depends on a branch: the waits count loads). In LDS unit u of row r
// lies at u ^ key(r), so that the 16 lanes of a fragment read that are served
// together (a quarter wave, or four lanes of each quarter) touch all 64 banks
// once.
template <typename T, int ROWS, int NT, int D, int SB>
struct RowTile {
  static constexpr int kRowUnits = SB / 16, kStage = SB / (int)sizeof(T);
  static constexpr int kUnits = ROWS * kRowUnits / NT;
  static constexpr int kBytes = ROWS * SB;
  static_assert(ROWS * kRowUnits % NT == 0 && NT % kRowUnits == 0, "whole units per thread");
  const char* base;         // of the tile's first row (uniform)
  uint32_t p[kUnits];       // byte offsets of the thread's units
  u32x4 r[D][kUnits];
  int K, tid;

  static __device__ __forceinline__ int key(int row) {
    return SB == 128 ? (row >> 1) & 7 : (4 - (row >> 2)) & 3;
  }
  __device__ __forceinline__ int unit() const { return tid % kRowUnits; }
  // rows [first, last] of the operand are the tile's: first <= last (which may be nearer than ROWS - 1)
  __device__ __forceinline__ void init(const T* from, int64_t ld, int64_t first, int64_t last, int K_, int tid_) {
    K = K_;
    tid = tid_;
    base = reinterpret_cast<const char*>(from + first * ld);
    const int most = last - first < ROWS ? (int)(last - first) : ROWS - 1;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int row = (tid + i * NT) / kRowUnits;
      p[i] = ((uint32_t)(row < most ? row : most) * (uint32_t)ld + unit() * kVec<T>) * (uint32_t)sizeof(T);
    }
  }
  __device__ __forceinline__ int whole() const { return K / kStage; }   // stages without an end inside
  __device__ __forceinline__ int left(int kt) const { return K - kt * kStage - unit() * kVec<T>; }
  __device__ __forceinline__ const T* at(int kt, uint32_t off) const {
    return reinterpret_cast<const T*>(base + (int64_t)kt * SB + off);
  }
  template <int SLOT>
  __device__ __forceinline__ void load_whole(int kt) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) r[SLOT][i] = load16(at(kt, p[i]));
  }
  template <int SLOT>
  __device__ __forceinline__ void load(int kt) {
    const int n = left(kt);
    if (K >= kVec<T>) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) r[SLOT][i] = load16(at(kt, p[i]) + (n < kVec<T> ? n - kVec<T> : 0));
    } else {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) r[SLOT][i] = n > 0 ? load_few(at(kt, p[i]), n) : u32x4{0, 0, 0, 0};
    }
  }
  template <int SLOT>
  __device__ __forceinline__ void store(int kt, char* lds) {
    if ((kt + 1) * kStage > K && K >= kVec<T>) {
      const int n = clamp_units(left(kt), kVec<T>);
#pragma unroll
      for (int i = 0; i < kUnits; ++i) r[SLOT][i] = keep_last<T>(r[SLOT][i], n);
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int row = (tid + i * NT) / kRowUnits;
      *reinterpret_cast<u32x4*>(lds + row * SB + ((unit() ^ key(row)) << 4)) = r[SLOT][i];
    }
  }
  // fragment of rows [m0, m0 + 16), half s of the stage
  static __device__ __forceinline__ u32x4 frag(const char* lds, int m0, int s, int lane) {
    const int row = m0 + lane % 16;
    return *reinterpret_cast<const u32x4*>(lds + row * SB + (((s * 4 + lane / 16) ^ key(row)) << 4));
  }
};

// A tile of COLS columns with k across the rows. Columns past the operand's
// last reach results that are not stored only; rows of k past the end are zero.
// In LDS a row of k is COLS elements and a pad that spreads the rows of a
// fragment read over the banks: bf16 fragments take the rows of k in fours
// (ds_read_b64_tr_b16: lane i of 16 gives the address of 4 columns of row i / 4
// and receives the 4 rows of column i), fp32 ones a word per row.
template <typename T, int COLS, int NT, int D, int SB>
struct ColTile {
  static constexpr int kRowUnits = COLS * (int)sizeof(T) / 16, kStage = SB / (int)sizeof(T);
  static constexpr int kUnits = kStage * kRowUnits / NT;
  static constexpr int kEvery = NT / kRowUnits;   // rows of k between a thread's units
  static constexpr int kPitch = COLS * (int)sizeof(T) + (sizeof(T) == 2 ? 32 : 16);
  static constexpr int kBytes = kStage * kPitch + (sizeof(T) == 2 ? kStage / 8 * 128 : 0);
  static_assert(kStage * kRowUnits % NT == 0 && NT % kRowUnits == 0, "whole units per thread");
  const T* p;            // the thread's column in its first row of k
  int64_t ld;
  int first, n;          // its first row; columns of its units that exist (kVec: all; 0: none)
  bool edge, narrow;     // the operand's columns end inside the tile; there are fewer than a unit holds
  int k0, k_end;         // rows of k [k0, k_end) are summed
  const uint8_t* live;   // rows of k to take (others are zero, whatever they hold), or NULL: all
  u32x4 r[D][kUnits];
  int tid;

  static __device__ __forceinline__ int at(int k) {
    return k * kPitch + (sizeof(T) == 2 ? (k >> 3) * 128 : 0);
  }
  // columns [from, C) of the operand
  __device__ __forceinline__ void init(const T* base, int64_t ld_, int from, int C, int k0_, int k_end_, int tid_,
                                       const uint8_t* live_ = nullptr) {
    ld = ld_;
    tid = tid_;
    k0 = k0_;
    k_end = k_end_;
    live = live_;
    first = tid / kRowUnits;
    const int c = from + (tid % kRowUnits) * kVec<T>;
    n = clamp_units(C - c, kVec<T>);
    edge = from + COLS > C;
    narrow = C < kVec<T>;
    // a unit that the operand's columns end in (or before) is read so that it ends with them
    p = base + (k0 + first) * ld + (n == kVec<T> ? c : (narrow ? 0 : C - kVec<T>));
  }
  __device__ __forceinline__ int whole() const { return live || narrow ? 0 : (k_end - k0) / kStage; }
  template <int SLOT>
  __device__ __forceinline__ void load_whole(int kt) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) r[SLOT][i] = load16(p + (int64_t)(kt * kStage + i * kEvery) * ld);
  }
  template <int SLOT>
  __device__ __forceinline__ void load(int kt) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int k = kt * kStage + i * kEvery, last = k_end - 1 - k0 - first;   // k to read, and the last there is
      const T* q = p + (int64_t)(k < last ? k : last) * ld;
      if (narrow) r[SLOT][i] = n > 0 ? load_few(q, n) : u32x4{0, 0, 0, 0};
      else r[SLOT][i] = load16(q);
      if (live && k <= last && !live[k0 + first + k]) r[SLOT][i] = u32x4{0, 0, 0, 0};
    }
  }
  template <int SLOT>
  __device__ __forceinline__ void store(int kt, char* lds) {
    if (edge && !narrow) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) r[SLOT][i] = keep_last<T>(r[SLOT][i], n);
    }
    if (k0 + (kt + 1) * kStage > k_end) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i)
        if (k0 + first + kt * kStage + i * kEvery >= k_end) r[SLOT][i] = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int idx = tid + i * NT;
      *reinterpret_cast<u32x4*>(lds + at(idx / kRowUnits) + (idx % kRowUnits) * 16) = r[SLOT][i];
    }
  }
  static __device__ __forceinline__ u32x4 frag(const char* lds, int m0, int s, int lane) {
    const int i = lane % 16, g = lane / 16;
    if constexpr (sizeof(T) == 2) {
      const char* q = lds + at(s * 32 + g * 8 + i / 4) + (m0 + (i % 4) * 4) * 2;
      typedef __attribute__((address_space(3))) s16x4 lds4;
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(q));
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(q + 4 * kPitch));
      return __builtin_bit_cast(u32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      u32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const uint32_t*>(lds + at(s * 16 + g * 4 + j) + (m0 + i) * 4);
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

// Sum of a fragment's values of k of one row.
template <typename T>
__device__ __forceinline__ float add_up(u32x4 a) {
  float v = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = a[i];
    if constexpr (sizeof(T) == 2)
      v += __builtin_bit_cast(float, w << 16) + __builtin_bit_cast(float, w & 0xffff0000u);
    else
      v += __builtin_bit_cast(float, w);
  }
  return v;
}

// Block shape: WM x WN waves, each MI x NJ fragments of 16 x 16; D stages of SB bytes in flight.
template <int WM_, int WN_, int MI_, int NJ_, int D_, int SB_>
struct Shape {
  static constexpr int WM = WM_, WN = WN_, MI = MI_, NJ = NJ_, D = D_, SB = SB_;
  static constexpr int kWaves = MI * NJ >= 16 ? 2 : 3;   // a SIMD, by the registers (and LDS) they take
  static constexpr int kBlocks = MI * NJ >= 32 ? 1 : (MI * NJ >= 16 ? 2 : 3);   // a CU
  static constexpr int NT = WM * WN * 64, BM = WM * MI * 16, BN = WN * NJ * 16;
};

// The sum over stages [0, steps) of P and Q, through two LDS buffers: before a
// stage is multiplied the next one, whose loads were issued D stages ago, is
// written to the other buffer, and the loads of the stage D behind it are issued.
// ALONE: also sums P by itself where `alone` is set; sum[i] of the four lanes of
// an m add up to it.
template <typename T, class S, class P, class Q, bool ALONE>
struct Sum {
  static constexpr int kBuf = P::kBytes + Q::kBytes;
  P p;
  Q q;
  char* lds;
  int steps;
  bool alone;
  f32x4 acc[S::MI][S::NJ];
  float sum[ALONE ? S::MI : 1];

  template <int SLOT, bool WHOLE>
  __device__ __forceinline__ void one(int kt) {
    constexpr int kNext = (SLOT + 1) % S::D;   // slot of the next stage, and of the one D behind it
    if (WHOLE || kt + 1 < steps) {
      char* to = lds + ((kt + 1) & 1) * kBuf;
      p.template store<kNext>(kt + 1, to);
      q.template store<kNext>(kt + 1, to + P::kBytes);
    }
    if constexpr (WHOLE) {
      p.template load_whole<kNext>(kt + 1 + S::D);
      q.template load_whole<kNext>(kt + 1 + S::D);
    } else if (kt + 1 + S::D < steps) {
      p.template load<kNext>(kt + 1 + S::D);
      q.template load<kNext>(kt + 1 + S::D);
    }
    const int wave = p.tid / 64, lane = p.tid % 64, m0 = (wave / S::WN) * S::MI * 16, n0 = (wave % S::WN) * S::NJ * 16;
    const char* at = lds + (kt & 1) * kBuf;
#pragma unroll
    for (int s = 0; s < S::SB / kHalf; ++s) {
      u32x4 a[S::MI], b[S::NJ];
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) b[j] = Q::frag(at + P::kBytes, n0 + j * 16, s, lane);
#pragma unroll
      for (int i = 0; i < S::MI; ++i) a[i] = P::frag(at, m0 + i * 16, s, lane);
#pragma unroll
      for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) acc[i][j] = mma<T>(b[j], a[i], acc[i][j]);
      if constexpr (ALONE) {
        if (alone) {
#pragma unroll
          for (int i = 0; i < S::MI; ++i) sum[i] += add_up<T>(a[i]);
        }
      }
    }
    __syncthreads();
  }
  template <int SLOT>
  __device__ __forceinline__ void first_loads() {
    if constexpr (SLOT < S::D) {
      if (SLOT < steps) {
        p.template load<SLOT>(SLOT);
        q.template load<SLOT>(SLOT);
      }
      first_loads<SLOT + 1>();
    }
  }
  template <int SLOT, bool WHOLE>
  __device__ __forceinline__ void round(int kt) {   // D stages from kt on (kt a multiple of D)
    if constexpr (SLOT < S::D) {
      if (!WHOLE && kt >= steps) return;
      one<SLOT, WHOLE>(kt);
      round<SLOT + 1, WHOLE>(kt + 1);
    }
  }
  // A sum in three parts: begin() issues the first loads (p, q and steps set),
  // first_stage() takes the first stage to LDS, run() multiplies.
  __device__ __forceinline__ void begin() { first_loads<0>(); }
  __device__ __forceinline__ void first_stage() {
    p.template store<0>(0, lds);
    q.template store<0>(0, lds + P::kBytes);
    if (S::D < steps) {
      p.template load<0>(S::D);
      q.template load<0>(S::D);
    }
  }
  __device__ __forceinline__ void run() {   // steps >= 1
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (ALONE) sum[i] = 0.f;
    }
    __syncthreads();
    // stages that are whole, as are those D behind them, take no branch
    const int wp = p.whole(), wq = q.whole(), whole = (wp < wq ? wp : wq);
    int kt = 0;
    for (; kt + 2 * S::D + 1 <= whole; kt += S::D) round<0, true>(kt);
    for (; kt < steps; kt += S::D) round<0, false>(kt);
  }
};

// ---- results ----------------------------------------------------------------

// Passes a block's results, rounded to U, through LDS to 16-byte units of a row.
// A fragment's own layout would store 32 bytes of 16 rows at a time; here a wave
// stores whole lines. Unit u of a row lies at u ^ (row % 16), so that neither the
// fragments' writes nor the units' reads meet in a bank. Where the LDS does not
// hold the tile it goes in passes.
//   value(i, j)   the fragment to put, final
//   after()       called when the first pass is in LDS (one pass: acc is free)
//   use(k, m, c, unit)   unit k of the thread's: of tile row m, from column c on
template <typename U, class S, int kLds>
struct Out {
  static constexpr int kPitch = S::BN * (int)sizeof(U), kAcross = kPitch / 16;
  static constexpr int kPasses = S::BM * kPitch <= kLds ? 1 : (S::BM * kPitch <= 2 * kLds ? 2 : 4), kMi = S::MI / kPasses;
  static constexpr int kUnits = S::WM * kMi * 16 * kAcross / S::NT;   // of a thread, a pass
  static_assert(S::WM * kMi * 16 * kPitch <= kLds && S::MI % kPasses == 0, "a pass fits");
  static_assert(S::WM * kMi * 16 * kAcross % S::NT == 0 && S::NT % kAcross == 0, "whole units per thread");
  static __device__ __forceinline__ int key(int row) { return row & (kAcross < 16 ? kAcross - 1 : 15); }

  static __device__ __forceinline__ int row_of(int pass, int k, int tid) {
    const int r = tid / kAcross + k * (S::NT / kAcross);
    return kPasses == 1 ? r : (r / (kMi * 16)) * S::MI * 16 + pass * kMi * 16 + r % (kMi * 16);
  }
  static __device__ __forceinline__ int column_of(int tid) { return tid % kAcross * (16 / (int)sizeof(U)); }

  template <class V, class A, class F>
  static __device__ __forceinline__ void run(char* lds, int tid, V value, A after, F use) {
    const int lane = tid % 64, wave = tid / 64, wm = wave / S::WN, wn = wave % S::WN, g = lane / 16;
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
      if (pass) __syncthreads();
#pragma unroll
      for (int i = 0; i < kMi; ++i) {
        const int r = (wm * kMi + i) * 16 + lane % 16;
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) {
          const f32x4 v = value(pass * kMi + i, j);
          const int at = (wn * S::NJ + j) * 16 + g * 4;
          char* to = lds + r * kPitch + (((at * (int)sizeof(U) / 16) ^ key(r)) << 4);
          if constexpr (sizeof(U) == 2) {
            bf16x4 o;
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = (__bf16)v[q];
            *reinterpret_cast<bf16x4*>(to + (g & 1) * 8) = o;
          } else {
            *reinterpret_cast<f32x4*>(to) = v;
          }
        }
      }
      __syncthreads();
      if (pass == 0) after();
#pragma unroll
      for (int k = 0; k < kUnits; ++k) {
        const int r = tid / kAcross + k * (S::NT / kAcross);
        use(pass * kUnits + k, row_of(pass, k, tid), column_of(tid),
            *reinterpret_cast<const u32x4*>(lds + r * kPitch + ((tid % kAcross ^ key(r)) << 4)));
      }
    }
  }
};

// Some of a unit's values to p (n: how many exist).
template <typename U>
__device__ __forceinline__ void store_few(U* p, u32x4 x, int n) {
  U e[kVec<U>];
  __builtin_memcpy(e, &x, 16);
#pragma unroll
  for (int i = 0; i < kVec<U>; ++i)
    if (i < n) p[i] = e[i];
}
// ---- groups ----------------------------------------------------------------

struct Part {     // the runs of `step` rows of a group
  int count;      // how many
  int before;     // runs of the groups before it
};

// Whether offsets are a CSR of n rows at most. Every wave looks for itself, 64
// groups at a time; the answer is the same in all lanes.
__device__ __forceinline__ bool csr_holds(const int32_t* off, int G, int n) {
  const int lane = (int)threadIdx.x % 64;
  for (int base = 0; base < G; base += 64) {
    const int g = base + lane;
    const int a = g < G ? off[g] : 0, b = g < G ? off[g + 1] : 0;
    const bool wrong = a < 0 || b < a || b > n || (g == 0 && a != 0);
    if (__ballot(wrong) != 0) return false;
  }
  return true;
}

// Runs of group g (part.before, part.count); false where the CSR is broken.
__device__ __forceinline__ bool find_group(const int32_t* off, int G, int n, int step, int g, Part& part) {
  if (!off) {
    part = Part{(int)(((int64_t)n + step - 1) / step), 0};
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
  part.before = before;
  return true;
}

// The groups' rows cut into runs of `step`, counted through the groups in order,
// kept in LDS by a block that takes many of them.
struct Groups {
  int start[IM_MAX_GROUPS + 1];   // runs before group g
  int total;                      // runs; -1: the CSR is broken

  __device__ __forceinline__ void init(const int32_t* off, int G, int n, int step) {
    const int lane = (int)threadIdx.x % 64;
    if (threadIdx.x >= 64) return;
    if (!off) {
      if (lane == 0) {
        start[0] = 0;
        start[1] = total = (int)(((int64_t)n + step - 1) / step);
      }
      return;
    }
    int before = 0;
    bool bad = false;
    for (int base = 0; base < G; base += 64) {
      const int g = base + lane;
      const int a = g < G ? off[g] : 0, b = g < G ? off[g + 1] : 0;
      const bool wrong = a < 0 || b < a || b > n || (g == 0 && a != 0);
      bad |= __ballot(wrong) != 0;
      if (bad) break;
      const int t = (int)(((int64_t)(b - a) + step - 1) / step);
      int s = t;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(s, d);
        if (lane >= d) s += o;
      }
      if (g < G) {
        start[g] = before + s - t;
      }
      before += __builtin_amdgcn_readlane(s, 63);
    }
    if (lane == 0) {
      start[G] = before;
      total = bad ? -1 : before;
    }
  }
  // The group of run `want` (< total) and its rows; the same in all lanes.
  __device__ __forceinline__ void find(const int32_t* off, int G, int n, int step, int want, int& g, int& lo,
                                       int& hi) const {
    const int lane = (int)threadIdx.x % 64;
    g = 0;
    if (G > 1) {   // the last group that starts at or before it
      const int each = (G + 63) / 64, first = lane * each;
      const int c = __builtin_popcountll(__ballot(first < G && start[first < G ? first : 0] <= want));
      const int base = (c - 1) * each, at = base + lane;
      const bool in = lane < each && at < G;
      g = base + __builtin_popcountll(__ballot(in && start[in ? at : 0] <= want)) - 1;
    }
    g = __builtin_amdgcn_readfirstlane(g);
    const int begin = off ? off[g] : 0, end = off ? off[g + 1] : n;
    lo = begin + (want - __builtin_amdgcn_readfirstlane(start[g])) * step;
    hi = end - lo > step ? lo + step : end;
  }
};

// How the parts cut the line of granules.
struct Line {
  int64_t units;
  int64_t parts;   // those that are not empty
  __device__ __forceinline__ int64_t begin(int64_t p) const { return p * units / parts; }
  // the part that granule u falls to
  __device__ __forceinline__ int64_t part_of(int64_t u) const {
    int64_t p = u * parts / units;
    while (p + 1 < parts && begin(p + 1) <= u) ++p;
    while (begin(p) > u) --p;
    return p;
  }
  // of granules [first, end): {first part, last part, 1 if the first one begins before them, 0}
  __device__ __forceinline__ int4 cut(int first, int end) const {
    int4 c = {0, -1, 0, 0};
    if (end > first) {
      c.x = (int)part_of(first);
      c.y = (int)part_of(end - 1);
      c.z = begin(c.x) >= first ? 0 : 1;
    }
    return c;
  }
};

// Tile (row, column) of number `b` of rows x cols tiles: the blocks of an XCD
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
