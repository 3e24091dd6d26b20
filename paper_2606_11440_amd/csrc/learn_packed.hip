// Rows in 8 bits: packing, unpacking, and the product of packed rows with packed weights.
//
// Pack and unpack are one pass over memory: 262144 rows of 512, bf16, 76 us (5.3 TB/s; 101
// with one row a wave at a time).
// The product goes as that of bf16 rows does (tiles, stages of 128 bytes, blocks that keep taking tiles), on
// v_mfma_i32_16x16x64_i8: twice the operations a byte of LDS, and an exact sum (127^2 65536 is below
// 2^31), which the scales of its row and column multiply once. Large tiles of aligned rows have a kernel
// of their own, below.
#include "learn_internal.h"
#include "learn_tile.h"
#include "wave.h"

namespace im {
namespace learn {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// a launch has less than 2^32 threads in a dimension: past this many blocks they take more rows each
unsigned blocks_of(int64_t n, int rows) {
  const int64_t blocks = (n + rows - 1) / rows, most = 1 << 20;
  return (unsigned)(blocks < most ? blocks : most);
}

template <typename T>
__device__ __forceinline__ void widen(u32x4 v, float (&f)[kVec<T>]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = v[i];
    if constexpr (sizeof(T) == 2) {
      f[2 * i] = __builtin_bit_cast(float, w << 16);
      f[2 * i + 1] = __builtin_bit_cast(float, w & 0xffff0000u);
    } else {
      f[i] = __builtin_bit_cast(float, w);
    }
  }
}

// First element of unit u of a row: the last unit ends with the row (with some elements that the
// one before it has too); a row shorter than a unit is one, taken element by element.
template <typename T>
__device__ __forceinline__ int unit_at(int u, int dim) {
  const int first = u * kVec<T>;
  return first + kVec<T> <= dim || dim < kVec<T> ? first : dim - kVec<T>;
}
template <typename T>
__device__ __forceinline__ u32x4 unit_load(const T* row, int u, int dim) {
  return dim < kVec<T> ? load_few(row, dim) : load16(row + unit_at<T>(u, dim));
}

// Largest magnitude of units, as the bits of a float: they order as magnitudes do, NaN above
// infinity. bf16: two at a time as 16-bit integers.
template <typename T>
struct Most {
  uint32_t v = 0;
  __device__ __forceinline__ void add(u32x4 x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        const uint32_t w = x[i] & 0x7fff7fffu;
        v = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, v), __builtin_bit_cast(u16x2, w)));
      } else {
        const uint32_t w = x[i] & 0x7fffffffu;
        v = w > v ? w : v;
      }
    }
  }
  __device__ __forceinline__ uint32_t bits() const {
    if constexpr (sizeof(T) == 2) return max(v << 16, v & 0xffff0000u);
    else return v;
  }
};

// Largest over L neighbouring lanes (Most's bits: no sign).
template <int L>
__device__ __forceinline__ uint32_t most_across(uint32_t x) {
  int32_t v = (int32_t)x;
  if constexpr (L > 1) v = max(v, dpp<0xB1>(v));     // quad_perm [1,0,3,2]
  if constexpr (L > 2) v = max(v, dpp<0x4E>(v));     // quad_perm [2,3,0,1]
  if constexpr (L > 4) v = max(v, dpp<0x141>(v));    // half-row mirror
  if constexpr (L > 8) v = max(v, dpp<0x140>(v));    // row mirror
  if constexpr (L > 16) v = max(v, xshfl<16>(v));
  if constexpr (L > 32) v = max(v, xshfl<32>(v));
  return (uint32_t)v;
}

struct Scale {
  float scale, inverse;   // not finite: NaN and 0
  __device__ __forceinline__ explicit Scale(uint32_t most) {
    const float top = __builtin_bit_cast(float, most);
    scale = fmaxf(top / 127.f, 0x1p-126f);
    inverse = 1.f / scale;
    if (most >= 0x7f800000u) {
      scale = __builtin_nanf("");
      inverse = 0.f;
    }
  }
};

// Codes of a unit: x times the inverse, rounded to nearest even by adding 1.5 2^23, whose sum's low byte is
// the code (at most 127: scale and inverse are off by half a unit each). keep: below 3/4 other numbers than zero
// count as that.
template <typename T, bool KEEP>
__device__ __forceinline__ void put_codes(int8_t* row, int u, int dim, u32x4 v, const Scale& s) {
#pragma clang fp contract(off)   // the product is rounded before the sum
  if (s.inverse == 0.f) v = u32x4{0, 0, 0, 0};   // no infinity times 0
  float f[kVec<T>];
  widen<T>(v, f);
  uint32_t q[kVec<T>];
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) {
    float p = f[i] * s.inverse;
    if (KEEP) p = f[i] == 0.f ? 0.f : copysignf(fmaxf(fabsf(p), 0.75f), f[i]);
    q[i] = __builtin_bit_cast(uint32_t, p + 12582912.f);
  }
  uint32_t c[kVec<T> / 4];   // four codes each: their low bytes
#pragma unroll
  for (int i = 0; i < kVec<T> / 4; ++i)
    c[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], 0x0c0c0400u),
                                 __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], 0x0c0c0400u), 0x05040100u);
  if (dim < kVec<T>) {
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i)
      if (i < dim) row[i] = (int8_t)(c[i / 4] >> (8 * (i % 4)));
  } else {
    __builtin_memcpy(row + unit_at<T>(u, dim), c, kVec<T>);
  }
}

// L lanes a row, N units a lane and R rows at once, kept in registers between the largest magnitude and
// the codes.
template <typename T, int L, int N, int R, bool KEEP>
__global__ __launch_bounds__(256) void pack_kernel(const PackArgs a) {
  constexpr int kRows = 256 / L;   // of a block, R times
  const int l = (int)threadIdx.x % L, units = (a.dim + kVec<T> - 1) / kVec<T>;
  for (int64_t first = (int64_t)blockIdx.x * (kRows * R); first < a.n; first += (int64_t)gridDim.x * (kRows * R)) {
    const int64_t at = first + (int)threadIdx.x / L;
    u32x4 v[R][N];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t row = at + k * kRows < a.n ? at + k * kRows : a.n - 1;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int u = l + i * L;
        v[k][i] = unit_load<T>(static_cast<const T*>(a.x) + row * a.ld_x, u < units ? u : units - 1, a.dim);
      }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      Most<T> seen;
#pragma unroll
      for (int i = 0; i < N; ++i) seen.add(v[k][i]);
      const uint32_t most = most_across<L>(seen.bits());
      const int64_t row = at + k * kRows;
      if (row >= a.n) continue;   // the last block's other lanes
      const Scale s(most);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int u = l + i * L;
        if (u < units) put_codes<T, KEEP>(a.codes + row * a.ld_codes, u, a.dim, v[k][i], s);
      }
      if (l == 0) a.scale[row] = s.scale;
    }
  }
}

// A block a row, for long rows: they are read again for the codes (from the L2).
template <typename T, bool KEEP>
__global__ __launch_bounds__(1024) void pack_long_kernel(const PackArgs a) {
  __shared__ uint32_t across[16];
  const int units = (a.dim + kVec<T> - 1) / kVec<T>;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* from = static_cast<const T*>(a.x) + row * a.ld_x;
    Most<T> seen;
#pragma unroll 4
    for (int u = threadIdx.x; u < units; u += 1024) seen.add(unit_load<T>(from, u, a.dim));
    uint32_t most = most_across<64>(seen.bits());
    __syncthreads();
    if (threadIdx.x % 64 == 0) across[threadIdx.x / 64] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) most = across[w] > most ? across[w] : most;
    const Scale s(most);
#pragma unroll 4
    for (int u = threadIdx.x; u < units; u += 1024)
      put_codes<T, KEEP>(a.codes + row * a.ld_codes, u, a.dim, unit_load<T>(from, u, a.dim), s);
    if (threadIdx.x == 0) a.scale[row] = s.scale;
  }
}

// x = scale code, L lanes a row.
template <typename T, int L>
__global__ __launch_bounds__(256) void unpack_kernel(const PackArgs a) {
  constexpr int kRows = 256 / L;
  const int l = (int)threadIdx.x % L, units = (a.dim + kVec<T> - 1) / kVec<T>;
  for (int64_t row = (int64_t)blockIdx.x * kRows + (int)threadIdx.x / L; row < a.n; row += (int64_t)gridDim.x * kRows) {
    const float scale = a.scale[row];
    const int8_t* from = a.codes + row * a.ld_codes;
    T* const to = static_cast<T*>(a.out) + row * a.ld_x;
    for (int u = l; u < units; u += L) {
      int8_t q[kVec<T>];
      if (a.dim < kVec<T>) {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) q[i] = i < a.dim ? from[i] : 0;
      } else {
        __builtin_memcpy(q, from + unit_at<T>(u, a.dim), kVec<T>);
      }
      T o[kVec<T>];
#pragma unroll
      for (int i = 0; i < kVec<T>; ++i) o[i] = (T)(scale * (float)q[i]);
      u32x4 v;
      __builtin_memcpy(&v, o, 16);
      if (a.dim < kVec<T>) store_few(to, v, a.dim);
      else *reinterpret_cast<u32x4_any*>(to + unit_at<T>(u, a.dim)) = v;
    }
  }
}

// ---- the product -----------------------------------------------------------------

__device__ __forceinline__ f32x4 load4(const float* p, int left) {
  typedef f32x4 any __attribute__((aligned(4)));
  if (left >= 4) return *reinterpret_cast<const any*>(p);
  f32x4 v;
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = r < left ? p[r] : 0.f;
  return v;
}

// y = act(sx sw sum + b) of one result.
template <bool RELU>
__device__ __forceinline__ float finish(int sum, float sx, float sw, float b) {
  const float v = fmaf((float)sum * sx, sw, b);
  return RELU ? __builtin_elementwise_maximum(v, 0.f) : v;   // NaN stays
}

template <typename U, class S, bool PARTIAL, bool RELU>
__global__ __launch_bounds__(S::NT, S::kWaves) void packed_kernel(const RowArgs a, const PackedScales scales) {
  using T = int8_t;
  using P = RowTile<T, S::BM, S::NT, S::D, S::SB>;
  using Q = RowTile<T, S::BN, S::NT, S::D, S::SB>;
  using Product = Sum<T, S, P, Q, false>;
  __shared__ __attribute__((aligned(16))) char lds[2 * Product::kBuf];
  __shared__ __attribute__((aligned(16))) float sides[PARTIAL ? 4 : S::BM + 2 * S::BN];   // scales of rows, of columns, bias
  __shared__ Groups groups;
  groups.init(a.offsets, a.G, a.n, S::BM);
  __syncthreads();
  if (groups.total < 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.error) atomicOr(a.error, IM_ERR_COUNT);
    return;
  }
  // with several runs of k a tile is as many units of work, one after the other
  const int row_tiles = groups.total, splits = PARTIAL ? a.splits : 1, total = row_tiles * a.col_tiles * splits;
  int tile = blockIdx.x;
  if (tile >= total) return;
  Product x;
  x.lds = lds;
  x.steps = (a.K + P::kStage - 1) / P::kStage;
  int rt, ct, g, lo, hi, split = 0;
  static_assert(S::NT >= S::BM && S::NT >= S::BN, "a thread a row, a thread a column");
  float side[3] = {0.f, 0.f, 0.f};   // the thread's row's and column's
  auto enter = [&](int t) {   // takes tile t: its first loads are on their way
    const int tid = fresh_thread();
    int k0 = 0, K = a.K;
    if constexpr (PARTIAL) {
      split = t % splits;
      t /= splits;
      k0 = split * a.split_k;
      K = a.K - k0 < a.split_k ? a.K - k0 : a.split_k;
      x.steps = (K + P::kStage - 1) / P::kStage;
    }
    tile_of(t, row_tiles, a.col_tiles, rt, ct);
    groups.find(a.offsets, a.G, a.n, S::BM, rt, g, lo, hi);
    x.p.init(static_cast<const T*>(a.A) + k0, a.lda, lo, hi - 1, K, tid);
    x.q.init(static_cast<const T*>(a.B) + g * a.b_group + k0, a.ldb, ct * S::BN, a.N - 1, K, tid);
    x.begin();
    if constexpr (!PARTIAL) {
      const int row = lo + tid < hi ? lo + tid : hi - 1, col = ct * S::BN + tid < a.N ? ct * S::BN + tid : a.N - 1;
      side[0] = scales.x[row];
      side[1] = scales.W[(int64_t)g * a.N + col];
      side[2] = a.bias ? a.bias[(int64_t)g * a.N + col] : 0.f;
    }
  };
  enter(tile);
  x.first_stage();
  while (true) {
    x.run();
    auto& acc = x.acc;
    const int tid = fresh_thread(), lane = tid % 64, wave = tid / 64, g4 = (lane / 16) * 4;
    const int wm = wave / S::WN, wn = wave % S::WN, m_at = wm * S::MI * 16 + lane % 16;
    const int at_lo = lo, at_hi = hi, at_split = split, n_first = ct * S::BN;
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
    if constexpr (PARTIAL) {
      using F = Out<float, S, (int)sizeof(lds)>;
      float* const part = a.part + (int64_t)at_split * a.n * a.N;
      // the sums' bits, moved only
      F::run(lds, tid, [&](int i, int j) { return __builtin_bit_cast(f32x4, acc[i][j]); }, next,
             [&](int, int m, int c, u32x4 v) {
        const int64_t row = (int64_t)at_lo + m;
        const int n = n_first + c, left = a.N - n;
        if (row >= at_hi || left <= 0) return;
        uint32_t* const to = reinterpret_cast<uint32_t*>(part + row * a.N + n);
        if (left >= 4) *reinterpret_cast<u32x4_any*>(to) = v;
        else store_few(to, v, left);
      });
      last(more);
    } else {
      if (tid < S::BM) sides[tid] = side[0];
      if (tid < S::BN) {
        sides[S::BM + tid] = side[1];
        sides[S::BM + S::BN + tid] = side[2];
      }
      __syncthreads();
      float sx[S::MI];
#pragma unroll
      for (int i = 0; i < S::MI; ++i) sx[i] = sides[m_at + i * 16];
      f32x4 out[S::MI][S::NJ];   // in the sums' place
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) {
        const int c = (wn * S::NJ + j) * 16 + g4;
        const f32x4 times = *reinterpret_cast<const f32x4*>(sides + S::BM + c);
        const f32x4 plus = *reinterpret_cast<const f32x4*>(sides + S::BM + S::BN + c);
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) out[i][j][r] = finish<RELU>(acc[i][j][r], sx[i], times[r], plus[r]);
      }
      auto value = [&](int i, int j) { return out[i][j]; };
      using O = Out<U, S, (int)sizeof(lds)>;
      char* const C = reinterpret_cast<char*>(static_cast<U*>(a.C) + (int64_t)at_lo * a.ldc + n_first);
      auto place = [&](int m, int c) { return ((uint32_t)m * (uint32_t)a.ldc + (uint32_t)c) * (uint32_t)sizeof(U); };
      if (at_hi - at_lo == S::BM && n_first + S::BN <= a.N) {   // no branch on the way out
        O::run(lds, tid, value, next, [&](int, int m, int c, u32x4 v) { *reinterpret_cast<u32x4_any*>(C + place(m, c)) = v; });
        last(more);
      } else {
        O::run(lds, tid, value, next, [&](int, int m, int c, u32x4 v) {
          const int left = a.N - n_first - c;
          if (at_lo + m >= at_hi || left <= 0) return;
          U* const to = reinterpret_cast<U*>(C + place(m, c));
          if (left >= kVec<U>) *reinterpret_cast<u32x4_any*>(to) = v;
          else store_few(to, v, left);
        });
        last(more);
      }
    }
    if (!more) break;
  }
}

// The same product for large tiles of rows that are whole 16-byte units at 16-byte addresses: the
// operands go from memory to LDS without registers (global_load_lds_dwordx4), which leaves room for the
// fragments of a stage while the next one's are read. A stage is 64 bytes of k. With B buffers stage t is multiplied
// from registers, t + 1 is read from LDS, those up to t + B - 1 are on their way, and t + B is asked for once every
// wave has t in registers (one barrier a stage). A block's results leave through the last buffer
// while the others take the next tile's first stages.
// What bounds it: LDS (12 fragments read for 32 products, and the operands' writes), which the products
// overlap but for each stage's barrier, and at k of some stages the tile's own start and results. 8192 x 8192 x 8192
// 605 us, 1.82 POP/s (a library product of that size 2.2); 262144 x 512 x 512 of 64 groups 151 us (75 at the rate of
// a copy). Taking rows of products from LDS ahead of the barrier and a wave's priority over its products changed nothing.
//
// The loads are written in assembly, and so are the waits for them: the compiler would have every read of
// LDS wait for all of them. They write no register, and a wave's loads and stores end in their order.
template <int WN, int BUFFERS, int BLOCKS>
struct Deep {
  static constexpr int kThreads = 128 * WN, kRows = 256, kCols = 64 * WN, kBytes = 64, kBuffers = BUFFERS;
  static constexpr int kRowBytes = kRows * kBytes, kBuffer = kRowBytes + kCols * kBytes;
  static constexpr int kLoads = kBuffer / 16 / kThreads, kRowLoads = kRowBytes / 16 / kThreads;   // of a thread, a stage
  static constexpr int kBlocks = BLOCKS, kWaves = BLOCKS * kThreads / 256;   // a CU, a SIMD
  static constexpr int kWN = WN, kOut = 16384;   // bytes of results that leave at a time
  static_assert(kOut + (kRows + 2 * kCols) * 4 <= kBuffer, "they fit the last buffer with the scales");
};

__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t offset, const char* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base)
               : "memory", "m0");
}
template <int LEFT>
__device__ __forceinline__ void wait_loads() {   // until that many are on their way at most
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}
__device__ __forceinline__ void barrier_behind_lds() {   // a barrier behind the wave's own LDS reads and writes
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const char*>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
                                       (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v));
}

template <typename U, class Deep, bool RELU>
__global__ __launch_bounds__(Deep::kThreads, Deep::kWaves) void packed_deep_kernel(const RowArgs a, const PackedScales scales) {
  using S = Shape<2, Deep::kWN, 8, 4, 1, Deep::kBytes>;
  using Tile = RowTile<int8_t, Deep::kRows, Deep::kThreads, 1, Deep::kBytes>;
  static_assert(S::BM == Deep::kRows && S::BN == Deep::kCols && S::NT == Deep::kThreads, "the tile's");
  __shared__ __attribute__((aligned(1024))) char lds[Deep::kBuffers * Deep::kBuffer];
  __shared__ Groups groups;
  groups.init(a.offsets, a.G, a.n, Deep::kRows);
  __syncthreads();
  if (groups.total < 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.error) atomicOr(a.error, IM_ERR_COUNT);
    return;
  }
  const int row_tiles = groups.total, total = row_tiles * a.col_tiles;
  int tile = blockIdx.x;
  if (tile >= total) return;
  char* const outs = lds + (Deep::kBuffers - 1) * Deep::kBuffer;
  float* const sides = reinterpret_cast<float*>(outs + Deep::kOut);   // scales of rows, of columns, bias
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
  const uint32_t place0 = __builtin_amdgcn_readfirstlane(
      (int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds) + (uint32_t)wave * 1024u;
  const int steps = (a.K + Deep::kBytes - 1) / Deep::kBytes, left = a.K - (steps - 1) * Deep::kBytes;   // bytes of the last stage

  // the thread's units of a stage: rows tid / 4 + kThreads / 4 i, the first of A, then of B
  uint32_t off[Deep::kLoads];
  const char *A, *B;
  int rt, ct, g, lo, hi;
  float side[3];
  auto logical = [](int tid) { return (tid % 4) ^ Tile::key(tid / 4); };   // the unit that lies at the thread's place
  auto ask = [&](int t) {   // loads of stage t
    const uint32_t to = place0 + (uint32_t)(t % Deep::kBuffers) * Deep::kBuffer;
    const int64_t k = (int64_t)t * Deep::kBytes;
    uint32_t back = 0;   // units past the end of k are read from its last one, and multiplied by zero
    if (left < Deep::kBytes && t == steps - 1) {
      const int u = logical(fresh_thread()) * 16;
      back = u + 16 > left ? (uint32_t)(u + 16 - left) : 0u;
    }
    const char *pa = uniform(A + k), *pb = uniform(B + k);
#pragma unroll
    for (int i = 0; i < Deep::kLoads; ++i) load_to_lds(to + i * Deep::kThreads * 16, off[i] - back, i < Deep::kRowLoads ? pa : pb);
  };
  auto enter = [&](int t) {   // takes tile t: its first loads are on their way
    const int tid = fresh_thread();
    tile_of(t, row_tiles, a.col_tiles, rt, ct);
    groups.find(a.offsets, a.G, a.n, Deep::kRows, rt, g, lo, hi);
    A = static_cast<const char*>(a.A) + (int64_t)lo * a.lda;
    B = static_cast<const char*>(a.B) + (int64_t)g * a.b_group + (int64_t)ct * Deep::kCols * a.ldb;
    const int rows = hi - lo, cols = a.N - ct * Deep::kCols, u = logical(tid) * 16;
#pragma unroll
    for (int i = 0; i < Deep::kLoads; ++i) {
      const bool of_a = i < Deep::kRowLoads;
      const int r = tid / 4 + (of_a ? i : i - Deep::kRowLoads) * (Deep::kThreads / 4), most = of_a ? rows : cols;
      off[i] = (uint32_t)(r < most ? r : most - 1) * (uint32_t)(of_a ? a.lda : a.ldb) + u;
    }
#pragma unroll
    for (int t0 = 0; t0 + 1 < Deep::kBuffers; ++t0)
      if (t0 < steps) ask(t0);
    const int row = lo + tid < hi ? lo + tid : hi - 1;
    const int col = ct * Deep::kCols + tid < a.N ? ct * Deep::kCols + tid : a.N - 1;
    side[0] = scales.x[row];
    side[1] = scales.W[(int64_t)g * a.N + col];
    side[2] = a.bias ? a.bias[(int64_t)g * a.N + col] : 0.f;
  };

  enter(tile);
  wait_loads<0>();
  barrier_behind_lds();
  if (steps >= Deep::kBuffers) ask(Deep::kBuffers - 1);
  while (true) {
    i32x4 acc[S::MI][S::NJ];
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    const int lane = fresh_thread() % 64, m0 = (wave / S::WN) * S::MI * 16, n0 = (wave % S::WN) * S::NJ * 16;
    u32x4 x[S::MI], w[S::NJ];
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) w[j] = Tile::frag(lds + Deep::kRowBytes, n0 + j * 16, 0, lane);
#pragma unroll
    for (int i = 0; i < S::MI; ++i) x[i] = Tile::frag(lds, m0 + i * 16, 0, lane);
    int buffer = 0;
    for (int t = 0; t < steps; ++t) {
      if (t + 2 >= Deep::kBuffers && t + 1 < steps) {   // stage t + 1 is here (those before the last buffer's are)
        if (t + Deep::kBuffers - 1 < steps) wait_loads<(Deep::kBuffers - 2) * Deep::kLoads>();
        else if (Deep::kBuffers > 3 && t + 2 < steps) wait_loads<Deep::kLoads>();
        else wait_loads<0>();
      }
      barrier_behind_lds();
      if (t + Deep::kBuffers < steps) ask(t + Deep::kBuffers);
      buffer = buffer + 1 == Deep::kBuffers ? 0 : buffer + 1;
      const char* at = lds + buffer * Deep::kBuffer;   // of no stage behind the last one: read, not used
      if (t == steps - 1 && (lane / 16) * 16 >= left) {   // the lane's units lie past the end of k
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) w[j] = u32x4{0, 0, 0, 0};
      }
      u32x4 next[S::NJ];
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) next[j] = Tile::frag(at + Deep::kRowBytes, n0 + j * 16, 0, lane);
#pragma unroll
      for (int i = 0; i < S::MI; ++i) {
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) acc[i][j] = mma<int8_t>(w[j], x[i], acc[i][j]);
        x[i] = Tile::frag(at, m0 + i * 16, 0, lane);
        __builtin_amdgcn_sched_barrier(0);   // the read goes beside the products that follow
      }
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) w[j] = next[j];
    }
    barrier_behind_lds();   // every wave is through with the buffers

    const int tid = fresh_thread(), at_lo = lo, at_hi = hi, n_first = ct * Deep::kCols, g4 = (tid % 64 / 16) * 4;
    if (tid < Deep::kRows) sides[tid] = side[0];
    if (tid < Deep::kCols) {
      sides[Deep::kRows + tid] = side[1];
      sides[Deep::kRows + Deep::kCols + tid] = side[2];
    }
    tile += gridDim.x;
    const bool more = tile < total, full = at_hi - at_lo == Deep::kRows && n_first + Deep::kCols <= a.N;
    if (more) enter(tile);
    barrier_behind_lds();
    // kI rows of fragments at a time, of all the waves' columns or half of each wave's
    constexpr int kJ = 32 * Deep::kCols * (int)sizeof(U) <= Deep::kOut ? 4 : 2;
    constexpr int kPitch = Deep::kWN * kJ * 16 * (int)sizeof(U), kUnits = kPitch / 16, kWaveUnits = kUnits / Deep::kWN;
    constexpr int kI = Deep::kOut / (32 * kPitch);
    static_assert(kI >= 1 && S::MI % kI == 0 && kUnits >= 16, "whole rows");
    char* const C = reinterpret_cast<char*>(static_cast<U*>(a.C) + (int64_t)at_lo * a.ldc + n_first);
#pragma unroll
    for (int pass = 0; pass < S::MI / kI * (S::NJ / kJ); ++pass) {
      const int i0 = pass / (S::NJ / kJ) * kI, j0 = pass % (S::NJ / kJ) * kJ;
#pragma unroll
      for (int i = 0; i < kI; ++i) {
        const float sx = sides[m0 + (i0 + i) * 16 + tid % 16];
        const int r = ((wave / S::WN) * kI + i) * 16 + tid % 16;
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
          const int c = n0 + (j0 + j) * 16 + g4;
          const f32x4 times = *reinterpret_cast<const f32x4*>(sides + Deep::kRows + c);
          const f32x4 plus = *reinterpret_cast<const f32x4*>(sides + Deep::kRows + Deep::kCols + c);
          f32x4 v;
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = finish<RELU>(acc[i0 + i][j0 + j][q], sx, times[q], plus[q]);
          const int byte = (wave % S::WN) * kWaveUnits * 16 + (j * 16 + g4) * (int)sizeof(U);
          char* const to = outs + r * kPitch + (((byte / 16) ^ (r % 16)) << 4) + byte % 16;
          if constexpr (sizeof(U) == 2) {
            bf16x4 o;
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = (__bf16)v[q];
            *reinterpret_cast<bf16x4*>(to) = o;
          } else {
            *reinterpret_cast<f32x4*>(to) = v;
          }
        }
      }
      barrier_behind_lds();
#pragma unroll
      for (int k = 0; k < 32 * kI * kUnits / Deep::kThreads; ++k) {
        const int row = tid / kUnits + k * (Deep::kThreads / kUnits), u = tid % kUnits;
        const u32x4 v = *reinterpret_cast<const u32x4*>(outs + row * kPitch + ((u ^ (row % 16)) << 4));
        const int m = (row / (16 * kI)) * S::MI * 16 + i0 * 16 + row % (16 * kI);
        const int c = (u / kWaveUnits) * S::NJ * 16 + j0 * 16 + (u % kWaveUnits) * kVec<U>;
        char* const to = C + ((uint32_t)m * (uint32_t)a.ldc + (uint32_t)c) * (uint32_t)sizeof(U);
        if (full) {
          *reinterpret_cast<u32x4_any*>(to) = v;
        } else {
          const int some = a.N - n_first - c;
          if (at_lo + m < at_hi && some > 0) {
            if (some >= kVec<U>) *reinterpret_cast<u32x4_any*>(to) = v;
            else store_few(reinterpret_cast<U*>(to), v, some);
          }
        }
      }
      barrier_behind_lds();   // the next rows take the LDS
    }
    if (!more) break;
    if (steps >= Deep::kBuffers) ask(Deep::kBuffers - 1);
    // the other stages were asked for before the stores of a full tile and this one
    constexpr int kStores = Deep::kRows * Deep::kCols * (int)sizeof(U) / 16 / Deep::kThreads;
    static_assert(Deep::kLoads + kStores < 64, "counted by the hardware");
    if (full && steps >= Deep::kBuffers) wait_loads<Deep::kLoads + kStores>();
    else wait_loads<0>();
    barrier_behind_lds();
  }
}

// Joins the runs of k: four columns of a row a thread.
template <typename U>
__global__ __launch_bounds__(256) void join_packed_kernel(const RowArgs a, const PackedScales scales) {
  const int quads = (a.N + 3) / 4;
  int end = a.n;
  if (a.offsets) {
    if (!csr_holds(a.offsets, a.G, a.n)) return;
    end = a.offsets[a.G];
  }
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x, row = idx / quads;
  if (row >= end) return;
  const int n = (int)(idx % quads) * 4, left = a.N - n;
  const int64_t step = (int64_t)a.n * a.N;
  const float* part = a.part + row * a.N + n;
  i32x4 sum = __builtin_bit_cast(i32x4, load4(part, left));
#pragma unroll 4
  for (int s = 1; s < a.splits; ++s) sum += __builtin_bit_cast(i32x4, load4(part + s * step, left));
  int g = 0, over = a.offsets ? a.G : 1;   // the last group that begins at or before the row
  while (over - g > 1) {
    const int mid = (g + over) / 2;
    if (a.offsets[mid] <= row) g = mid;
    else over = mid;
  }
  const f32x4 times = load4(scales.W + (int64_t)g * a.N + n, left);
  const f32x4 plus = a.bias ? load4(a.bias + g * a.bias_group + n, left) : f32x4{0.f, 0.f, 0.f, 0.f};
  const float sx = scales.x[row];
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (r < left)
      static_cast<U*>(a.C)[row * a.ldc + n + r] = (U)(a.relu ? finish<true>(sum[r], sx, times[r], plus[r])
                                                             : finish<false>(sum[r], sx, times[r], plus[r]));
}

using Large = Shape<2, 4, 8, 4, 1, 128>;    // 256 x 256, 512 threads
using Middle = Shape<2, 2, 4, 4, 1, 128>;   // 128 x 128
using Narrow = Shape<4, 1, 2, 4, 1, 128>;   // 128 x 64
using Small = Shape<2, 2, 2, 2, 2, 128>;    // 64 x 64

template <typename U, class S, bool PARTIAL>
hipError_t launch(const RowArgs& a, const PackedScales& p, hipStream_t s) {
  const int tiles = a.row_tiles * a.col_tiles * (PARTIAL ? a.splits : 1), most = a.cus * S::kBlocks;
  const dim3 grid((unsigned)(tiles < most ? tiles : most)), block(S::NT);
  if (PARTIAL || !a.relu) hipLaunchKernelGGL((packed_kernel<U, S, PARTIAL, false>), grid, block, 0, s, a, p);
  else hipLaunchKernelGGL((packed_kernel<U, S, PARTIAL, true>), grid, block, 0, s, a, p);
  return hipGetLastError();
}
template <typename U, class Deep>
hipError_t launch_deep(RowArgs a, const PackedScales& p, hipStream_t s) {
  a.col_tiles = (a.N + Deep::kCols - 1) / Deep::kCols;
  const int tiles = a.row_tiles * a.col_tiles, most = Deep::kBlocks * a.cus;
  const dim3 grid((unsigned)(tiles < most ? tiles : most)), block(Deep::kThreads);
  if (a.relu) hipLaunchKernelGGL((packed_deep_kernel<U, Deep, true>), grid, block, 0, s, a, p);
  else hipLaunchKernelGGL((packed_deep_kernel<U, Deep, false>), grid, block, 0, s, a, p);
  return hipGetLastError();
}
template <typename U>
hipError_t launch_type(const RowArgs& a, const PackedScales& p, int shape, hipStream_t s) {
  if (a.splits > 1) {
    const hipError_t e = shape == 1 ? launch<U, Middle, true>(a, p, s) : launch<U, Small, true>(a, p, s);
    if (e != hipSuccess) return e;
    const int64_t quads = (int64_t)a.n * ((a.N + 3) / 4);
    hipLaunchKernelGGL(join_packed_kernel<U>, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, s, a, p);
    return hipGetLastError();
  }
  const uint64_t all = reinterpret_cast<uintptr_t>(a.A) | reinterpret_cast<uintptr_t>(a.B) | (uint64_t)a.lda |
                       (uint64_t)a.ldb | (uint64_t)a.K;
  // One block a CU of 256 x 256 and four buffers for long sums, two of 256 x 128 and three buffers, whose results and
  // products overlap, for others. Both sides, us with two blocks / one: 8192 x 8192 x 8192 691 / 605, 8192 x 4096 x
  // 4096 153 / 140; k 2048 with ragged experts 168 / 184, 512 with 64 groups 151 / 167.
  if (shape == 0 && all % 16 == 0)
    return a.K >= 4096 ? launch_deep<U, Deep<4, 4, 1>>(a, p, s) : launch_deep<U, Deep<2, 3, 2>>(a, p, s);
  switch (shape) {
    case 0: return launch<U, Large, false>(a, p, s);
    case 1: return launch<U, Middle, false>(a, p, s);
    case 2: return launch<U, Narrow, false>(a, p, s);
    default: return launch<U, Small, false>(a, p, s);
  }
}

template <typename T, int L, int N, int R>
hipError_t pack_rows(const PackArgs& a, hipStream_t s) {
  const dim3 grid(blocks_of(a.n, 256 / L * R)), block(256);
  if (a.keep) hipLaunchKernelGGL((pack_kernel<T, L, N, R, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((pack_kernel<T, L, N, R, false>), grid, block, 0, s, a);
  return hipGetLastError();
}
// R rows at once where there are enough to fill the card so; single ones otherwise.
template <typename T, int L, int N, int R>
hipError_t pack_some(const PackArgs& a, hipStream_t s) {
  return a.n >= 4096 * 64 / L * R ? pack_rows<T, L, N, R>(a, s) : pack_rows<T, L, N, 1>(a, s);
}
template <typename T>
hipError_t pack(const PackArgs& a, hipStream_t s) {
  const int units = (a.dim + kVec<T> - 1) / kVec<T>;
  if (units <= 4) return pack_some<T, 4, 1, 4>(a, s);
  if (units <= 8) return pack_some<T, 8, 1, 4>(a, s);
  if (units <= 16) return pack_some<T, 16, 1, 4>(a, s);
  if (units <= 32) return pack_some<T, 32, 1, 4>(a, s);
  if (units <= 64) return pack_some<T, 64, 1, 4>(a, s);
  if (units <= 128) return pack_some<T, 64, 2, 2>(a, s);
  if (units <= 256) return pack_rows<T, 64, 4, 1>(a, s);
  if (units <= 512) return pack_rows<T, 64, 8, 1>(a, s);
  if (a.keep) hipLaunchKernelGGL((pack_long_kernel<T, true>), dim3(blocks_of(a.n, 1)), dim3(1024), 0, s, a);
  else hipLaunchKernelGGL((pack_long_kernel<T, false>), dim3(blocks_of(a.n, 1)), dim3(1024), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t unpack(const PackArgs& a, hipStream_t s) {
  const int units = (a.dim + kVec<T> - 1) / kVec<T>;
  const dim3 block(256);
  if (units <= 4) hipLaunchKernelGGL((unpack_kernel<T, 4>), dim3(blocks_of(a.n, 64)), block, 0, s, a);
  else if (units <= 16) hipLaunchKernelGGL((unpack_kernel<T, 16>), dim3(blocks_of(a.n, 16)), block, 0, s, a);
  else hipLaunchKernelGGL((unpack_kernel<T, 64>), dim3(blocks_of(a.n, 4)), block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pack(const PackArgs& a, int dtype, hipStream_t s) {
  return dtype == IM_BF16 ? pack<__bf16>(a, s) : pack<float>(a, s);
}
hipError_t launch_unpack(const PackArgs& a, int dtype, hipStream_t s) {
  return dtype == IM_BF16 ? unpack<__bf16>(a, s) : unpack<float>(a, s);
}

// A stage holds twice the k of a bf16 one and takes as long: the shapes are chosen as there. Of 20 sizes the choice took
// 4 % more than the best of the four shapes at most (4096 x 1024 -> 1024: 11.3 us of 16.5, 11.9, 11.5, 13.1; 16384 x
// 2048 -> 4096 in 8 groups 157 of 154, 177, 245, 266) but for one of 64 groups, 512 -> 512, which varied by 7 % between runs, and
// two that 64 x 64 tiles would suit: 300000 x 256 -> 15 34 us (29), 512 rows, 4096 -> 4096 in 8 groups 33 (26).
RowPlan plan_packed(int64_t n, int64_t G, int64_t N, int64_t K, int cus) {
  RowPlan p = plan_rows(IM_BF16, n, G, N, (K + 1) / 2, cus, true);
  p.split_k *= 2;
  return p;
}

hipError_t launch_packed_product(const RowArgs& a, const PackedScales& p, int dtype, int shape, hipStream_t s) {
  return dtype == IM_BF16 ? launch_type<__bf16>(a, p, shape, s) : launch_type<float>(a, p, shape, s);
}

}  // namespace learn
}  // namespace im
