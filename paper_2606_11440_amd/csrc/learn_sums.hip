// Sums over rows: the gradients of weights and biases. The groups' rows, cut into
// granules, are one line; `parts` equal runs of it are taken by as many blocks
// for every tile of the gradient, so that one small matrix over many rows and
// many ragged groups alike fill the card, and the blocks of a run read the same
// rows at the same time. A group within a run is stored at once; of one that a
// run's end cuts each block keeps its piece (at most two a block: where its run
// begins and where it ends), and a second kernel adds the pieces in their order
// (no atomics: the same bits each time).
//
// Both operands lie with k across their rows, so a stage is 64 bytes of k (32
// rows in bf16) and two stages are in flight: the transposing reads of LDS take
// 4 rows each, and a longer stage would need LDS that the second buffer has.
// Measured, once the clock has settled: 64 ragged groups of 262144 rows, 512 x 512, bf16,
// 170 us and 29 for the join (0.81 PFLOP/s, matrix cores busy 42 %); one piece of a head of
// 50021 classes, 1024 wide, over 8192 rows 212 us (0.99 PFLOP/s, 52 %); 256 x 256 over 16384 rows,
// fp32, 34 us with the join (16.4 at the fp32 rate of the matrix cores). A block
// keeps both accumulators and two stages, so one or two share a CU, and the start
// and end of each group's sum wait. The join reads what the blocks leave.
#include <type_traits>

#include "learn_internal.h"
#include "learn_tile.h"

namespace im {
namespace learn {
namespace {

template <typename T>
__device__ __forceinline__ void store_some(T* p, f32x4 v, int left) {
  typedef T vec __attribute__((ext_vector_type(4)));
  typedef vec any __attribute__((aligned(sizeof(T))));
  vec o;
#pragma unroll
  for (int r = 0; r < 4; ++r) o[r] = (T)v[r];
  if (left >= 4) {
    *reinterpret_cast<any*>(p) = o;
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r < left) p[r] = o[r];
  }
}

// CODES: Q is int8 codes with a scale a row, decoded on their way to LDS: 64 ragged groups of 262144 rows, 512 x
// 512, bf16, 190 us where bf16 rows take 170; the conversions (five operations for two values) are more than
// the half as many bytes save.
template <typename T, class S, bool CODES>
__global__ __launch_bounds__(S::NT, S::MI * S::NJ >= 32 ? 2 : 3) void sums_kernel(const SumArgs a) {
  using P = ColTile<T, S::BM, S::NT, S::D, S::SB>;
  using Q = typename std::conditional<CODES, CodeTile<T, S::BN, S::NT, S::D, S::SB>,
                                      ColTile<T, S::BN, S::NT, S::D, S::SB>>::type;
  using Product = Sum<T, S, P, Q, true>;
  __shared__ __attribute__((aligned(16))) char lds[2 * Product::kBuf];
  __shared__ Groups groups;
  groups.init(a.offsets, a.G, a.n, a.granule);
  __syncthreads();
  if (groups.total < 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.error) atomicOr(a.error, IM_ERR_COUNT);
    if (blockIdx.x == 0 && a.cuts)   // nothing to join
      for (int g = threadIdx.x; g < a.G; g += S::NT) a.cuts[g] = int4{0, 0, 0, 0};
    return;
  }
  const int tiles = a.row_tiles * a.col_tiles;
  Line line;
  line.units = groups.total;
  line.parts = a.parts < groups.total ? a.parts : groups.total;
  if (blockIdx.x == 0 && a.cuts)   // where the parts cut the groups, for the kernel that joins
    for (int g = threadIdx.x; g < a.G; g += S::NT) a.cuts[g] = line.cut(groups.start[g], groups.start[g + 1]);
  if (a.G == 1 && a.parts == 1 && groups.total == 0) {   // an empty group: zeros
    const int rt = blockIdx.x / a.col_tiles, ct = blockIdx.x % a.col_tiles;
    for (int e = threadIdx.x; e < S::BM * S::BN; e += S::NT) {
      const int m = rt * S::BM + e / S::BN, n = ct * S::BN + e % S::BN;
      if (a.dW && m < a.M && n < a.N) static_cast<T*>(a.dW)[(int64_t)m * a.N + n] = T(0.f);
    }
    for (int m = rt * S::BM + threadIdx.x; a.db && ct == 0 && m < a.M && m < (rt + 1) * S::BM; m += S::NT) a.db[m] = 0.f;
    return;
  }
  // the tiles of a part follow one another on one XCD: they share its rows in the L2
  int tile;
  int64_t run;
  {
    const int total = (int)line.parts * tiles, each = total / 8, more = total % 8, x = blockIdx.x % 8;
    if ((int)blockIdx.x >= total) return;
    const int at = x * each + (x < more ? x : more) + (int)blockIdx.x / 8;
    run = at / tiles;
    tile = at % tiles;
  }
  const int begin = (int)line.begin(run), end = (int)line.begin(run + 1);
  for (int u = begin; u < end;) {
    int g, lo, hi;
    groups.find(a.offsets, a.G, a.n, a.granule, u, g, lo, hi);
    const int first = __builtin_amdgcn_readfirstlane(groups.start[g]);
    const int count = __builtin_amdgcn_readfirstlane(groups.start[g + 1]) - first;
    const int k = u - first, length = end - u < count - k ? end - u : count - k;
    const int rows1 = a.offsets ? a.offsets[g + 1] : a.n;
    hi = rows1 - lo > (int64_t)length * a.granule ? lo + length * a.granule : rows1;

    const int rt = tile / a.col_tiles, ct = tile % a.col_tiles;
    const int m_first = rt * S::BM, n_first = ct * S::BN, tid = fresh_thread();
    const int lane = tid % 64, wave = tid / 64, wm = wave / S::WN, wn = wave % S::WN;
    const bool bias = a.db && ct == 0 && wn == 0;
    // rows to leave out are looked at one by one only where there are any
    const uint8_t* live = nullptr;
    if (!CODES && a.live) {
      int out = 0;
      for (int i = lo + tid; i < hi; i += S::NT) out |= !a.live[i];
      if (__syncthreads_or(out)) live = a.live;
    }
    Product x;
    x.lds = lds;
    x.steps = (hi - lo + P::kStage - 1) / P::kStage;
    x.alone = bias;
    x.p.init(static_cast<const T*>(a.P), a.ldp, m_first, a.M, lo, hi, tid);
    if constexpr (CODES) x.q.init(static_cast<const int8_t*>(a.Q), a.scale, a.ldq, n_first, a.N, lo, hi, tid);
    else x.q.init(static_cast<const T*>(a.Q), a.ldq, n_first, a.N, lo, hi, tid, live);
    x.begin();   // a part of the line is not empty
    x.first_stage();
    x.run();
    auto& acc = x.acc;
    if (bias) {
#pragma unroll
      for (int i = 0; i < S::MI; ++i) {
        x.sum[i] += __shfl_xor(x.sum[i], 16);
        x.sum[i] += __shfl_xor(x.sum[i], 32);
      }
    }
    if (length == count) {
      if (bias) {
#pragma unroll
        for (int i = 0; i < S::MI; ++i) {
          const int m = m_first + (wm * S::MI + i) * 16 + lane;
          if (lane < 16 && m < a.M) a.db[(int64_t)g * a.M + m] = x.sum[i];
        }
      }
      if (a.dW) {
        T* const to = static_cast<T*>(a.dW) + g * a.w_group + (int64_t)m_first * a.N + n_first;
        Out<T, S, (int)sizeof(lds)>::run(lds, tid, [&](int i, int j) { return acc[i][j]; }, [] {},
                                         [&](int, int m, int c, u32x4 v) {
          const int left = a.N - n_first - c;
          if (m_first + m >= a.M || left <= 0) return;
          T* const p = to + (int64_t)m * a.N + c;
          if (left >= kVec<T>) *reinterpret_cast<u32x4_any*>(p) = v;
          else store_few(p, v, left);
        });
        __syncthreads();   // the next group's stages take the LDS
      }
    } else {   // as the registers lie
      float* to = a.part + ((2 * run + (u == begin ? 0 : 1)) * tiles + tile) * (S::BM * S::BN + S::BM);
#pragma unroll
      for (int i = 0; i < S::MI; ++i) {
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) *reinterpret_cast<f32x4*>(to + ((i * S::NJ + j) * S::NT + tid) * 4) = acc[i][j];
        if (bias && lane < 16) to[S::BM * S::BN + (wm * S::MI + i) * 16 + lane] = x.sum[i];
      }
    }
    u += length;
  }
}

// Adds the pieces of the groups that several parts cut, and clears the gradient
// of empty groups. `share` threads (a power of two) go through a tile's pieces
// for four neighbouring elements, and add up in a fixed order.
template <typename T, class S>
__global__ __launch_bounds__(256) void join_pieces_kernel(const SumArgs a, int share) {
  __shared__ f32x4 sums[256];
  constexpr int kQuads = (S::BM * S::BN + S::BM) / 4, kTile = S::BM * S::BN / 4;
  const int tiles = a.row_tiles * a.col_tiles, g = blockIdx.z, tile = blockIdx.x;   // only x holds more than 65535
  const int4 cut = a.cuts ? a.cuts[g] : int4{0, -1, 0, 0};   // no rows at all: zeros
  const int p0 = cut.x, p1 = cut.y, from = cut.z;   // its parts; 1: the first of them begins in a group before it
  if (p0 == p1) return;   // stored already
  const int wide = 256 / share, at = (int)threadIdx.x % wide, turn = threadIdx.x / wide;
  const int rt = tile / a.col_tiles, ct = tile % a.col_tiles;
  for (int q0 = blockIdx.y * wide; q0 < kQuads; q0 += gridDim.y * wide) {
    const int q = q0 + at;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    const bool in = q < kTile ? a.dW != nullptr : (q < kQuads && a.db && ct == 0);
    if (in) {
#pragma unroll 4
      for (int p = p0 + turn; p <= p1; p += share)
        v += *reinterpret_cast<const f32x4*>(
            a.part + ((2 * p + (p == p0 ? from : 0)) * (int64_t)tiles + tile) * (S::BM * S::BN + S::BM) + (int64_t)q * 4);
    }
    if (share > 1) {
      __syncthreads();
      sums[threadIdx.x] = v;
      __syncthreads();
      for (int t = 1; t < share; ++t) v += sums[(turn == 0 ? t * wide : 0) + at];
    }
    if (turn != 0 || !in) continue;
    if (q < kTile) {   // (i, j, thread) as the registers lay
      const int tid = q % S::NT, i = q / S::NT / S::NJ, j = q / S::NT % S::NJ;
      const int lane = tid % 64, wave = tid / 64, wm = wave / S::WN, wn = wave % S::WN;
      const int m = rt * S::BM + (wm * S::MI + i) * 16 + lane % 16;
      const int n = ct * S::BN + (wn * S::NJ + j) * 16 + (lane / 16) * 4, left = a.N - n;
      if (m < a.M && left > 0) store_some(static_cast<T*>(a.dW) + g * a.w_group + (int64_t)m * a.N + n, v, left);
    } else {
      const int m = rt * S::BM + (q - kTile) * 4, left = a.M - m;
      if (left > 0) store_some(a.db + (int64_t)g * a.M + m, v, left);
    }
  }
}

// db of a head: column sums of the row tiles' column sums; 64 threads a column.
__global__ __launch_bounds__(1024) void bias_sum_kernel(const int32_t* offsets, int G, int n, int step,
                                                        const float* __restrict__ part, int64_t width, float* db) {
  __shared__ float across[16][17];
  const int g = blockIdx.y, c = threadIdx.x % 16, k = threadIdx.x / 16;
  Part run;
  if (!find_group(offsets, G, n, step, g, run)) return;
  const int64_t col = (int64_t)blockIdx.x * 16 + c;
  float v = 0.f;
  if (col < width) {
    const float* from = part + run.before * width + col;
#pragma unroll 4
    for (int t = k; t < run.count; t += 64) v += from[t * width];
  }
  v += __shfl_xor(v, 16);
  v += __shfl_xor(v, 32);
  if (threadIdx.x % 64 < 16) across[threadIdx.x / 64][c] = v;
  __syncthreads();
  if (threadIdx.x >= 16 || col >= width) return;
  v = across[0][c];
  for (int w = 1; w < 16; ++w) v += across[w][c];
  db[g * width + col] = v;
}

using Large = Shape<2, 4, 8, 4, 2, 64>;    // 256 x 256, 512 threads
using Middle = Shape<2, 2, 4, 4, 2, 64>;   // 128 x 128
using Small = Shape<2, 2, 2, 2, 4, 64>;    // 64 x 64

template <typename T, class S, bool CODES>
hipError_t launch(const SumArgs& a, hipStream_t s) {
  const int tiles = a.row_tiles * a.col_tiles;
  if (a.parts > 0) {
    hipLaunchKernelGGL((sums_kernel<T, S, CODES>), dim3((unsigned)(a.parts * tiles)), dim3(S::NT), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.G == 1 && a.parts == 1) return hipSuccess;   // one group in one part: stored already
  int share = 1;
  while (share < 16 && share * 2 * a.G <= a.parts) share *= 2;
  // blocks for a tile: some thousands in all
  const int quads = (S::BM * S::BN + S::BM) / 4, wide = 256 / share, most = (quads + wide - 1) / wide;
  const int64_t each = 4096 / ((int64_t)tiles * a.G) + 1;
  hipLaunchKernelGGL((join_pieces_kernel<T, S>), dim3((unsigned)tiles, (unsigned)(each < most ? each : most), (unsigned)a.G),
                     dim3(256), 0, s, a, share);
  return hipGetLastError();
}
template <typename T, bool CODES>
hipError_t launch_type(const SumArgs& a, int shape, hipStream_t s) {
  switch (shape) {
    case 0: return launch<T, Large, CODES>(a, s);
    case 1: return launch<T, Middle, CODES>(a, s);
    default: return launch<T, Small, CODES>(a, s);
  }
}

}  // namespace

int rows_per_sum(int shape) { return shape == 0 ? Large::BM : (shape == 1 ? Middle::BM : Small::BM); }
int threads_per_sum(int shape) { return shape == 0 ? Large::NT : (shape == 1 ? Middle::NT : Small::NT); }

// Shape and parts are those with the least time: of the rounds that the blocks
// take, each of the granules of its part at kAlone us a granule for one block on
// a CU and kFull where its CU is full (all measured), and of the epilogues and
// starts of its groups; and with more parts than one of the join's launch and
// latency (kJoin) and its pieces.
// Blocks beside each other on a CU gain little in fp32 and add pieces: the
// candidates are one block a CU, two, up to a full CU, and whole rounds of those.
// Both sides, us of dW with its join: 512 x 512 over 4096 rows, bf16, tiles of 64:
// 1 part 32, 4 (one block a CU) 18, 16 (four) 26, 64 34; tiles of 256: 105 with 1,
// 29 with 8. 256 x 256 over 16384 rows, fp32, tiles of 128: 64 parts (one block a
// CU) 34, 128 37, 32 50; over 262144 rows, bf16: 65 with tiles of 128, 72 of 256, 89
// of 64. 2048 x 2048 over 8192 rows, bf16: 89 with tiles of 256, 94 of 128, 174 of 64.
SumPlan plan_sums(int dtype, int64_t n, int64_t G, int64_t M, int64_t N, int cus) {
  static const int tile[] = {Large::BM, Middle::BM, Small::BM}, per_cu[] = {1, 2, 4};
  static const double kAlone[2][3] = {{7.9, 2.35, 0.83}, {1.55, 0.75, 0.43}};
  static const double kFull[2][3] = {{7.9, 4.7, 3.0}, {1.55, 1.34, 1.19}};
  static const double kEpilogueUs[3] = {8.0, 4.0, 3.0};
  constexpr double kJoin = 8.0;
  const bool half = dtype == IM_BF16;
  const double read = (double)n * (M + N) * (half ? 2 : 4) / 5.4e6;   // us of reading the rows once
  SumPlan best = {};
  double least = 0;
  for (int s = 0; s < 3; ++s) {
    SumPlan p;
    p.shape = s;
    p.row_tiles = (M + tile[s] - 1) / tile[s];
    p.col_tiles = (N + tile[s] - 1) / tile[s];
    p.granule = half ? 64 : 32;
    p.piece = (int64_t)tile[s] * tile[s] + tile[s];
    const int64_t tiles = p.row_tiles * p.col_tiles;
    const int64_t granules = n > 0 ? (n + p.granule - 1) / p.granule + (G > 1 ? G - 1 : 0) : 0;
    // one part; so many that each CU has 1, 2, .. blocks; 2, 3 and 4 rounds of full CUs
    for (int step = 0; step <= per_cu[s] + 3; ++step) {
      const int64_t a_cu = step <= per_cu[s] ? step : (int64_t)per_cu[s] * (step - per_cu[s] + 1);
      int64_t parts = a_cu * cus / tiles;
      if (parts < 1) parts = 1;
      if (parts > granules) parts = granules;
      p.parts = parts;
      double us = 0;
      if (parts > 0) {
        const int64_t blocks = parts * tiles, slots = (int64_t)cus * per_cu[s];
        const int64_t rounds = (blocks + slots - 1) / slots, beside = rounds > 1 ? per_cu[s] : (blocks + cus - 1) / cus;
        const double each = per_cu[s] > 1 ? kAlone[half][s] + (kFull[half][s] - kAlone[half][s]) * (beside - 1) / (per_cu[s] - 1)
                                          : kAlone[half][s];
        us = rounds * ((double)((granules + parts - 1) / parts) * each + kEpilogueUs[s] * (1 + (double)(G - 1) / parts));
        if (us < read) us = read;
        // a part leaves a piece, and one more where a group begins within it
        if (parts > 1) us += kJoin + (double)(parts + (G > 1 ? (G < parts ? G : parts) : 0)) * tiles * p.piece * 4 / 4e6;
      }
      if ((s == 0 && step == 0) || us < least) {
        best = p;
        least = us;
      }
    }
  }
  return best;
}

hipError_t launch_sums(const SumArgs& a, int dtype, int shape, hipStream_t s) {
  if (a.scale) return dtype == IM_BF16 ? launch_type<__bf16, true>(a, shape, s) : launch_type<float, true>(a, shape, s);
  return dtype == IM_BF16 ? launch_type<__bf16, false>(a, shape, s) : launch_type<float, false>(a, shape, s);
}

hipError_t launch_bias_sum(const int32_t* offsets, int G, int n, int step, const float* part, int64_t width, float* db,
                           hipStream_t s) {
  hipLaunchKernelGGL(bias_sum_kernel, dim3((unsigned)((width + 15) / 16), (unsigned)G), dim3(1024), 0, s, offsets, G, n,
                     step, part, width, db);
  return hipGetLastError();
}

}  // namespace learn
}  // namespace im
