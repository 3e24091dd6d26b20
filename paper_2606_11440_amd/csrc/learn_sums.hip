// Sums over rows: the gradients of weights and biases. The rows of a group are
// cut into chunks, so that a few small matrices over many rows still fill the
// card; a group of one chunk stores its gradient at once, the others' chunks
// are joined in their order by a second kernel (no atomics: the same bits each
// time).
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

template <typename T, class S>
__global__ __launch_bounds__(S::NT, S::MI * S::NJ >= 32 ? 2 : 3) void sums_kernel(const SumArgs a) {
  using P = ColTile<T, S::BM, S::NT, S::D, S::SB>;
  using Q = ColTile<T, S::BN, S::NT, S::D, S::SB>;
  using Product = Sum<T, S, P, Q, true>;
  __shared__ __attribute__((aligned(16))) char lds[2 * Product::kBuf];
  // the tiles of a chunk follow one another, so that they share its rows in an XCD's L2
  int chunk, tile;
  {
    const int tiles = a.row_tiles * a.col_tiles, total = a.chunks * tiles, each = total / 8, more = total % 8;
    const int x = blockIdx.x % 8, at = x * each + (x < more ? x : more) + (int)blockIdx.x / 8;
    chunk = at / tiles;
    tile = at % tiles;
  }
  const int rt = tile / a.col_tiles, ct = tile % a.col_tiles;
  Part part;
  bool bad;
  const bool found = find_part(a.offsets, a.G, a.n, a.chunk, chunk, part, bad);
  if (bad && blockIdx.x == 0 && threadIdx.x == 0 && a.error) atomicOr(a.error, IM_ERR_COUNT);
  if (!found) return;

  const int m_first = rt * S::BM, n_first = ct * S::BN, rows = part.hi - part.lo;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, wm = wave / S::WN, wn = wave % S::WN;
  const bool bias = a.db && ct == 0 && wn == 0;
  // rows to leave out are looked at one by one only where the chunk has any
  const uint8_t* live = nullptr;
  if (a.live) {
    int out = 0;
    for (int i = part.lo + (int)threadIdx.x; i < part.hi; i += S::NT) out |= !a.live[i];
    if (__syncthreads_or(out)) live = a.live;
  }
  Product x;
  x.lds = lds;
  x.steps = (rows + P::kStage - 1) / P::kStage;
  x.alone = bias;
  x.p.init(static_cast<const T*>(a.P), a.ldp, m_first, a.M, part.lo, part.hi, (int)threadIdx.x);
  x.q.init(static_cast<const T*>(a.Q), a.ldq, n_first, a.N, part.lo, part.hi, (int)threadIdx.x, live);
  x.begin();   // a run of rows is not empty
  x.first_stage();
  x.run();
  auto& acc = x.acc;
  auto& sum = x.sum;

  const bool only = part.count == 1;
  float* to = only ? nullptr : a.part + (int64_t)chunk * a.part_width;
  T* dW = static_cast<T*>(a.dW) + part.g * a.w_group;
#pragma unroll
  for (int i = 0; i < S::MI; ++i) {
    const int m = m_first + (wm * S::MI + i) * 16 + lane % 16;
    if (bias) {
      sum[i] += __shfl_xor(sum[i], 16);
      sum[i] += __shfl_xor(sum[i], 32);
      if (lane < 16 && m < a.M) (only ? a.db + (int64_t)part.g * a.M : to + a.db_at)[m] = sum[i];
    }
    if (m >= a.M) continue;
    if (!a.dW) continue;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
      const int n = n_first + (wn * S::NJ + j) * 16 + (lane / 16) * 4, left = a.N - n;
      if (left <= 0) continue;
      if (only) store_some(dW + (int64_t)m * a.N + n, acc[i][j], left);
      else store_some(to + (int64_t)m * a.N + n, acc[i][j], left);
    }
  }
}

// Joins the chunks of the groups that have none (zeros) or several. A thread
// takes four neighbouring elements.
template <typename T>
__global__ __launch_bounds__(256) void join_chunks_kernel(const SumArgs a) {
  Part part;
  const int g = blockIdx.y;
  if (!find_group(a.offsets, a.G, a.n, a.chunk, g, part) || part.count == 1) return;
  const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, mn = (int64_t)a.M * a.N;
  if (e >= a.db_at + a.M) return;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  const f32x4* from = reinterpret_cast<const f32x4*>(a.part + part.before * a.part_width + e);
  const int64_t step = a.part_width / 4;
  int c = 0;
  for (; c + 4 <= part.count; c += 4) {
    const f32x4 x0 = from[c * step], x1 = from[(c + 1) * step], x2 = from[(c + 2) * step], x3 = from[(c + 3) * step];
    v += x0;
    v += x1;
    v += x2;
    v += x3;
  }
  for (; c < part.count; ++c) v += from[c * step];
  if (e < a.db_at) {
    const int64_t left = mn - e;
    if (a.dW && left > 0) store_some(static_cast<T*>(a.dW) + g * a.w_group + e, v, left < 4 ? (int)left : 4);
  } else if (a.db) {
    const int64_t m = e - a.db_at, left = a.M - m;
    store_some(a.db + (int64_t)g * a.M + m, v, left < 4 ? (int)left : 4);
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

template <typename T, class S>
hipError_t launch(const SumArgs& a, hipStream_t s) {
  if (a.chunks > 0) {
    hipLaunchKernelGGL((sums_kernel<T, S>), dim3((unsigned)(a.chunks * a.row_tiles * a.col_tiles)), dim3(S::NT), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.offsets && a.chunks == 1) return hipSuccess;   // one group of one chunk: stored already
  const int64_t quads = (a.db_at + a.M + 3) / 4;
  hipLaunchKernelGGL(join_chunks_kernel<T>, dim3((unsigned)((quads + 255) / 256), (unsigned)a.G), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_type(const SumArgs& a, int shape, hipStream_t s) {
  switch (shape) {
    case 0: return launch<T, Large>(a, s);
    case 1: return launch<T, Middle>(a, s);
    default: return launch<T, Small>(a, s);
  }
}

}  // namespace

int rows_per_sum(int shape) { return shape == 0 ? Large::BM : (shape == 1 ? Middle::BM : Small::BM); }

SumPlan plan_sums(int dtype, int64_t n, int64_t G, int64_t M, int64_t N, int cus) {
  SumPlan p;
  const int64_t least = M < N ? M : N;
  p.shape = least > 128 ? 0 : (least > 64 ? 1 : 2);
  const int b = p.shape == 0 ? Large::BM : (p.shape == 1 ? Middle::BM : Small::BM);
  const int per_cu = p.shape == 0 ? 1 : (p.shape == 1 ? 2 : 4);
  p.row_tiles = (M + b - 1) / b;
  p.col_tiles = (N + b - 1) / b;
  const int64_t want = (2 * per_cu * cus + p.row_tiles * p.col_tiles - 1) / (p.row_tiles * p.col_tiles);
  const int64_t stage = kHalf / (dtype == IM_BF16 ? 2 : 4);
  int64_t chunk = (n + want - 1) / want;
  if (chunk < 8 * stage) chunk = 8 * stage;
  p.chunk = (chunk + stage - 1) / stage * stage;
  p.chunks = n > 0 ? (n + p.chunk - 1) / p.chunk + G - 1 : 0;
  return p;
}

hipError_t launch_sums(const SumArgs& a, int dtype, int shape, hipStream_t s) {
  return dtype == IM_BF16 ? launch_type<__bf16>(a, shape, s) : launch_type<float>(a, shape, s);
}

hipError_t launch_bias_sum(const int32_t* offsets, int G, int n, int step, const float* part, int64_t width, float* db,
                           hipStream_t s) {
  hipLaunchKernelGGL(bias_sum_kernel, dim3((unsigned)((width + 15) / 16), (unsigned)G), dim3(1024), 0, s, offsets, G, n,
                     step, part, width, db);
  return hipGetLastError();
}

}  // namespace learn
}  // namespace im
