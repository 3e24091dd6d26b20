// Rows to experts and back: the places of (row, choice) pairs ordered by expert, the rows
// sent there, and the weighted sums that return.
//
// The plan is a stable counting sort: pairs of an expert in the blocks and waves before, then ranks within
// 64 pairs by ballots of the experts' bits; 262144 pairs of 64 experts 11 us, its two launches and their latency (2 MB of
// pairs and places), 96 pairs 2.6 us in one. The rest is memory: a row is spread over up to 64 lanes in
// 16-byte units. 65536 rows of 512, bf16: sent to 4 places each 60 us (5.6 TB/s), the weighted sum's gradient
// 116 us (5.1 TB/s); 30011 rows of 387, fp32, summed from 3 places each 37 us (4.7 TB/s; 41
// with the units of a lane one after the other).
#include "learn_internal.h"
#include "learn_tile.h"
#include "wave.h"

namespace im {
namespace learn {
namespace {

// a launch has less than 2^32 threads in a dimension: past this many blocks they take more rows each
unsigned blocks_of(int64_t n, int rows) {
  const int64_t blocks = (n + rows - 1) / rows, most = 1 << 20;
  return (unsigned)(blocks < most ? blocks : most);
}

// ---- the plan ------------------------------------------------------------------

constexpr int kPlanThreads = 512, kPlanWaves = kPlanThreads / 64;

// The pair's expert, -1 for none; `wrong` where it is no expert and not -1.
__device__ __forceinline__ int expert_of(const PlanArgs& a, int64_t pair, int64_t end, bool& wrong) {
  if (pair >= end) return -1;
  const int e = a.expert[pair];
  const bool none = e < 0 || e >= a.E;
  wrong |= none && e != -1;
  return none ? -1 : e;
}

// Pairs of each expert in the pairs of a block.
__global__ __launch_bounds__(kPlanThreads) void count_kernel(const PlanArgs a) {
  __shared__ int32_t count[IM_MAX_GROUPS];
  for (int e = threadIdx.x; e < a.E; e += kPlanThreads) count[e] = 0;
  __syncthreads();
  const int64_t begin = blockIdx.x * a.each, end = begin + a.each < a.pairs ? begin + a.each : a.pairs;
  bool wrong = false;
  for (int64_t p = begin + threadIdx.x; p < end; p += kPlanThreads) {
    const int e = expert_of(a, p, end, wrong);
    if (e >= 0) atomicAdd(&count[e], 1);   // whole numbers: any order
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kPlanThreads) a.count[(int64_t)blockIdx.x * a.E + e] = count[e];
}

// Places of a block's pairs: those of an expert begin behind the experts before it and its
// pairs in the blocks before; each wave has a run of the block's pairs, and goes through it
// 64 at a time. No order depends on time.
__global__ __launch_bounds__(kPlanThreads) void place_kernel(const PlanArgs a) {
  __shared__ int32_t next[kPlanWaves][IM_MAX_GROUPS];   // next place of an expert's pair in a wave's run
  __shared__ int32_t total[IM_MAX_GROUPS], before[IM_MAX_GROUPS], sums[kPlanWaves];
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, E = a.E;
  for (int e = tid; e < E; e += kPlanThreads) {
    total[e] = before[e] = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) next[w][e] = 0;
  }
  __syncthreads();
  const int64_t run = a.each / kPlanWaves, first = blockIdx.x * a.each + wave * run;
  const int64_t end = first + run < a.pairs ? first + run : a.pairs;
  bool wrong = false;
  for (int64_t p = first + lane; p < end; p += 64) {
    const int e = expert_of(a, p, end, wrong);
    if (e >= 0) atomicAdd(&next[wave][e], 1);
  }
  if (wrong && a.error) atomicOr(a.error, IM_ERR_ACTION);
  if (a.blocks > 1) {   // threads share the blocks' counts of an expert
    const int share = kPlanThreads / E > 0 ? kPlanThreads / E : 1;
    for (int e = tid % (share > 1 ? E : kPlanThreads); e < E; e += kPlanThreads) {
      const int part = share > 1 ? tid / E : 0;
      if (part >= share) break;
      int all = 0, mine = 0;
#pragma unroll 8
      for (int b = part; b < a.blocks; b += share) {
        const int c = a.count[(int64_t)b * E + e];
        all += c;
        mine += b < (int)blockIdx.x ? c : 0;
      }
      atomicAdd(&total[e], all);
      atomicAdd(&before[e], mine);
    }
  }
  __syncthreads();
  // offsets: the sum of the experts' totals before each
  constexpr int kEach = IM_MAX_GROUPS / kPlanThreads;
  int mine[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int e = tid * kEach + i;
    mine[i] = 0;
    if (e < E) {
      mine[i] = total[e];
      if (a.blocks == 1) {
#pragma unroll
        for (int w = 0; w < kPlanWaves; ++w) mine[i] += next[w][e];
      }
    }
    sum += mine[i];
  }
  int scan = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(scan, d);
    if (lane >= d) scan += o;
  }
  if (lane == 63) sums[wave] = scan;
  __syncthreads();
  int base = scan - sum;
  for (int w = 0; w < wave; ++w) base += sums[w];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int e = tid * kEach + i;
    if (e < E) {
      if (blockIdx.x == 0) a.offsets[e] = base;
      int at = base + before[e];
#pragma unroll
      for (int w = 0; w < kPlanWaves; ++w) {
        const int c = next[w][e];
        next[w][e] = at;
        at += c;
      }
      base += mine[i];
      if (blockIdx.x == 0 && e == E - 1) a.offsets[E] = base;
    }
  }
  __syncthreads();
  const int bits = 32 - __builtin_clz(E);
  for (int64_t p0 = first; p0 < end; p0 += 64) {
    const int64_t p = p0 + lane;
    const int e = expert_of(a, p, end, wrong);
    uint64_t same = ballot(e >= 0);   // lanes with the same expert
    for (int b = 0; b < bits; ++b) {
      const uint64_t set = ballot((e >> b) & 1);
      same &= (e >> b) & 1 ? set : ~set;
    }
    if (e >= 0) {
      const int at = next[wave][e];
      const int rank = prefix_count(same);
      a.slot[p] = at + rank;
      if ((same >> lane) == 1) next[wave][e] = at + rank + 1;   // the last of them
    } else if (p < end) {
      a.slot[p] = -1;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- rows -----------------------------------------------------------------------

typedef u32x4 u32x4_byte __attribute__((aligned(1)));

// A choice's slot, -1 for none; `wrong` where it is no slot and not -1.
__device__ __forceinline__ int slot_of(const ExchangeArgs& a, int64_t row, int c, bool& wrong) {
  if (c >= a.k) return -1;
  const int s = a.slot[row * a.k + c];
  const bool none = s < 0 || s >= a.n_slots;
  wrong |= none && s != -1;
  return none ? -1 : s;
}

// to[slot] = from_i: rows of `bytes` bytes of elements of E bytes, by T lanes a row. A row is read
// once and written as often as it was chosen. The last 16 bytes of a row are taken whole,
// with some that the lane before it takes too.
template <int E, int T>
__global__ __launch_bounds__(256) void send_kernel(const ExchangeArgs a) {
  const int l = (int)threadIdx.x % T;
  const int bytes = a.dim * E;
  constexpr int kRows = 256 / T;
  bool wrong = false;
  for (int64_t row = (int64_t)blockIdx.x * kRows + (int)threadIdx.x / T; row < a.n; row += (int64_t)gridDim.x * kRows) {
    const char* from = static_cast<const char*>(a.from) + row * a.ld_from * E;
    char* const to = static_cast<char*>(a.to);
    if (bytes >= 16) {
      for (int u = l * 16; u < bytes; u += T * 16) {
        const int at = u + 16 <= bytes ? u : bytes - 16;
        const u32x4 v = *reinterpret_cast<const u32x4_byte*>(from + at);
        for (int c = 0; c < a.k; ++c) {
          const int s = slot_of(a, row, c, wrong);
          if (s >= 0) *reinterpret_cast<u32x4_byte*>(to + (int64_t)s * a.ld_to * E + at) = v;
        }
      }
    } else {
      for (int j = l; j < a.dim; j += T)
        for (int c = 0; c < a.k; ++c) {
          const int s = slot_of(a, row, c, wrong);
          if (s >= 0) __builtin_memcpy(to + ((int64_t)s * a.ld_to + j) * E, from + j * E, E);
        }
    }
  }
  if (wrong && a.error) atomicOr(a.error, IM_ERR_ACTION);
}

// A unit of a row of `dim` elements: 16 bytes that end with the row where it ends inside
// them, single elements where the row is shorter.
template <typename T>
struct Piece {
  int at, fresh;   // first element; elements at its end that no unit before it has
  __device__ __forceinline__ Piece(int u, int dim) {
    const int first = u * kVec<T>;
    fresh = dim - first < kVec<T> ? dim - first : kVec<T>;
    at = dim < kVec<T> || fresh == kVec<T> ? first : dim - kVec<T>;
  }
  __device__ __forceinline__ u32x4 load(const T* row, int dim) const {
    return dim < kVec<T> ? load_few(row, dim) : load16(row + at);
  }
  __device__ __forceinline__ void store(T* row, int dim, u32x4 v) const {
    if (dim < kVec<T>) store_few(row, v, dim);
    else *reinterpret_cast<u32x4_any*>(row + at) = v;
  }
};
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
template <typename T>
__device__ __forceinline__ u32x4 narrow_to(const float (&f)[kVec<T>]) {
  T o[kVec<T>];
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) o[i] = (T)f[i];
  u32x4 v;
  __builtin_memcpy(&v, o, 16);
  return v;
}

constexpr int kTogether = 4;   // choices whose rows are on their way at once

// to_i = sum_c weight_ic from[slot_ic], by T lanes a row, N units a lane at once.
template <typename E, int T, int N>
__global__ __launch_bounds__(256) void gather_kernel(const ExchangeArgs a) {
  const int l = (int)threadIdx.x % T, units = (a.dim + kVec<E> - 1) / kVec<E>;
  constexpr int kRows = 256 / T;
  bool wrong = false;
  for (int64_t row = (int64_t)blockIdx.x * kRows + (int)threadIdx.x / T; row < a.n; row += (int64_t)gridDim.x * kRows) {
    for (int u0 = l; u0 < units; u0 += T * N) {
      float sum[N][kVec<E>];
#pragma unroll
      for (int m = 0; m < N; ++m)
#pragma unroll
        for (int i = 0; i < kVec<E>; ++i) sum[m][i] = 0.f;
      for (int c0 = 0; c0 < a.k; c0 += kTogether) {
        u32x4 v[kTogether][N];
        float w[kTogether];
#pragma unroll
        for (int j = 0; j < kTogether; ++j) {
          const int s = slot_of(a, row, c0 + j, wrong);
          w[j] = s < 0 ? 0.f : (a.weight ? a.weight[row * a.k + c0 + j] : 1.f);
#pragma unroll
          for (int m = 0; m < N; ++m) v[j][m] = u32x4{0, 0, 0, 0};
          if (s >= 0) {
            const E* from = static_cast<const E*>(a.from) + s * a.ld_from;
#pragma unroll
            for (int m = 0; m < N; ++m)   // past the row's units its last one, which is not stored
              v[j][m] = Piece<E>(u0 + m * T < units ? u0 + m * T : units - 1, a.dim).load(from, a.dim);
          }
        }
#pragma unroll
        for (int j = 0; j < kTogether; ++j)
#pragma unroll
          for (int m = 0; m < N; ++m) {
            float f[kVec<E>];
            widen<E>(v[j][m], f);
#pragma unroll
            for (int i = 0; i < kVec<E>; ++i) sum[m][i] = fmaf(w[j], f[i], sum[m][i]);
          }
      }
#pragma unroll
      for (int m = 0; m < N; ++m)
        if (u0 + m * T < units)
          Piece<E>(u0 + m * T, a.dim).store(static_cast<E*>(a.to) + row * a.ld_to, a.dim, narrow_to<E>(sum[m]));
    }
  }
  if (wrong && a.error) atomicOr(a.error, IM_ERR_ACTION);
}

// to[slot_ic] = weight_ic from_i and dweight_ic = from_i . ys[slot_ic], by T lanes a row.
template <typename E, int T>
__global__ __launch_bounds__(256) void combine_backward_kernel(const ExchangeArgs a) {
  const int l = (int)threadIdx.x % T, units = (a.dim + kVec<E> - 1) / kVec<E>;
  constexpr int kRows = 256 / T;
  bool wrong = false;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.n; first += (int64_t)gridDim.x * kRows) {
    const int64_t at = first + (int)threadIdx.x / T, row = at < a.n ? at : a.n - 1;
    const bool in = at < a.n;   // every lane takes part in the sums across lanes
    const E* from = static_cast<const E*>(a.from) + row * a.ld_from;
    for (int c0 = 0; c0 < a.k; c0 += kTogether) {
      int s[kTogether];
      float w[kTogether], dot[kTogether];
#pragma unroll
      for (int j = 0; j < kTogether; ++j) {
        s[j] = in ? slot_of(a, row, c0 + j, wrong) : -1;
        w[j] = s[j] >= 0 && a.weight ? a.weight[row * a.k + c0 + j] : 0.f;
        dot[j] = 0.f;
      }
      for (int u = l; u < units; u += T) {
        const Piece<E> p(u, a.dim);
        u32x4 v[kTogether];
#pragma unroll
        for (int j = 0; j < kTogether; ++j) {
          v[j] = u32x4{0, 0, 0, 0};
          if (s[j] >= 0 && a.dweight) v[j] = p.load(static_cast<const E*>(a.ys) + s[j] * a.ld_ys, a.dim);
        }
        float g[kVec<E>];
        widen<E>(p.load(from, a.dim), g);
        const int skip = a.dim < kVec<E> ? 0 : kVec<E> - p.fresh;   // elements that the unit before has
#pragma unroll
        for (int j = 0; j < kTogether; ++j) {
          if (s[j] < 0) continue;
          float f[kVec<E>];
          widen<E>(v[j], f);
#pragma unroll
          for (int i = 0; i < kVec<E>; ++i) dot[j] = i < skip ? dot[j] : fmaf(g[i], f[i], dot[j]);
          if (a.to) {
#pragma unroll
            for (int i = 0; i < kVec<E>; ++i) f[i] = w[j] * g[i];
            p.store(static_cast<E*>(a.to) + s[j] * a.ld_to, a.dim, narrow_to<E>(f));
          }
        }
      }
      if (!a.dweight) continue;
#pragma unroll
      for (int j = 0; j < kTogether; ++j) {
#pragma unroll
        for (int d = 1; d < T; d *= 2) dot[j] += __shfl_xor(dot[j], d);
        if (in && l == 0 && c0 + j < a.k) a.dweight[row * a.k + c0 + j] = dot[j];
      }
    }
  }
  if (wrong && a.error) atomicOr(a.error, IM_ERR_ACTION);
}

// Lanes of a row: as many as it has units of 16 bytes, up to a wave.
int lanes_for(int64_t bytes) {
  int t = 1;
  while (t < 64 && t * 16 < bytes) t *= 2;
  return t;
}

template <int T>
struct Kernels {
  static void send(const ExchangeArgs& a, int e, hipStream_t s) {
    const dim3 grid(blocks_of(a.n, 256 / T)), block(256);
    if (e == 1) hipLaunchKernelGGL((send_kernel<1, T>), grid, block, 0, s, a);
    else if (e == 2) hipLaunchKernelGGL((send_kernel<2, T>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((send_kernel<4, T>), grid, block, 0, s, a);
  }
  static void gather(const ExchangeArgs& a, int e, hipStream_t s) {
    const dim3 grid(blocks_of(a.n, 256 / T)), block(256);
    if (T == 64 && (int64_t)a.dim * e > 1024) {   // more units than lanes
      if (e == 2) hipLaunchKernelGGL((gather_kernel<__bf16, T, 2>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((gather_kernel<float, T, 2>), grid, block, 0, s, a);
    } else {
      if (e == 2) hipLaunchKernelGGL((gather_kernel<__bf16, T, 1>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((gather_kernel<float, T, 1>), grid, block, 0, s, a);
    }
  }
  static void backward(const ExchangeArgs& a, int e, hipStream_t s) {
    const dim3 grid(blocks_of(a.n, 256 / T)), block(256);
    if (e == 2) hipLaunchKernelGGL((combine_backward_kernel<__bf16, T>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((combine_backward_kernel<float, T>), grid, block, 0, s, a);
  }
};

int element(int dtype) { return dtype == IM_CODES ? 1 : (dtype == IM_BF16 ? 2 : 4); }

#define BY_LANES(call)                          \
  switch (lanes_for((int64_t)a.dim * e)) {      \
    case 1: Kernels<1>::call; break;            \
    case 2: Kernels<2>::call; break;            \
    case 4: Kernels<4>::call; break;            \
    case 8: Kernels<8>::call; break;            \
    case 16: Kernels<16>::call; break;          \
    case 32: Kernels<32>::call; break;          \
    default: Kernels<64>::call; break;          \
  }

}  // namespace

int64_t plan_blocks(int64_t pairs, int cus, int64_t& each) {
  // one block, and one launch, for few pairs (4096: 4.1 us); more take blocks of 1024 each until a block a CU
  // (262144 pairs, 64 experts: 16 us in blocks of 4096)
  int64_t blocks = pairs <= 4096 ? 1 : (pairs + 1023) / 1024;
  blocks = blocks > cus ? cus : blocks;
  each = ((pairs + blocks - 1) / blocks + kPlanThreads - 1) / kPlanThreads * kPlanThreads;
  return each > 0 ? (pairs + each - 1) / each : 1;
}

hipError_t launch_dispatch_plan(const PlanArgs& a, hipStream_t s) {
  if (a.blocks > 1) {
    hipLaunchKernelGGL(count_kernel, dim3((unsigned)a.blocks), dim3(kPlanThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(place_kernel, dim3((unsigned)a.blocks), dim3(kPlanThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_send(const ExchangeArgs& a, int dtype, hipStream_t s) {
  const int e = element(dtype);
  BY_LANES(send(a, e, s))
  return hipGetLastError();
}
hipError_t launch_gather(const ExchangeArgs& a, int dtype, hipStream_t s) {
  const int e = element(dtype);
  BY_LANES(gather(a, e, s))
  return hipGetLastError();
}
hipError_t launch_combine_backward(const ExchangeArgs& a, int dtype, hipStream_t s) {
  const int e = element(dtype);
  BY_LANES(backward(a, e, s))
  return hipGetLastError();
}

}  // namespace learn
}  // namespace im
