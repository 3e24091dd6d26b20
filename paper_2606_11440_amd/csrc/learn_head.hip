// Gradient of a narrow softmax head (64 classes, 512 wide at most, bf16: a
// policy's head) in one pass over its rows: h is read once, dh written once, and
// logits and dz stay on the chip.
//
// A wave owns 64 of the columns for everything: of the logits it sums the part
// over its columns (the parts are added through LDS), then from the dz of all
// classes it forms its columns of dh = dz W and adds to its columns of dW =
// sum dz^T h, which stay in registers while the rows of a group pass. W stays
// there too, in the orders that the two products take it. dz enters the products
// as two bf16 numbers, its rounding and what that leaves, so that only the
// results are rounded (the products are a small part of the time). A block takes
// 32 rows at a time: two barriers a tile, the next tile's rows on their way.
//
// Measured, 262144 rows: 64 classes, 512 wide, 16 groups 220 us in one pass against
// 356 us as products that keep dz in memory (reading h and writing dh: 101 at the
// rate of a copy); 15 classes, 256 wide 113 against 181 (51). (All in the first calls after
// a pause; once the clock has settled they are 184 and 85.) Other widths than 256 and 512 have
// branches around every store and take the next larger of the two: with 64 classes 384
// columns 204 us, 500 220; 264 191; 200 124 where 256 take 113. dz as two numbers costs
// 13 %. Up to 32 classes take a kernel of half the products and LDS: 135 ->
// 113 us with 15 classes, 178 -> 156 with 32 and 512 columns. What bounds it: the chain
// of LDS, products and dz within a tile, at two waves a SIMD (W and dW fill the
// registers): without the loads 10 % less, without the stores 9, without dh 38. Also
// tried: dz of the next tile beside the products of this one, each wave with all of k
// for 16 classes, one long phase a tile: 277 us (registers spill), 138 at 256 columns.
//
// As in the sums over rows, the groups' rows are a line of granules that the
// blocks cut into equal runs; what a run's end cuts is joined in order.
#include <type_traits>

#include "learn_internal.h"
#include "learn_softmax.h"
#include "learn_tile.h"

namespace im {
namespace learn {
namespace {

constexpr int kRows = 32, kSlice = 64;

struct NarrowRow {
  int y;
  float lse, A, B, up;
  uint32_t mask[2];
  int live;
};

__device__ __forceinline__ u32x4 zeros() { return u32x4{0, 0, 0, 0}; }

// LDS of the rows' h: unit u (16 bytes) of row r at u ^ 2 (r % 8): the rows of a
// fragment read, and the rows and halves of a transposing one, meet in no bank.
template <int NW>
__device__ __forceinline__ int h_at(int row, int unit) {
  return row * (NW * 128) + ((unit ^ ((row & 7) << 1)) << 4);
}
// LDS of dz [rows][classes], 128 bytes a row.
__device__ __forceinline__ int dz_at(int row, int unit) { return row * 128 + ((unit ^ ((row >> 1) & 7)) << 4); }

// LDS of a wave's part of the logits [rows][C classes], 128 or 256 bytes a row.
template <int C>
__device__ __forceinline__ int z_at(int row, int unit) {
  return row * (C * 4) + ((unit ^ (C == 32 ? (row >> 1) & 7 : row & 15)) << 4);
}

// 16 columns (from c0) of 32 rows, as a fragment whose k are the rows 4 g + j and
// 16 + 4 g + j of lane group g: with rows in fours every half wave reads 8 rows.
template <class At>
__device__ __forceinline__ u32x4 across_rows(const char* lds, int lane, int c0, At at) {
  typedef __attribute__((address_space(3))) s16x4 lds4;
  const int i = lane % 16, g = lane / 16, c = c0 + (i % 4) * 4, row = g * 4 + i / 4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(lds + at(row, c / 8) + (c & 4) * 2));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(lds + at(row + 16, c / 8) + (c & 4) * 2));
  return __builtin_bit_cast(u32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// NW waves, so NW * kSlice columns; C classes (32 or 64)
template <int NW, int C>
__global__ __launch_bounds__(NW * 64, 2) void narrow_gradient_kernel(const NarrowArgs a) {
  using T = __bf16;
  constexpr int NT = NW * 64, kUnits = kRows * NW * 8 / NT, kHBytes = kRows * NW * 128;
  constexpr int kPart = kRows * C * 4, kQuad = C / 4;   // quads of classes
  constexpr int kQuads = kRows * kQuad > NT ? kRows * kQuad / NT : 1, CB = C / 16, CS = C / 32;
  static_assert(kUnits == 4 && (C == 32 || C == 64) && kPart >= C * 128 && kPart >= kRows * 128, "");
  __shared__ __attribute__((aligned(16))) char h_lds[2][kHBytes];
  __shared__ __attribute__((aligned(16))) char parts[NW][kPart];   // of the logits; then a wave's dh
  __shared__ __attribute__((aligned(16))) char dz_lds[2][kRows * 128];   // dz rounded to bf16, and what that leaves
  __shared__ NarrowRow info[2][kRows];
  __shared__ Groups groups;

  groups.init(a.offsets, a.G, a.n, a.granule);
  __syncthreads();
  if (groups.total < 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.error) atomicOr(a.error, IM_ERR_COUNT);
    if (blockIdx.x == 0 && a.cuts)   // nothing to join
      for (int g = threadIdx.x; g < a.G; g += NT) a.cuts[g] = int4{0, 0, 0, 0};
    return;
  }
  Line line;
  line.units = groups.total;
  line.parts = a.parts < groups.total ? a.parts : groups.total;
  if (blockIdx.x == 0 && a.cuts)
    for (int g = threadIdx.x; g < a.G; g += NT) a.cuts[g] = line.cut(groups.start[g], groups.start[g + 1]);
  if ((int)blockIdx.x >= (int)line.parts) return;
  const int run = blockIdx.x, begin = (int)line.begin(run), end = (int)line.begin(run + 1);
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, l16 = lane % 16, g4 = lane / 16;
  const int c_first = wave * kSlice;   // the wave's columns
  const T* const H = static_cast<const T*>(a.h);

  for (int u = begin; u < end;) {
    int g, lo, hi;
    groups.find(a.offsets, a.G, a.n, a.granule, u, g, lo, hi);
    const int first = __builtin_amdgcn_readfirstlane(groups.start[g]);
    const int count = __builtin_amdgcn_readfirstlane(groups.start[g + 1]) - first;
    const int k = u - first, length = end - u < count - k ? end - u : count - k;
    const int rows1 = a.offsets ? a.offsets[g + 1] : a.n;
    hi = rows1 - lo > (int64_t)length * a.granule ? lo + length * a.granule : rows1;
    const int tiles = (hi - lo + kRows - 1) / kRows;

    // W of the wave's columns: by columns (for the logits) and by classes (for dh)
    const T* const W = static_cast<const T*>(a.W) + g * (int64_t)a.V * a.d;
    u32x4 wc[CB][2], wv[4][CS];
#pragma unroll
    for (int b = 0; b < CB; ++b)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int cls = b * 16 + l16, col = c_first + s * 32 + g4 * 8, left = a.d - col;
        const T* const p = W + (int64_t)cls * a.d + col;
        wc[b][s] = cls >= a.V || left <= 0 ? zeros() : (left >= 8 ? load16(p) : load_few(p, left));
      }
    // by classes: through the wave's LDS (free here), turned on the way out
    __syncthreads();   // the LDS of the group before
#pragma unroll
    for (int b = 0; b < CB; ++b)
#pragma unroll
      for (int s = 0; s < 2; ++s) *reinterpret_cast<u32x4*>(parts[wave] + dz_at(b * 16 + l16, s * 4 + g4)) = wc[b][s];
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int s = 0; s < CS; ++s) {
        typedef __attribute__((address_space(3))) s16x4 lds4;
        const int c = b * 16 + (l16 % 4) * 4, row = s * 32 + g4 * 8 + l16 / 4;
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(parts[wave] + dz_at(row, c / 8) + (c & 4) * 2));
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(parts[wave] + dz_at(row + 4, c / 8) + (c & 4) * 2));
        wv[b][s] = __builtin_bit_cast(u32x4, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    // the biases of the thread's classes in the sum over the parts
    const int quad = tid % kQuad;
    f32x4 plus = {0.f, 0.f, 0.f, 0.f}, colsum = {0.f, 0.f, 0.f, 0.f};
    if (a.bias)
#pragma unroll
      for (int r = 0; r < 4; ++r) plus[r] = quad * 4 + r < a.V ? a.bias[(int64_t)g * a.V + quad * 4 + r] : 0.f;

    f32x4 dw[CB][4];   // [classes][columns]
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) dw[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // a tile's h on its way: thread's unit of rows tid / (8 NW) + 8 i
    u32x4 ahead[kUnits];
    auto load_h = [&](int t, auto full) {
      const int tid = fresh_thread(), unit = tid % (NW * 8), u_left = a.d - unit * 8;
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int row = lo + t * kRows + tid / (NW * 8) + i * (NT / (NW * 8));
        const T* const p = H + (int64_t)(row < hi ? row : hi - 1) * a.ld_h + unit * 8;
        if constexpr (full) ahead[i] = load16(p);
        else if (a.d >= 8) ahead[i] = u_left > 0 ? load16(p + (u_left < 8 ? u_left - 8 : 0)) : zeros();
        else ahead[i] = u_left > 0 ? load_few(p, u_left) : zeros();
      }
    };
    auto store_h = [&](int t, auto full) {   // rows that add nothing are zero, whatever they hold
      const int tid = fresh_thread(), unit = tid % (NW * 8), u_left = a.d - unit * 8;
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int row = tid / (NW * 8) + i * (NT / (NW * 8));
        u32x4 v = ahead[i];
        if constexpr (!full) {
          if (u_left < 8 && u_left > 0 && a.d >= 8) v = keep_last<T>(v, u_left);
        }
        if (!info[t & 1][row].live) v = zeros();
        *reinterpret_cast<u32x4*>(h_lds[t & 1] + h_at<NW>(row, unit)) = v;
      }
    };
    // a tile's rows: loaded by the first threads, checked when they go to LDS
    NarrowRow mine;
    auto load_info = [&](int t) {
      const int tid = fresh_thread();
      const int64_t row = (int64_t)lo + t * kRows + tid;
      mine = NarrowRow{-1, INFINITY, 0.f, 0.f, 0.f, {0xffffffffu, 0xffffffffu}, 0};
      if (tid >= kRows || row >= hi) return;
      mine.y = a.target[row];
      mine.lse = a.lse[row];
      mine.up = a.dlogp[row];
      mine.A = a.dentropy ? a.entropy[row] : 0.f;
      mine.B = a.dentropy ? a.dentropy[row] : 0.f;
      mine.live = 1;
      if (a.valid) {
        mine.mask[0] = a.valid[row * a.words];
        mine.mask[1] = a.words > 1 ? a.valid[row * a.words + 1] : 0u;
      }
    };
    auto store_info = [&](int t) {
      const int tid = fresh_thread();
      if (tid >= kRows) return;
      if (mine.live) {
        const int y = mine.y;
        const bool wrong = y < -1 || y >= a.V || (y >= 0 && !(((y < 32 ? mine.mask[0] : mine.mask[1]) >> (y & 31)) & 1u));
        if (wrong && a.error) atomicOr(a.error, IM_ERR_ACTION);
        if (wrong) mine.y = -1;
        const float H = mine.A, ent = mine.B, lse = mine.lse, up = mine.y < 0 ? 0.f : mine.up;
        mine.live = (up != 0.f || ent != 0.f) && !(lse <= kMasked);
        mine.up = mine.live ? up : 0.f;
        mine.A = mine.live ? -up - ent * H + (lse - lse) : 0.f;   // an lse that is not finite makes the row NaN
        mine.B = mine.live ? -ent * kLn2 : 0.f;
        mine.lse = mine.live ? lse : INFINITY;
      }
      info[t & 1][tid] = mine;
    };

    load_info(0);
    load_h(0, std::false_type{});
    store_info(0);
    if (tiles > 1) load_info(1);
    __syncthreads();
    store_h(0, std::false_type{});
    if (tiles > 1) load_h(1, std::false_type{});
    __syncthreads();
    // full: all of the tile's rows and of the waves' columns exist, and two more tiles follow.
    // Such a tile takes no branch around its stores, so that the wait for the rows that are
    // on their way leaves the stores behind them alone.
    auto tile = [&](int t, auto full) {
      const char* const ht = h_lds[t & 1];
      {   // the logits over the wave's columns
        const int lane = fresh_thread() % 64, l16 = lane % 16, g4 = lane / 16;
        f32x4 z[2][CB];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int b = 0; b < CB; ++b) z[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const u32x4 p = *reinterpret_cast<const u32x4*>(ht + h_at<NW>(i * 16 + l16, wave * 8 + s * 4 + g4));
#pragma unroll
            for (int b = 0; b < CB; ++b) z[i][b] = mma<T>(wc[b][s], p, z[i][b]);
          }
#pragma unroll
          for (int b = 0; b < CB; ++b)
            *reinterpret_cast<f32x4*>(parts[wave] + z_at<C>(i * 16 + l16, b * 4 + g4)) = z[i][b];
        }
      }
      if (full || t + 1 < tiles) store_info(t + 1);
      __syncthreads();
      if (full || t + 1 < tiles) store_h(t + 1, full);
      if (full || t + 2 < tiles) {
        load_info(t + 2);
        load_h(t + 2, full);
      }
#pragma unroll
      for (int e = 0; e < kQuads; ++e) {   // dz of four classes of a row
        const int tid = fresh_thread(), quad = tid % kQuad;
        const int row = tid / kQuad + e * (NT / kQuad);
        if (kRows * kQuad < NT && row >= kRows) break;   // whole waves
        f32x4 z = {0.f, 0.f, 0.f, 0.f}, dz;
#pragma unroll
        for (int w = 0; w < NW; ++w) z += *reinterpret_cast<const f32x4*>(parts[w] + z_at<C>(row, quad));
        const NarrowRow& of = info[t & 1][row];
        const uint32_t bits = of.mask[quad / 8] >> (quad % 8 * 4);
        const float lse = of.lse, A = of.A, B = of.B, up = of.up;
        const int y = of.y;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float zr = z[r] + plus[r], tr = log2_share(zr - lse);
          float v = exp2_(tr) * fmaf(B, tr, A);
          v += quad * 4 + r == y && zr != -INFINITY ? up : 0.f;
          dz[r] = (bits >> r) & 1u && quad * 4 + r < a.V ? v : 0.f;
        }
        colsum += dz;
        bf16x4 o, rest;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          o[r] = (T)dz[r];
          rest[r] = (T)(dz[r] - (float)o[r]);
        }
        *reinterpret_cast<bf16x4*>(dz_lds[0] + dz_at(row, quad / 2) + (quad & 1) * 8) = o;
        *reinterpret_cast<bf16x4*>(dz_lds[1] + dz_at(row, quad / 2) + (quad & 1) * 8) = rest;
      }
      __syncthreads();
      // dW of the wave's columns
      if (a.dW) {
        const int lane = fresh_thread() % 64;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          u32x4 p[CB];
#pragma unroll
          for (int i = 0; i < CB; ++i) p[i] = across_rows(dz_lds[half], lane, i * 16, dz_at);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u32x4 q = across_rows(ht, lane, c_first + j * 16, h_at<NW>);
#pragma unroll
            for (int i = 0; i < CB; ++i) dw[i][j] = mma<T>(q, p[i], dw[i][j]);
          }
        }
      }
      // dh of the wave's columns, through the wave's own LDS to whole lines
      if (full || a.dh) {
        const int lane = fresh_thread() % 64, l16 = lane % 16, g4 = lane / 16;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          f32x4 o[4];
          u32x4 p[2 * CS];   // what the rounding left first
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < 2 * CS; ++s)
            p[s] = *reinterpret_cast<const u32x4*>(dz_lds[1 - s / CS] + dz_at(i * 16 + l16, s % CS * 4 + g4));
#pragma unroll
          for (int s = 0; s < 2 * CS; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = mma<T>(wv[j][s % CS], p[s], o[j]);
          const int row = i * 16 + l16;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int c = j * 16 + g4 * 4;
            bf16x4 v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = (T)o[j][r];
            *reinterpret_cast<bf16x4*>(parts[wave] + dz_at(row, c / 8) + (c & 4) * 2) = v;
          }
        }
        // a wave's LDS operations are done in their order
        const int c = c_first + lane % 8 * 8, left = a.d - c;
        u32x4 out[kRows / 8];
#pragma unroll
        for (int i = 0; i < kRows / 8; ++i)
          out[i] = *reinterpret_cast<const u32x4*>(parts[wave] + dz_at(i * 8 + lane / 8, lane % 8));
        if (a.relu_in) {
          u32x4 x[kRows / 8];
#pragma unroll
          for (int i = 0; i < kRows / 8; ++i)
            x[i] = *reinterpret_cast<const u32x4*>(ht + h_at<NW>(i * 8 + lane / 8, wave * 8 + lane % 8));
#pragma unroll
          for (int i = 0; i < kRows / 8; ++i) out[i] = where_positive<T>(out[i], x[i]);
        }
#pragma unroll
        for (int i = 0; i < kRows / 8; ++i) {
          const int64_t at = (int64_t)lo + t * kRows + i * 8 + lane / 8;
          const u32x4 v = out[i];
          T* const to = static_cast<T*>(a.dh) + at * a.ld_dh + c;
          if constexpr (full) {
            *reinterpret_cast<u32x4_any*>(to) = v;
            continue;
          }
          if (at >= hi || left <= 0) continue;
          if (left >= 8) *reinterpret_cast<u32x4_any*>(to) = v;
          else store_few(to, v, left);
        }
      }
    };
    int t = 0;
    if (a.d == NW * kSlice && a.dh)
      for (; t + 2 < tiles; ++t) tile(t, std::true_type{});
    for (; t < tiles; ++t) tile(t, std::false_type{});

    // the group's gradient, or this run's piece of it
    const bool all = length == count;
    float* const piece = all ? nullptr : a.pieces + (2 * (int64_t)run + (u == begin ? 0 : 1)) * a.piece;
    if (a.dW) {
#pragma unroll
      for (int i = 0; i < CB; ++i) {
        const int cls = i * 16 + l16;
        if (cls >= a.V) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = c_first + j * 16 + g4 * 4, left = a.d - c;
          if (left <= 0) continue;
          if (all) {
            T* const to = static_cast<T*>(a.dW) + ((int64_t)g * a.V + cls) * a.d + c;
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (r < left) to[r] = (T)dw[i][j][r];
          } else {   // rows of a.pitch columns, a multiple of 4 past d
            *reinterpret_cast<f32x4*>(piece + (int64_t)cls * a.pitch + c) = dw[i][j];
          }
        }
      }
    }
    if (a.db) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int o = kQuad; o < 64; o *= 2) colsum[r] += __shfl_xor(colsum[r], o);
      __syncthreads();   // dz has been read
      f32x4* const across = reinterpret_cast<f32x4*>(dz_lds[0]);   // [NW][kQuad]
      if (lane < kQuad) across[wave * kQuad + lane] = colsum;
      __syncthreads();
      if (tid < kQuad) {
        f32x4 v = across[tid];
        for (int w = 1; w < NW; ++w) v += across[w * kQuad + tid];
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (tid * 4 + r < a.V)
            (all ? a.db + (int64_t)g * a.V : piece + (int64_t)a.V * a.pitch)[tid * 4 + r] = v[r];
      }
    }
    u += length;
  }
}

// Adds the pieces of the groups that several runs cut (in their order), and
// clears the gradient of empty ones. One element a thread.
__global__ __launch_bounds__(256) void join_narrow_kernel(const NarrowArgs a) {
  const int g = blockIdx.y;
  const int4 cut = a.cuts ? a.cuts[g] : int4{0, -1, 0, 0};
  if (cut.x == cut.y) return;   // stored already
  const int e = blockIdx.x * 256 + threadIdx.x, wide = a.V * a.d;
  if (e >= wide + a.V || (e < wide ? a.dW == nullptr : a.db == nullptr)) return;
  const int64_t at = e < wide ? (int64_t)(e / a.d) * a.pitch + e % a.d : (int64_t)a.V * a.pitch + e - wide;
  float v = 0.f;
#pragma unroll 8
  for (int p = cut.x; p <= cut.y; ++p) v += a.pieces[(2 * (int64_t)p + (p == cut.x ? cut.z : 0)) * a.piece + at];
  if (e < wide) static_cast<__bf16*>(a.dW)[(int64_t)g * wide + e] = (__bf16)v;
  else a.db[(int64_t)g * a.V + e - wide] = v;
}

}  // namespace

// W and dW of such a head fit the registers of one block (8 waves of 64 columns);
// wider or longer ones, and fp32, whose fragments take twice the registers, go
// through the general products.
bool narrow_supported(int dtype, int64_t d, int64_t V) { return dtype == IM_BF16 && d <= 8 * kSlice && V <= 64; }

// A granule is two tiles, a run two granules at least; as many blocks as run at once.
NarrowPlan plan_narrow(int64_t n, int64_t G, int64_t d, int64_t V, int cus) {
  NarrowPlan p;
  p.granule = 2 * kRows;
  const int64_t granules = n > 0 ? (n + p.granule - 1) / p.granule + G - 1 : 0;
  const int64_t most = (granules + 1) / 2, slots = (int64_t)cus * (d <= 4 * kSlice ? 2 : 1);
  p.parts = most < slots ? most : slots;
  p.pitch = (d + 3) & ~(int64_t)3;
  p.piece = (V * p.pitch + V + 3) & ~(int64_t)3;
  return p;
}

hipError_t launch_narrow(const NarrowArgs& a, hipStream_t s) {
  if (a.parts > 0) {
    const bool thin = a.d <= 4 * kSlice;
    const auto kernel = a.V <= 32 ? (thin ? narrow_gradient_kernel<4, 32> : narrow_gradient_kernel<8, 32>)
                                  : (thin ? narrow_gradient_kernel<4, 64> : narrow_gradient_kernel<8, 64>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.parts), dim3(thin ? 256 : 512), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.dW && !a.db) return hipSuccess;
  const int all = a.V * a.d + a.V;
  hipLaunchKernelGGL(join_narrow_kernel, dim3((unsigned)((all + 255) / 256), (unsigned)a.G), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace learn
}  // namespace im
