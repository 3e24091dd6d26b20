// Kernel argument blocks and launchers of the learner's operators.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "inframind_learn.h"

namespace im {
namespace learn {

// What a row product does with its results.
enum Epilogue {
  kStore = 0,     // y = act(sum + b)
  kStoreInput,    // dx = sum, zero where x <= 0 with relu_in
  kStats,         // per row and column tile: largest logit, sum exp, sum exp (z - largest)
  kGradLogits,    // dz of a piece of the classes
  kPartial        // the sums of a run of k, in fp32 (joined by a kernel of their own)
};

// A product of the groups' rows with their weights: out[i][j] = sum_k A[i][k] B_g(j, k).
struct RowArgs {
  const int32_t* offsets;
  int32_t G, n, K, N;         // N: output columns (of the piece, for a head)
  const void* A;
  int64_t lda;
  const void* B;              // rows [N x K], or columns [K x N], per group
  int64_t ldb, b_group;       // strides in elements
  const float* bias;          // [G x bias_group] or NULL
  int64_t bias_group;
  void* C;
  int64_t ldc;
  int32_t relu;
  int32_t* error;
  int32_t row_tiles, col_tiles;   // at most, and exactly
  int32_t cus;                    // compute units of the device
  int32_t splits, split_k;        // runs of k, and their length (a multiple of the stage); 1: the whole
  float* part;                    // [splits][n][N] with splits > 1
  // kStoreInput
  const void* X;              // relu_in: the layer's input
  int64_t ldx;
  float* sum;                 // fp32 running sums [n x N] over the pieces of a head, or NULL
  int32_t first, last;        // piece of a head: the first starts the sums, the last stores C
  // heads
  int32_t V, words, col0;     // classes, mask words of a row, first class of the piece
  const uint32_t* valid;
  const int32_t* target;
  float* stats;               // [col_tiles][n][3]
  float* taken;               // [n] logit of the target
  float* logp;
  float* entropy;             // kStats: out; kGradLogits: in
  float* lse;                 // kStats: out; kGradLogits: in
  const float* dlogp;
  const float* dentropy;
  float* db_part;             // [row_tiles][db_width] column sums of dz
  int64_t db_width;
  uint8_t* live;              // [n] kGradLogits: 1 where the row adds to the gradient
};

// dW_g = sum over the group's rows of P[i][m] Q[i][n] (and db_g = sum P[i][m]).
struct SumArgs {
  const int32_t* offsets;
  int32_t G, n, M, N;
  const void* P;
  int64_t ldp;
  const void* Q;
  int64_t ldq;
  const uint8_t* live;        // rows of Q to take, or NULL (all)
  void* dW;                   // [G x w_group], rows of N
  int64_t w_group;
  float* db;                  // [G x M] or NULL
  float* part;                // [2 parts][tiles][tile and its rows]: pieces of groups that parts cut
  int4* cuts;                 // [G] {first part, last part, the first one's piece, 0}, or NULL (no rows)
  int32_t granule, parts;     // rows of a granule; parts of the line of granules
  int32_t row_tiles, col_tiles;
  int32_t* error;
};

// The gradient of a narrow head in one pass.
struct NarrowArgs {
  const int32_t* offsets;
  int32_t G, n, d, V, words, relu_in;
  const void* h;
  int64_t ld_h;
  const void* W;
  const float* bias;
  const uint32_t* valid;
  const int32_t* target;
  const float *lse, *entropy, *dlogp, *dentropy;
  void* dh;
  int64_t ld_dh;
  void* dW;
  float* db;
  float* pieces;              // [2 parts][piece]: V rows of `pitch`, then V
  int4* cuts;                 // [G], or NULL (no rows)
  int64_t piece, pitch;
  int32_t granule, parts;
  int32_t* error;
};
struct NarrowPlan {
  int64_t granule, parts, pitch, piece;
};
bool narrow_supported(int dtype, int64_t d, int64_t V);
NarrowPlan plan_narrow(int64_t n, int64_t G, int64_t d, int64_t V, int cus);
hipError_t launch_narrow(const NarrowArgs& a, hipStream_t s);

// Tile shape of a row product of n rows in G groups with N columns, and its tiles
// (row tiles: at most; the groups' sizes are known on the device only).
struct RowPlan {
  int shape;
  int64_t row_tiles, col_tiles, splits, split_k;
};
// may_split: the epilogue can follow a join of several runs of k
RowPlan plan_rows(int dtype, int64_t n, int64_t G, int64_t N, int64_t K, int cus, bool may_split);
hipError_t launch_rows_product(const RowArgs& a, int dtype, int shape, int epilogue, hipStream_t s);

struct SumPlan {
  int shape;
  int64_t row_tiles, col_tiles, granule, parts, piece;   // piece: floats of a block's piece
};
SumPlan plan_sums(int dtype, int64_t n, int64_t G, int64_t M, int64_t N, int cus);
hipError_t launch_sums(const SumArgs& a, int dtype, int shape, hipStream_t s);
// db_g = sum of the column sums of the group's row tiles (of `step` rows).
hipError_t launch_bias_sum(const int32_t* offsets, int G, int n, int step, const float* part, int64_t width, float* db,
                           hipStream_t s);
int rows_per_tile(int shape);   // of a row product
int cols_per_tile(int shape);
int rows_per_sum(int shape);    // rows of W a tile of the sums covers
int threads_per_sum(int shape);

}  // namespace learn
}  // namespace im
