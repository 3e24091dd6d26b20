// Kernel arguments of the AdamW step.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "inframind_learn.h"

namespace im {
namespace learn {

constexpr int kRun = 4096;   // elements of a block's run (a multiple of IM_STATE_BLOCK)

struct AdamwRun {
  int64_t first;             // element of the tensor (a multiple of kRun)
  int32_t tensor;
  int32_t aligned;           // 1: four elements of every buffer can be moved at once
};

struct AdamwArgs {
  const AdamwRun* table;
  const im_adamw_tensor* tensors;
  int64_t runs;
  int64_t blocks;            // grid at most: blocks share the runs
  int64_t* step;
  const float* scale;
  uint32_t* done;
  double beta1, beta2;
  float lr, beta1f, omb1, beta2f, omb2, eps, keep;   // omb: 1 - beta; keep: 1 - lr weight_decay
};

hipError_t launch_adamw(const AdamwArgs& a, int bits, int grad_dtype, hipStream_t s);

}  // namespace learn
}  // namespace im
