// Exponentials and limits of the softmax.
#pragma once
#include <hip/hip_runtime.h>

namespace im {
namespace learn {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -300.f, kLeastE = -208.f;   // 2^-300 and e^-208 are 0 in fp32
// An lse of -1e30 or less is of a row whose valid classes are all masked by their biases. Floats are
// 2^76 apart there, so it says nothing of how the classes share: the row has no gradient.
constexpr float kMasked = -1e30f;
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float exp_(float x) { return exp2_(x * kLog2e); }
// log2 pi from ln pi = z - lse, in [kLeast, 0]: lse is rounded, so that a pi near 1 could come out
// above it (at |lse| of 2^24 by any factor). NaN: kLeast.
__device__ __forceinline__ float log2_share(float x) { return __builtin_amdgcn_fmed3f(x * kLog2e, kLeast, 0.f); }

}  // namespace learn
}  // namespace im
