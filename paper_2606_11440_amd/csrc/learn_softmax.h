// Constants of the softmax in powers of two: t = z log2 e.
#pragma once
#include <hip/hip_runtime.h>

namespace im {
namespace learn {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -300.f;   // 2^-300 is 0 in fp32
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
// log2 pi from ln pi = z - lse, in [kLeast, 0]: lse is rounded, so that a pi near 1 could come out
// above it (at |lse| of 2^24 by any factor). NaN: kLeast.
__device__ __forceinline__ float log2_share(float x) { return __builtin_amdgcn_fmed3f(x * kLog2e, kLeast, 0.f); }

}  // namespace learn
}  // namespace im
