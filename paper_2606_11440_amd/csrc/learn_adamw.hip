// One AdamW step over many tensors: bound by memory (28 bytes an element with
// fp32 states and gradients, 16 with 8-bit states), so one launch reads and
// writes everything once. A block takes a run of kRun elements of one tensor
// from a table made with the plan; a wave takes 256 neighbouring elements at a
// time, four a lane: one block of an 8-bit state, whose largest magnitude is a
// maximum over the wave.
#include "learn_adamw.h"

#include "learn_tile.h"

namespace im {
namespace learn {
namespace {

// Each operation is rounded by itself (no contraction), so that the step is
// the same fp32 arithmetic wherever it is done.
#pragma clang fp contract(off)

// Pointers read from a table: known to be global memory (plain loads, not flat ones).
template <typename T>
using Global = __attribute__((address_space(1))) T*;
template <typename T>
__device__ __forceinline__ Global<T> global(const void* p) {
  return (Global<T>)(reinterpret_cast<uintptr_t>(p));
}

__device__ __forceinline__ f32x4 load_f(Global<const float> p, int left, bool aligned) {
  if (left >= 4 && aligned) return *(Global<const f32x4>)p;
  f32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = i < left ? p[i] : 0.f;
  return v;
}
__device__ __forceinline__ void store_f(Global<float> p, f32x4 v, int left, bool aligned) {
  if (left >= 4 && aligned) {
    *(Global<f32x4>)p = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) p[i] = v[i];
}
__device__ __forceinline__ f32x4 load_h(Global<const __bf16> p, int left, bool aligned) {
  f32x4 v;
  if (left >= 4 && aligned) {
    const bf16x4 x = *(Global<const bf16x4>)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)x[i];
    return v;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = i < left ? (float)p[i] : 0.f;
  return v;
}
__device__ __forceinline__ uint32_t load_b(Global<const uint8_t> p, int left, bool aligned) {
  if (left >= 4 && aligned) return *(Global<const uint32_t>)p;
  uint32_t v = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) v |= (uint32_t)p[i] << (8 * i);
  return v;
}
__device__ __forceinline__ void store_b(Global<uint8_t> p, uint32_t v, int left, bool aligned) {
  if (left >= 4 && aligned) {
    *(Global<uint32_t>)p = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) p[i] = (uint8_t)(v >> (8 * i));
}

__device__ __forceinline__ f32x4 from_e4m3(uint32_t c) {
  return f32x4{__builtin_amdgcn_cvt_f32_fp8(c, 0), __builtin_amdgcn_cvt_f32_fp8(c, 1), __builtin_amdgcn_cvt_f32_fp8(c, 2),
               __builtin_amdgcn_cvt_f32_fp8(c, 3)};
}
__device__ __forceinline__ uint32_t to_e4m3(f32x4 x) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], v, true);
}

// Scale of a wave's block of 256 and its codes. The maximum is taken over the
// magnitudes' bits, which order like the values with NaN on top.
__device__ __forceinline__ uint32_t encode(f32x4 y, bool least, float& scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float v = y[i];
    const uint32_t b = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
    top = b > top ? b : top;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = (uint32_t)__shfl_xor((int)top, d);
    top = o > top ? o : top;
  }
  const float largest = __builtin_bit_cast(float, top);
  scale = largest * (1.0f / 448.0f);
  scale = scale < 0x1p-126f ? 0x1p-126f : scale;   // NaN stays
  if (top >= 0x7f800000u) scale = __builtin_nanf("");
  f32x4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float q = __fdiv_rn(y[i], scale);
    q = q > 448.f ? 448.f : (q < -448.f ? -448.f : q);
    if (least && q > 0.f && q < 0x1p-9f) q = 0x1p-9f;
    x[i] = q;
  }
  return to_e4m3(x);
}

template <int BITS, bool HALF>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamwArgs a) {
  __shared__ float rate[2];
  if (threadIdx.x == 0) {
    const double t = (double)(*a.step + 1);
    rate[0] = (float)(1.0 / (1.0 - pow(a.beta1, t)));
    rate[1] = (float)(1.0 / (1.0 - pow(a.beta2, t)));
  }
  __syncthreads();
  const float r1 = rate[0], r2 = rate[1], scale = a.scale ? *a.scale : 1.f;
  if (a.runs > 0) {
    const AdamwRun run = a.table[blockIdx.x];
    const im_adamw_tensor t = a.tensors[run.tensor];
    const Global<float> param = global<float>(t.param), mf = global<float>(t.m), vf = global<float>(t.v);
    const Global<float> m_scale = global<float>(t.m_scale), v_scale = global<float>(t.v_scale);
    const Global<uint8_t> mb = global<uint8_t>(t.m), vb = global<uint8_t>(t.v);
    const float keep = t.decay ? a.keep : 1.f;
    const bool al = run.aligned;
    const int64_t end = run.first + kRun < t.n ? run.first + kRun : t.n;
    const int lane = threadIdx.x % 64;
    for (int64_t at = run.first + (threadIdx.x / 64) * 256; at < end; at += 1024) {
      const int64_t e = at + lane * 4;
      const int left = end - e >= 4 ? 4 : (int)(end - e);
      f32x4 p = load_f(param + e, left, al), m, v;
      const f32x4 g0 = HALF ? load_h(global<const __bf16>(t.grad) + e, left, al)
                            : load_f(global<const float>(t.grad) + e, left, al);
      if constexpr (BITS == 32) {
        m = load_f(mf + e, left, al);
        v = load_f(vf + e, left, al);
      } else {
        const uint32_t cm = load_b(mb + e, left, al);
        const uint32_t cv = load_b(vb + e, left, al);
        const float ms = m_scale[at / 256], vs = v_scale[at / 256];
        m = from_e4m3(cm);
        v = from_e4m3(cv);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          m[i] = m[i] * ms;
          const float r = v[i] * vs;
          v[i] = r * r;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float g = g0[i] * scale;
        m[i] = m[i] * a.beta1f + g * a.omb1;
        v[i] = v[i] * a.beta2f + g * g * a.omb2;
        const float d = __fsqrt_rn(v[i] * r2) + a.eps;
        p[i] = p[i] * keep - __fdiv_rn(m[i] * r1, d) * a.lr;
      }
      store_f(param + e, p, left, al);
      if (t.copy) {
        const Global<__bf16> c = global<__bf16>(t.copy) + e;
        if (left >= 4 && al) {
          bf16x4 o;
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = (__bf16)p[i];
          *(Global<bf16x4>)c = o;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (i < left) c[i] = (__bf16)p[i];
        }
      }
      if constexpr (BITS == 32) {
        store_f(mf + e, m, left, al);
        store_f(vf + e, v, left, al);
      } else {
        f32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          r[i] = i < left ? __fsqrt_rn(v[i]) : 0.f;
          m[i] = i < left ? m[i] : 0.f;
        }
        float ms, vs;
        store_b(mb + e, encode(m, false, ms), left, al);
        store_b(vb + e, encode(r, true, vs), left, al);
        if (lane == 0) {
          m_scale[at / 256] = ms;
          v_scale[at / 256] = vs;
        }
      }
    }
  }
  // the last block to end counts the step (every block has read it by then)
  if (threadIdx.x == 0) {
    const uint32_t done = __hip_atomic_fetch_add(a.done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    if (done == gridDim.x - 1) {
      *a.step += 1;
      *a.done = 0;
    }
  }
}

}  // namespace

hipError_t launch_adamw(const AdamwArgs& a, int bits, int grad_dtype, hipStream_t s) {
  const dim3 grid((unsigned)(a.runs > 0 ? a.runs : 1)), block(256);
  if (bits == 32) {
    if (grad_dtype == IM_BF16) hipLaunchKernelGGL((adamw_kernel<32, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((adamw_kernel<32, false>), grid, block, 0, s, a);
  } else {
    if (grad_dtype == IM_BF16) hipLaunchKernelGGL((adamw_kernel<8, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((adamw_kernel<8, false>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace learn
}  // namespace im
