// One AdamW step over many tensors, bound by memory: an element reads and writes
// 28 bytes with fp32 states and gradients, 14 with 8-bit states and bf16
// gradients, 2 more with a bf16 copy; one launch moves everything once. A block
// takes runs of kRun elements of one tensor from a table made with the plan; a
// wave takes 256 neighbouring elements at a time, four a lane: one block of an
// 8-bit state, whose largest magnitude is a maximum over the wave. All loads of a
// run are issued before its first step. Measured at 2^26 elements: 5.3 TB/s with
// 32-bit states (a large copy reaches 5.4), 4.9 TB/s with 8-bit ones, where the
// conversions (about 50 operations an element) share the time.
#include "learn_adamw.h"

#include "learn_tile.h"

namespace im {
namespace learn {
namespace {

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
  scale = scale < 0x1p-126f ? 0x1p-126f : scale;
  if (top >= 0x7f800000u) scale = __builtin_nanf("");   // not finite: the block is NaN
  const float inverse = __fdiv_rn(1.0f, scale);
  f32x4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // y / scale: the product with the reciprocal, corrected once. Its magnitude is 448 at
    // most but for a rounding, which the conversion takes back.
    float q = y[i] * inverse;
    q = fmaf(fmaf(-q, scale, y[i]), inverse, q);
    if (least) q = y[i] > 0.f ? fmaxf(q, 0x1p-9f) : q;
    x[i] = q;
  }
  return to_e4m3(x);
}

// Square root to 1 unit. The instruction takes what lies below 2^-126 for 0 (there
// a v is of gradients below 1e-19, and their quotient would be infinite): such go in scaled.
__device__ __forceinline__ float root(float x) {
  const bool small = x < 0x1p-96f;
  const float r = __builtin_amdgcn_sqrtf(small ? x * 0x1p64f : x);
  return small ? r * 0x1p-32f : r;
}

// x^t by squaring: relative error below t 2^-52, and t x^t is bounded.
__device__ __forceinline__ double power(double x, int64_t t) {
  double y = 1.0;
  for (; t > 0; t >>= 1) {
    if (t & 1) y *= x;
    x *= x;
  }
  return y;
}

// Four elements a lane: one block of an 8-bit state a wave.
template <int BITS>
struct Four {
  f32x4 p, g, m, v;
  uint32_t cm, cv;
  float ms, vs;
};

template <int BITS, bool HALF>
struct Step {
  const AdamwArgs& a;
  Global<float> param, mf, vf, m_scale, v_scale;
  Global<uint8_t> mb, vb;
  Global<const float> gf;
  Global<const __bf16> gh;
  Global<__bf16> copy;
  float keep, r1, r2, scale;
  bool copies;

  __device__ __forceinline__ Step(const AdamwArgs& args, const im_adamw_tensor& t, float r1_, float r2_, float scale_)
      : a(args), r1(r1_), r2(r2_), scale(scale_) {
    param = global<float>(t.param);
    mf = global<float>(t.m), vf = global<float>(t.v);
    mb = global<uint8_t>(t.m), vb = global<uint8_t>(t.v);
    m_scale = global<float>(t.m_scale), v_scale = global<float>(t.v_scale);
    gf = global<const float>(t.grad), gh = global<const __bf16>(t.grad);
    copy = global<__bf16>(t.copy), copies = t.copy != nullptr;
    keep = t.decay ? a.keep : 1.f;
  }
  // the wave's elements at .. at + 255, of which lane l has left (from l 4 on; 4 and al: at once)
  __device__ __forceinline__ void load(Four<BITS>& f, int64_t at, int left, bool al) const {
    const int64_t e = at + (int)(threadIdx.x % 64) * 4;
    f.p = load_f(param + e, left, al);
    f.g = HALF ? load_h(gh + e, left, al) : load_f(gf + e, left, al);
    if constexpr (BITS == 32) {
      f.m = load_f(mf + e, left, al);
      f.v = load_f(vf + e, left, al);
    } else {
      f.cm = load_b(mb + e, left, al);
      f.cv = load_b(vb + e, left, al);
      f.ms = m_scale[at / 256];
      f.vs = v_scale[at / 256];
    }
  }
  __device__ __forceinline__ void step(Four<BITS>& f, int64_t at, int left, bool al) const {
    const int64_t e = at + (int)(threadIdx.x % 64) * 4;
    if constexpr (BITS == 8) {
      f.m = from_e4m3(f.cm);
      f.v = from_e4m3(f.cv);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f.m[i] = f.m[i] * f.ms;
        const float r = f.v[i] * f.vs;
        f.v[i] = r * r;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      {
        // every product rounded by itself: a state on the border between two codes falls to
        // the side where elementary fp32 operations put it (a flipped code is 6 % of it)
#pragma clang fp contract(off)
        const float g = f.g[i] * scale;
        f.m[i] = f.m[i] * a.beta1f + g * a.omb1;
        f.v[i] = f.v[i] * a.beta2f + g * g * a.omb2;
      }
      // root and reciprocal to 1 unit: the parameter's own rounding is coarser
      const float d = root(f.v[i] * r2) + a.eps;   // 0 or 2^-126 at least: the reciprocal takes those
      f.p[i] = f.p[i] * keep - f.m[i] * r1 * __builtin_amdgcn_rcpf(d) * a.lr;
    }
    store_f(param + e, f.p, left, al);
    if (copies) {
      if (left >= 4 && al) {
        bf16x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = (__bf16)f.p[i];
        *(Global<bf16x4>)(copy + e) = o;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i < left) copy[e + i] = (__bf16)f.p[i];
      }
    }
    if constexpr (BITS == 32) {
      store_f(mf + e, f.m, left, al);
      store_f(vf + e, f.v, left, al);
    } else {
      f32x4 r;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        r[i] = i < left ? root(f.v[i]) : 0.f;
        f.m[i] = i < left ? f.m[i] : 0.f;
      }
      float ms, vs;
      store_b(mb + e, encode(f.m, false, ms), left, al);
      store_b(vb + e, encode(r, true, vs), left, al);
      if (threadIdx.x % 64 == 0) {
        m_scale[at / 256] = ms;
        v_scale[at / 256] = vs;
      }
    }
  }
};

template <int BITS, bool HALF>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamwArgs a) {
  const int64_t t = *a.step + 1;
  const float r1 = (float)(1.0 / (1.0 - power(a.beta1, t))), r2 = (float)(1.0 / (1.0 - power(a.beta2, t)));
  const float scale = a.scale ? *a.scale : 1.f;
  const int wave = threadIdx.x / 64, lane4 = (threadIdx.x % 64) * 4;
  for (int64_t k = blockIdx.x; k < a.runs; k += gridDim.x) {
    const AdamwRun run = a.table[k];
    const im_adamw_tensor tensor = a.tensors[run.tensor];
    const Step<BITS, HALF> s(a, tensor, r1, r2, scale);
    const int64_t first = run.first + wave * 256;
    if (run.aligned && run.first + kRun <= tensor.n) {   // all of the wave's loads in flight at once
      Four<BITS> f[kRun / 1024];
#pragma unroll
      for (int i = 0; i < kRun / 1024; ++i) s.load(f[i], first + i * 1024, 4, true);
#pragma unroll
      for (int i = 0; i < kRun / 1024; ++i) s.step(f[i], first + i * 1024, 4, true);
    } else {
      const int64_t end = run.first + kRun < tensor.n ? run.first + kRun : tensor.n;
      for (int64_t at = first; at < end; at += 1024) {
        const int64_t over = end - at - lane4;
        const int left = over >= 4 ? 4 : (int)over;
        Four<BITS> f;
        s.load(f, at, left, run.aligned);
        s.step(f, at, left, run.aligned);
      }
    }
  }
  // The last block to end counts the step: every block has read it by then (its value went
  // into what the barrier waits for). Nothing else passes between blocks: no fence, which
  // would write the L2 back for each (measured: 40 ns a block, 1.3 ms with 16,384 blocks).
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t done = __hip_atomic_fetch_add(a.done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (done == gridDim.x - 1) {
      *a.step = t;
      *a.done = 0;
    }
  }
}

}  // namespace

hipError_t launch_adamw(const AdamwArgs& a, int bits, int grad_dtype, hipStream_t s) {
  const dim3 grid((unsigned)(a.runs < 1 ? 1 : (a.runs < a.blocks ? a.runs : a.blocks))), block(256);
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
