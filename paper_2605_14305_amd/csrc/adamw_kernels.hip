// One AdamW step over a list of tensors (fef_adamw_step): elementwise, one pass over parameters, gradients and states.
//
// What bounds it: bytes.  bf16 parameters with float32 copies and states move 28 bytes per element, with states in 8 bits 16.06: 218 M elements
// in nine tensors 1125 us (5.4 TB/s), 518 M elements with states in 8 bits 1510 us (5.5 TB/s), where torch's in-place addition reaches 5.9 and its copy
// 4.8; eleven small tensors of 0.1 M elements 7 us, a launch.
//
// A workgroup takes 4096 consecutive elements of one tensor; the table of tensors is in the kernel's arguments, so one launch serves
// kAdamwTensors of them.  A wavefront takes 256 elements at a time, four neighbours per lane, which is a block of the 8-bit states: their
// largest magnitude is a maximum over one wavefront.
//
// Every operation is one rounding to float32 in the order of the header (no contraction to fused multiply-adds), so an element's result does
// not depend on the tensor's alignment or length, or on what else is in the list.
#include <type_traits>

#include "fef_device.hpp"

namespace fef {
namespace {

constexpr int kThreads = 256, kLane = 4, kUnits = 4;  // elements per lane and unit; units of 256 elements per wavefront
constexpr int kBlock = kWave * kLane;
static_assert(kBlock == kAdamwBlock && kAdamwChunk == kThreads * kLane * kUnits, "");

struct AdamwLaunch {
  AdamwConst c;
  int count;
  int first[kAdamwTensors];  // first workgroup of each tensor
  AdamwTensor t[kAdamwTensors];
};
static_assert(sizeof(AdamwLaunch) <= 4096, "kernel arguments");

// Four neighbours as the widest loads and stores there are (WIDE: 16-byte aligned rows, all four exist), or one by one.
template <bool WIDE, class T>
__device__ __forceinline__ void load4(T (&x)[4], const T* p, long at, long n) {
  if constexpr (WIDE) {
    using V = std::conditional_t<sizeof(T) == 4, uint4, std::conditional_t<sizeof(T) == 2, uint2, unsigned>>;
    const V v = *reinterpret_cast<const V*>(p + at);
    __builtin_memcpy(x, &v, sizeof v);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = at + j < n ? p[at + j] : T(0);
  }
}
template <bool WIDE, class T>
__device__ __forceinline__ void store4(const T (&x)[4], T* p, long at, long n) {
  if constexpr (WIDE) {
    using V = std::conditional_t<sizeof(T) == 4, uint4, std::conditional_t<sizeof(T) == 2, uint2, unsigned>>;
    V v;
    __builtin_memcpy(&v, x, sizeof v);
    *reinterpret_cast<V*>(p + at) = v;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at + j < n) p[at + j] = x[j];
  }
}

// Largest of a wavefront, as bit patterns of magnitudes: a NaN is larger than all numbers and stays.
__device__ __forceinline__ float top_of(const float (&x)[4]) {
  unsigned m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) m = max(m, __builtin_bit_cast(unsigned, x[j]) & 0x7fffffffu);
#pragma unroll
  for (int d = 32; d; d >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, d));
  const float top = __builtin_bit_cast(float, m);
  return top < kAdamwLeast ? 0.f : top;  // the reciprocal of a smaller one is not a number
}

__device__ __forceinline__ void decode4(float (&x)[4], const uint8_t (&code)[4], float scale) {
  int w;
  __builtin_memcpy(&w, code, 4);
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  x[0] = lo[0] * scale; x[1] = lo[1] * scale; x[2] = hi[0] * scale; x[3] = hi[1] * scale;
}
// The two quotients of a block's codes and scale, in one rounding each or by reciprocals, as the header says: one bit here moves the elements next
// to the middle of two codes.
__device__ __forceinline__ float of_448(float top, int reciprocal) {
  const float q = (reciprocal ? 1.f : 448.f) / top;  // one division, whichever it is
  return reciprocal ? q * 448.f : q;
}
__device__ __forceinline__ float scale_of(float top, int reciprocal) {
  return reciprocal ? top * (1.f / 448.f) : top / 448.f;
}
// (top is 0 where the block is held as zeros)
__device__ __forceinline__ void encode4(uint8_t (&code)[4], const float (&x)[4], float top, int reciprocal) {
  const float inv = of_448(top, reciprocal);
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
  w = top == 0.f ? 0 : w;
  __builtin_memcpy(code, &w, 4);
}

template <class P, class G, bool EIGHT, bool WIDE>
__device__ __forceinline__ void adamw_chunk(const AdamwConst& c, const AdamwTensor& t, long base) {
#pragma clang fp contract(off)
  using S = std::conditional_t<EIGHT, uint8_t, float>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float lr = c.schedule ? c.schedule[0] : c.lr, c1 = c.schedule ? c.schedule[1] : c.c1, c2 = c.schedule ? c.schedule[2] : c.c2;
  const float gs = c.grad_scale ? *c.grad_scale : 1.f;
  const float keep = 1.f - lr * t.weight_decay, rate = lr * c1;
  P p[kUnits][4];
  G g[kUnits][4];
  float x[kUnits][4], m_top[kUnits], v_top[kUnits];
  S m[kUnits][4], v[kUnits][4];
  long at[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const long unit = base / kBlock + u * (kThreads / kWave) + wave;
    at[u] = unit * kBlock + lane * kLane;
    load4<WIDE>(g[u], (const G*)t.grad, at[u], t.n);
    if (t.master) load4<WIDE>(x[u], t.master, at[u], t.n);
    else load4<WIDE>(p[u], (const P*)t.param, at[u], t.n);
    load4<WIDE>(m[u], (const S*)t.m, at[u], t.n);
    load4<WIDE>(v[u], (const S*)t.v, at[u], t.n);
    if constexpr (EIGHT) {
      const bool some = unit * kBlock < t.n;
      m_top[u] = some ? t.m_scale[unit] : 0.f;
      v_top[u] = some ? t.v_scale[unit] : 0.f;
    }
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    float mf[4], vf[4];
    if constexpr (EIGHT) {
      decode4(mf, m[u], m_top[u]);
      decode4(vf, v[u], v_top[u]);
#pragma unroll
      for (int j = 0; j < 4; ++j) vf[j] = vf[j] * vf[j];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) { mf[j] = m[u][j]; vf[j] = v[u][j]; }
    }
    float r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float gj = (float)g[u][j] * gs;
      if (!t.master) x[u][j] = (float)p[u][j];
      mf[j] = mf[j] * c.b1 + gj * c.one_b1;
      vf[j] = vf[j] * c.b2 + gj * gj * c.one_b2;
      r[j] = sqrtf(vf[j]);
      x[u][j] = x[u][j] * keep - mf[j] / (r[j] * c2 + c.eps) * rate;
      p[u][j] = (P)x[u][j];
    }
    if constexpr (EIGHT) {
      if (!WIDE) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (at[u] + j >= t.n) mf[j] = r[j] = 0.f;
      }
      const float mt = top_of(mf), vt = top_of(r);
      encode4(m[u], mf, mt, c.reciprocal);
      encode4(v[u], r, vt, c.reciprocal);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (vt > 0.f && r[j] > 0.f && v[u][j] == 0) v[u][j] = 1;  // the smallest code: a step is never divided by eps alone for lack of bits
      if (lane == 0 && at[u] < t.n) {
        const long unit = at[u] / kBlock;
        t.m_scale[unit] = scale_of(mt, c.reciprocal);
        t.v_scale[unit] = scale_of(vt, c.reciprocal);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) { m[u][j] = mf[j]; v[u][j] = vf[j]; }
    }
    if (t.master) store4<WIDE>(x[u], t.master, at[u], t.n);
    store4<WIDE>(p[u], (P*)t.param, at[u], t.n);
    store4<WIDE>(m[u], (S*)t.m, at[u], t.n);
    store4<WIDE>(v[u], (S*)t.v, at[u], t.n);
  }
}

template <class P, class G, bool EIGHT>
__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamwLaunch a) {
  int i = 0;  // the tensor of this workgroup
  for (int j = 1; j < a.count; ++j)
    if ((int)blockIdx.x >= a.first[j]) i = j;
  const AdamwTensor& t = a.t[i];
  const long base = (long)((int)blockIdx.x - a.first[i]) * kAdamwChunk;
  if (t.wide && base + kAdamwChunk <= t.n) adamw_chunk<P, G, EIGHT, true>(a.c, t, base);
  else adamw_chunk<P, G, EIGHT, false>(a.c, t, base);
}

}  // namespace

hipError_t launch_adamw(const AdamwConst& c, const AdamwTensor* tensors, int count, bool bf16, bool grad_bf16, bool eight, hipStream_t stream) {
  AdamwLaunch a;
  a.c = c;
  for (int i = 0; i < count;) {
    long groups = 0;
    a.count = 0;
    for (; i < count && a.count < kAdamwTensors; ++i) {
      const long more = (tensors[i].n + kAdamwChunk - 1) / kAdamwChunk;
      if (!more) continue;
      if (a.count && groups + more > kAdamwGroups) break;
      a.first[a.count] = (int)groups;
      a.t[a.count++] = tensors[i];
      groups += more;
    }
    if (!groups) break;
    const dim3 grid((unsigned)groups), threads(kThreads);
    if (bf16 && grad_bf16) {
      if (eight) hipLaunchKernelGGL((adamw_kernel<__bf16, __bf16, true>), grid, threads, 0, stream, a);
      else hipLaunchKernelGGL((adamw_kernel<__bf16, __bf16, false>), grid, threads, 0, stream, a);
    } else if (bf16) {
      if (eight) hipLaunchKernelGGL((adamw_kernel<__bf16, float, true>), grid, threads, 0, stream, a);
      else hipLaunchKernelGGL((adamw_kernel<__bf16, float, false>), grid, threads, 0, stream, a);
    } else if (grad_bf16) {
      if (eight) hipLaunchKernelGGL((adamw_kernel<float, __bf16, true>), grid, threads, 0, stream, a);
      else hipLaunchKernelGGL((adamw_kernel<float, __bf16, false>), grid, threads, 0, stream, a);
    } else {
      if (eight) hipLaunchKernelGGL((adamw_kernel<float, float, true>), grid, threads, 0, stream, a);
      else hipLaunchKernelGGL((adamw_kernel<float, float, false>), grid, threads, 0, stream, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fef
