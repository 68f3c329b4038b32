// Logits of the vocabulary head from weights in 4 bits (OCP MX, MXFP4): logits[r, v] = inv_tau sum_k h[r, k] w[v, k],
// w[v, k] = e2m1(code) 2^(scale - 127) with a scale per 32 codes.
//
// Numbers.  A code times its scale has two significant bits, so it is exact in bf16, and v_cvt_scalef32_pk_bf16_fp4 makes two of
// them with their scale in one instruction (checked over all codes and scales: exact, subnormals too, scale 255 gives NaN).  The
// products run on v_mfma_f32_16x16x32_bf16 with float32 sums.  The scaled 8-bit multiplies would take the codes as they are, but add
// with 13 to 15 bits only (measured: error 2^-13.5 of the sum of magnitudes), and two of them per bf16 value cost as much time.
// Hidden states in float32 are cut into three bf16 parts, 8 bits each, whose sum is the value itself.
//
// Layout.  The multiply adds over k in any order as long as both operands agree on it.  Lane l = (token or row l % 16, group g = l / 16)
// takes the 32 codes of block 4 u + g (16 bytes and one scale), which feed four multiplies of 8 codes per lane; of h it takes the same
// columns.  Tokens are the rows of D, so a lane ends with four consecutive tokens of one row of h.
#include "head_common.hpp"

namespace fef {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int intx4 __attribute__((ext_vector_type(4)));

// Eight codes of a dword as bf16, k ascending.
__device__ __forceinline__ bf16x8 unpack8(int codes, float scale) {
  union { bf16x2 p[4]; bf16x8 v; } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return u.v;
}

// x = hi + mid + lo with 8 significant bits each, cut off towards zero; infinities and NaN are in hi alone.
__device__ __forceinline__ void split3(const float* x, bf16x8 (&part)[3]) {
  union { unsigned short s[8]; bf16x8 v; } u[3];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const unsigned b = __builtin_bit_cast(unsigned, x[i]);
    const bool finite = (b & 0x7f800000u) != 0x7f800000u;
    const float hi = __builtin_bit_cast(float, b & 0xffff0000u);
    const float r = finite ? x[i] - hi : 0.f;
    const unsigned rb = __builtin_bit_cast(unsigned, r);
    const float lo = r - __builtin_bit_cast(float, rb & 0xffff0000u);
    const unsigned quiet = !finite && (b & 0x007fffffu) ? 0x00400000u : 0u;
    u[0].s[i] = (unsigned short)((b | quiet) >> 16);
    u[1].s[i] = (unsigned short)(rb >> 16);
    u[2].s[i] = (unsigned short)(__builtin_bit_cast(unsigned, lo) >> 16);
  }
#pragma unroll
  for (int p = 0; p < 3; ++p) part[p] = u[p].v;
}

constexpr int kRowsPerWave = 64;

// A wavefront per 16 tokens and 64 rows; grid (groups of 64 tokens, groups of 64 rows).
template <bool F32>
__global__ __launch_bounds__(256) void mx4_kernel(Mx4Args a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i16 = lane & 15, g = lane >> 4;
  const int nb = a.d / 32;  // blocks of 32 codes per row
  const int tok0 = (blockIdx.x * 4 + wave) * 16;
  if (tok0 >= a.V) return;
  const int tok = min(tok0 + i16, a.V - 1);
  const uint8_t* codes = a.codes + (size_t)tok * (a.d / 2);
  const uint8_t* scales = a.scales + (size_t)tok * nb;
  for (int row0 = blockIdx.y * kRowsPerWave; row0 < a.R; row0 += gridDim.y * kRowsPerWave) {
    floatx4 acc[4] = {};
    for (int u = 0; u < (nb + 3) / 4; ++u) {
      const int kb = 4 * u + g;
      const bool in = kb < nb;
      const intx4 c = in ? *reinterpret_cast<const intx4*>(codes + kb * 16) : intx4{0, 0, 0, 0};
      const float s = __builtin_bit_cast(float, (in ? (int)scales[kb] : 127) << 23);
      bf16x8 w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = unpack8(c[j], s);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = min(row0 + 16 * q + i16, a.R - 1);
        const size_t at = (size_t)row * a.d + (size_t)kb * 32;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (F32) {
            float x[8] = {};
            if (in) {
              *reinterpret_cast<floatx4*>(x) = *reinterpret_cast<const floatx4*>((const float*)a.h + at + 8 * j);
              *reinterpret_cast<floatx4*>(x + 4) = *reinterpret_cast<const floatx4*>((const float*)a.h + at + 8 * j + 4);
            }
            bf16x8 part[3];
            split3(x, part);
#pragma unroll
            for (int p = 2; p >= 0; --p) acc[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j], part[p], acc[q], 0, 0, 0);
          } else {
            bf16x8 x = {};
            if (in) x = *reinterpret_cast<const bf16x8*>((const __bf16*)a.h + at + 8 * j);
            acc[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j], x, acc[q], 0, 0, 0);
          }
        }
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) asm volatile("" : "+v"(acc[q]));  // the multiplies need all lanes: none may move under a condition
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int row = row0 + 16 * q + i16;
      if (row >= a.R) continue;
      float* out = a.logits + (size_t)row * a.ld;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (tok0 + 4 * g + i < a.V) out[tok0 + 4 * g + i] = acc[q][i] * a.inv_tau;
    }
  }
}

}  // namespace

hipError_t launch_mx4(const Mx4Args& a) {
  const int groups = (a.R + kRowsPerWave - 1) / kRowsPerWave;
  const dim3 grid((a.V + 63) / 64, groups < 1024 ? groups : 1024);
  if (a.f32) FEF_LAUNCH_HEAD(mx4_kernel<true>, grid, dim3(256), a, a);
  else FEF_LAUNCH_HEAD(mx4_kernel<false>, grid, dim3(256), a, a);
  return hipGetLastError();
}

}  // namespace fef
