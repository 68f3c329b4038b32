// The two products of the cross-entropy's gradients for float32 inputs (see head_grad.hip): C[m, n] = sum_k A[m, k] B[k, n] on
// v_mfma_f32_16x16x4_f32, products and sums in binary32.  Any sizes; used by small models.
//
// Workgroup tile 64 x 64, four wavefronts of 32 x 32, k-steps of 32 through LDS and registers.
#include "head_common.hpp"

namespace fef {
namespace {

constexpr int kThreads = 256, BT = 64, BK = 32, kPitch = BT + 4;

// AT: A is [K][M], else [M][K].
template <bool AT>
__global__ __launch_bounds__(kThreads) void grad_product_f32_kernel(ProductF32Args a) {
  __shared__ float sA[2][BK * kPitch], sB[2][BK * kPitch];  // [k][m], [k][n]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1, i16 = lane & 15, g = lane >> 4;
  const int mt = (a.M + BT - 1) / BT, nt = (a.N + BT - 1) / BT;
  const int tile = blockIdx.x % (mt * nt), share = blockIdx.x / (mt * nt);
  const int m0 = tile / nt * BT, n0 = tile % nt * BT;
  const int nk_all = (a.K + BK - 1) / BK;
  const int k_begin = (int)((long)share * nk_all / a.shares), k_end = (int)((long)(share + 1) * nk_all / a.shares);
  float ra[8], rb[8];
  auto fetch = [&](int step) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = j * kThreads + tid;
      {
        const int k = AT ? e / BT : e % BK, m = AT ? e % BT : e / BK;
        const int kk = step * BK + k, mm = m0 + m;
        ra[j] = kk < a.K && mm < a.M ? a.A[AT ? (size_t)kk * a.lda + mm : (size_t)mm * a.lda + kk] : 0.f;
      }
      {
        const int k = e / BT, n = e % BT, kk = step * BK + k, nn = n0 + n;
        rb[j] = kk < a.K && nn < a.N ? a.B[(size_t)kk * a.N + nn] : 0.f;
      }
    }
  };
  auto put = [&](int s) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = j * kThreads + tid;
      sA[s][(AT ? e / BT : e % BK) * kPitch + (AT ? e % BT : e / BK)] = ra[j];
      sB[s][e / BT * kPitch + e % BT] = rb[j];
    }
  };
  floatx4 acc[2][2] = {};
  if (k_begin < k_end) {
    fetch(k_begin);
    put(0);
  }
  __syncthreads();
  for (int step = k_begin; step < k_end; ++step) {
    const int s = (step - k_begin) & 1;
    if (step + 1 < k_end) fetch(step + 1);
#pragma unroll
    for (int c = 0; c < BK / 4; ++c) {
      float x[2], y[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        x[t] = sB[s][(4 * c + g) * kPitch + wn * 32 + t * 16 + i16];
        y[t] = sA[s][(4 * c + g) * kPitch + wm * 32 + t * 16 + i16];
      }
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t) acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[t], y[n], acc[n][t], 0, 0, 0);
    }
    if (step + 1 < k_end) put(s ^ 1);
    __syncthreads();
  }
  float* C = a.C + (size_t)share * a.stride;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int m = m0 + wm * 32 + n * 16 + i16, c = n0 + wn * 32 + t * 16 + 4 * g;
      if (m < a.M)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + i < a.N) {
            float* p = C + (size_t)m * a.N + c + i;
            *p = a.add ? *p + acc[n][t][i] : acc[n][t][i];
          }
    }
}

}  // namespace

int grad_f32_shares(int M, int N, int K) {
  const long tiles = (long)((M + BT - 1) / BT) * ((N + BT - 1) / BT), steps = (K + BK - 1) / BK;
  const long want = tiles >= 256 ? 1 : 256 / tiles, most = (steps + 3) / 4;
  return (int)(want < most ? want : most);
}

hipError_t launch_grad_product_f32(const ProductF32Args& a, bool at, hipStream_t stream) {
  const dim3 grid((unsigned)((long)((a.M + BT - 1) / BT) * ((a.N + BT - 1) / BT) * a.shares)), threads(kThreads);
  if (at) hipLaunchKernelGGL(grad_product_f32_kernel<true>, grid, threads, 0, stream, a);
  else hipLaunchKernelGGL(grad_product_f32_kernel<false>, grid, threads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace fef
