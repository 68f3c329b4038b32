// The two products of the cross-entropy's gradients for float32 inputs (see head_grad.hip): C[m, n] = sum_k A[m, k] B[k, n] on
// v_mfma_f32_16x16x4_f32, products and sums in binary32.
#include "head_common.hpp"

namespace fef {
namespace {

constexpr int kThreads = 256, BT = 64, BK = 32, kPitch = BT + 4;

// Rows that are not whole pieces of 16 bytes: tiles of 64 x 64, four wavefronts of 32 x 32, k-steps of 32 through LDS and registers.
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
        rb[j] = kk < a.K && nn < a.N && kk < a.b_rows ? a.B[(size_t)kk * a.N + nn] : 0.f;
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
            *p = a.labels && a.labels[m] < 0 ? 0.f : a.add ? *p + acc[n][t][i] : acc[n][t][i];
          }
    }
}


// Rows of whole pieces of 16 bytes (N a multiple of 4, K of 32, A's rows of 64): four wavefronts, tiles of 16 MT WM rows x 128 columns, k-steps
// of 32 straight from memory to LDS, one ahead, in 64 KB, so that two workgroups share a CU.
//
// What bounds it: the multiplies (157 TFLOP/s at 2.4 GHz): 1000 rows of d = 2048, V = 126464 3.8 ms each (137 TFLOP/s).  With tiles of 64 x 64
// and everything through registers a call of 2048 rows of d = 1024, V = 100000 took 14.9 ms, now 10.2.  Few rows: bytes and the first trip, 16 rows of d = 1024, V = 32000 25 us for grad_h
// and 40 for grad_w (131 MB written).
//
// The order of the four k of a multiply is free as long as both operands have the same: multiply j of 16 columns takes k = 4 g + j from lane
// group g, so where k is contiguous a lane reads its four multiplies' operands in one piece of 16 bytes.  Rows of 32 k (A, not AT): chunk c of 16
// bytes of row r at c ^ ((r >> 1) & 7).  Rows of columns: chunk c of 64 bytes of row k at c ^ ((k >> 2) & 3), so that the four lane groups, in
// rows 4 apart, read from different banks.
template <bool AT, int MT, int WM>
__global__ __launch_bounds__(kThreads, 2) void grad_product_f32_wide_kernel(ProductF32Args a) {
  constexpr int WN = 4 / WM, NT = 8 / WN, BM = 16 * MT * WM, BN = 128;
  constexpr int kStageA = BM * BK * 4, kStageB = BN * BK * 4;
  constexpr int kLoadsA = kStageA / 1024, LA = kLoadsA / 4, LB = kStageB / 1024 / 4;
  static_assert(kLoadsA % 4 == 0 && LA <= 4 && LB == 4 && (!AT || BM >= 64), "four chunks to a row");
  __shared__ __align__(16) char lds[2 * (kStageA + kStageB)];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN, i16 = lane & 15, g = lane >> 4;
  const int mt = (a.M + BM - 1) / BM, nt = (a.N + BN - 1) / BN;
  // consecutive tiles on one XCD
  const int tiles = mt * nt * a.shares, per = (tiles + 7) / 8;
  const int id = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || id >= tiles) return;
  const int share = id / (mt * nt), at = id - share * (mt * nt);
  const int m0 = (AT ? at / nt : at % mt) * BM, n0 = (AT ? at % nt : at / mt) * BN;
  const int nk_all = a.K / BK;
  const int k_begin = (int)((long)share * nk_all / a.shares), nk = (int)((long)(share + 1) * nk_all / a.shares) - k_begin;
  const float* ga[LA];
  const float* gb[LB];
#pragma unroll
  for (int q = 0; q < LA; ++q) {
    const int s = (wave * LA + q) * 64 + lane;
    if constexpr (AT) {
      const int k = s / (BM / 4), p = s % (BM / 4);
      const int m = m0 + ((p >> 2) ^ ((k >> 2) & 3)) * 16 + (p & 3) * 4;
      ga[q] = a.A + (size_t)(k_begin * BK + k) * a.lda + min(m, (a.M - 1) & ~3) - q * 256;
    } else {
      const int m = s / 8, c = (s & 7) ^ ((m >> 1) & 7);
      ga[q] = a.A + (size_t)min(m0 + m, a.M - 1) * a.lda + k_begin * BK + c * 4 - q * 256;
    }
  }
  int rows[LB];
#pragma unroll
  for (int q = 0; q < LB; ++q) {
    const int s = (wave * LB + q) * 64 + lane;
    const int k = s / (BN / 4), p = s % (BN / 4);
    const int n = n0 + ((p >> 2) ^ ((k >> 2) & 3)) * 16 + (p & 3) * 4;
    rows[q] = k_begin * BK + k;
    gb[q] = a.B + min(n, a.N - 4) - q * 256;
  }
  const uint32_t slotA = lds_offset(lds) + wave * LA * 1024, slotB = lds_offset(lds) + 2 * kStageA + wave * LB * 1024;
  auto group = [&](const float* const (&p)[4], uint32_t off) __attribute__((always_inline)) {
    const __bf16* const q[4] = {(const __bf16*)p[0], (const __bf16*)p[1], (const __bf16*)p[2], (const __bf16*)p[3]};
    load_group_to_lds<false>(q, off);
  };
  auto load = [&](int stage) __attribute__((always_inline)) {
    const uint32_t off = __builtin_amdgcn_readfirstlane(slotA + stage * kStageA);
    if constexpr (LA == 4) group(ga, off);
    else
#pragma unroll
      for (int q = 0; q < LA; ++q) load_to_lds_16(ga[q] + q * 256, off + q * 1024);
#pragma unroll
    for (int q = 0; q < LA; ++q) ga[q] += AT ? (long)BK * a.lda : (long)BK;
    const float* p[4];
#pragma unroll
    for (int q = 0; q < LB; ++q) {
      p[q] = gb[q] + (size_t)min(rows[q], a.b_rows - 1) * a.N;  // rows past the last meet zeros of A
      rows[q] += BK;
    }
    group(p, __builtin_amdgcn_readfirstlane(slotB + stage * kStageB));
  };
  floatx4 acc[MT][NT];
#pragma unroll
  for (int n = 0; n < MT; ++n)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[n][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  if (nk > 0) load(0);
  for (int k = 0; k < nk; ++k) {
    wait_newer<0>();
    lds_barrier();
    if (k + 1 < nk) load((k + 1) & 1);
    const float* sA = reinterpret_cast<const float*>(lds + (k & 1) * kStageA);
    const float* sB = reinterpret_cast<const float*>(lds + 2 * kStageA + (k & 1) * kStageB);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {  // 16 columns of k
      float x[NT][4], y[MT][4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int t = 0; t < NT; ++t) x[t][j] = sB[(ks * 16 + 4 * g + j) * BN + ((wn * NT + t) ^ g) * 16 + i16];
#pragma unroll
      for (int n = 0; n < MT; ++n) {
        if constexpr (AT) {
#pragma unroll
          for (int j = 0; j < 4; ++j) y[n][j] = sA[(ks * 16 + 4 * g + j) * BM + ((wm * MT + n) ^ g) * 16 + i16];
        } else {
          const int m = (wm * MT + n) * 16 + i16;
          *reinterpret_cast<floatx4*>(y[n]) = *reinterpret_cast<const floatx4*>(sA + m * BK + (((ks * 4 + g) ^ ((m >> 1) & 7)) * 4));
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < MT; ++n)
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[t][j], y[n][j], acc[n][t], 0, 0, 0);
    }
  }
  float* C = a.C + (size_t)share * a.stride;
#pragma unroll
  for (int n = 0; n < MT; ++n)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int m = m0 + (wm * MT + n) * 16 + i16, c = n0 + (wn * NT + t) * 16 + 4 * g;
      if (m < a.M && c < a.N) {
        floatx4* p = reinterpret_cast<floatx4*>(C + (size_t)m * a.N + c);
        *p = a.labels && a.labels[m] < 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : a.add ? *p + acc[n][t] : acc[n][t];
      }
    }
}

template <bool AT, int MT, int WM>
hipError_t launch_wide(const ProductF32Args& a, hipStream_t stream) {
  constexpr int BM = 16 * MT * WM;
  const long tiles = (long)((a.M + BM - 1) / BM) * ((a.N + 127) / 128) * a.shares;
  if (tiles >= 1L << 24) return hipErrorInvalidValue;  // 2^32 threads
  const dim3 grid((unsigned)(8 * ((tiles + 7) / 8))), threads(kThreads);
  hipLaunchKernelGGL((grad_product_f32_wide_kernel<AT, MT, WM>), grid, threads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace

// Rows of a tile where the rows of B are pieces of 16 bytes (no more than there are: 16 rows of d = 1024, V = 32000 take 25 us in tiles of 32), and
// shares of k: two workgroups per CU, steps of 32.
static int wide_rows(int M) { return M <= 32 ? 32 : M <= 64 ? 64 : 128; }
int grad_f32_shares(int M, int N, int K) {
  const bool wide = N % 4 == 0;
  const long tiles = wide ? (long)((M + wide_rows(M) - 1) / wide_rows(M)) * ((N + 127) / 128) : (long)((M + BT - 1) / BT) * ((N + BT - 1) / BT);
  const long steps = (K + BK - 1) / BK, want = tiles >= 512 ? 1 : 512 / tiles;
  return (int)(want < steps ? want : steps);
}

hipError_t launch_grad_product_f32(const ProductF32Args& a, bool at, hipStream_t stream) {
  if (a.N % 4 == 0) {
    // grad_w of a short vocabulary: lower tiles, so that more CUs have one (61 rows of d = 64, V = 1000: 16 tiles of 64, or 8 of 128)
    if (at && (long)((a.M + 127) / 128) * ((a.N + 127) / 128) < 128) return launch_wide<true, 4, 1>(a, stream);
    if (at) return launch_wide<true, 4, 2>(a, stream);
    switch (wide_rows(a.M)) {
      case 32: return launch_wide<false, 2, 1>(a, stream);
      case 64: return launch_wide<false, 4, 1>(a, stream);
      default: return launch_wide<false, 4, 2>(a, stream);
    }
  }
  const dim3 grid((unsigned)((long)((a.M + BT - 1) / BT) * ((a.N + BT - 1) / BT) * a.shares)), threads(kThreads);
  if (at) hipLaunchKernelGGL(grad_product_f32_kernel<true>, grid, threads, 0, stream, a);
  else hipLaunchKernelGGL(grad_product_f32_kernel<false>, grid, threads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace fef
