// Edits of logits between a head and the token law: penalties for tokens that occurred, biases, grammar masks, and the row's
// log-sum-exp beside the edited logits.
//
//   edit_kernel      a workgroup takes a chunk of kChunk tokens of one sequence through all its slots.  It counts the sequence's
//                    history and sums its biases for these tokens in LDS, holds both per token in registers, and per slot reads the
//                    logits once, writes them once and leaves a (max, sum exp) pair per wavefront.  Slot m + 1 differs from slot m by
//                    one token of the prefix, which is added to the table on the way.
//   edit_lse_kernel  a wavefront per row merges the pairs.
//
// Counts are whole numbers, and a token's biases are added in the order of their list, so nothing depends on the order in which
// threads arrive.
//
// Log-sum-exp.  Maxima are clamped to the finite numbers, m in [-FLT_MAX, FLT_MAX], and differences x - m are taken before anything is
// multiplied: a row of nothing but -inf sums to 0 and ends at -inf, one of the type's lowest value keeps it, +inf gives +inf, NaN NaN.
#include <float.h>

#include "head_common.hpp"
#include "wave_ops.hpp"

namespace fef {
namespace {

constexpr int NT = 256, NW = NT / kWave;
constexpr int kPer = 8;              // tokens per thread: two runs of four
constexpr int kChunk = NT * kPer;
constexpr unsigned kInPrompt = 1u << 31;  // of a table entry; the other bits are the count
constexpr float kLog2e = 1.44269504088896340736f;

struct __attribute__((packed, aligned(4))) Float4 { float v[4]; };
struct __attribute__((packed, aligned(2))) Half4 { unsigned short v[4]; };

__device__ __forceinline__ float finite_max(float m) { return fminf(fmaxf(m, -FLT_MAX), FLT_MAX); }
__device__ __forceinline__ float exp_diff(float x, float m) { return __builtin_amdgcn_exp2f((x - m) * kLog2e); }

// Biases of the chunk's tokens, summed per token in the order of the list: the entries that name one of them are packed in order, and
// the first of each token adds up its like.
__device__ void sum_biases(const EditArgs& a, int b, int c0, float* s_bias, int* s_id, float* s_val, int* s_base) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t* ids = a.bias_ids + (size_t)b * a.n_bias;
  const float* vals = a.bias_values + (size_t)b * a.n_bias;
  for (int t0 = 0; t0 < a.n_bias; t0 += NT) {
    const int t = t0 + tid;
    const unsigned id = t < a.n_bias ? (unsigned)ids[t] : 0xffffffffu;
    const bool mine = id < (unsigned)a.V && id - (unsigned)c0 < (unsigned)kChunk;
    const unsigned long long vote = __ballot(mine);
    if (lane == 0) s_base[wave] = __popcll(vote);
    __syncthreads();
    int before = __popcll(vote & ((1ull << lane) - 1)), total = 0;
    for (int w = 0; w < NW; ++w) {
      if (w < wave) before += s_base[w];
      total += s_base[w];
    }
    if (mine) {
      s_id[before] = (int)id - c0;
      s_val[before] = vals[t];
    }
    __syncthreads();
    if (tid < total) {
      const int id0 = s_id[tid];
      bool first = true;
      for (int j = 0; j < tid; ++j) first = first && s_id[j] != id0;
      if (first) {
        float sum = s_bias[id0];
        for (int j = tid; j < total; ++j) sum += s_id[j] == id0 ? s_val[j] : 0.f;
        s_bias[id0] = sum;
      }
    }
    __syncthreads();
  }
}

template <bool BF16>
__global__ __launch_bounds__(NT) void edit_kernel(EditArgs a, int chunks, long work) {
  __shared__ unsigned s_cnt[kChunk];
  __shared__ float s_bias[kChunk];
  __shared__ int s_id[NT];
  __shared__ float s_val[NT];
  __shared__ int s_base[NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool counts = a.repetition || a.presence || a.frequency;
  for (long w = blockIdx.x; w < work; w += gridDim.x) {
    const int b = (int)(w / chunks), chunk = (int)(w - (long)b * chunks), c0 = chunk * kChunk;
    __syncthreads();  // the tables of the chunk before are no longer read
    for (int i = tid; i < kChunk; i += NT) {
      s_cnt[i] = 0;
      s_bias[i] = 0.f;
    }
    __syncthreads();
    if (counts && a.history_max) {
      const int len = a.history_len ? min(max(a.history_len[b], 0), a.history_max) : a.history_max;
      const int prompt = a.prompt_len ? min(max(a.prompt_len[b], 0), len) : 0;
      const int32_t* h = a.history + (size_t)b * a.history_max;
      for (int i = tid; i < len; i += NT) {
        const unsigned at = (unsigned)h[i] - (unsigned)c0;
        if (at < (unsigned)kChunk) {
          if (i < prompt) atomicOr(&s_cnt[at], kInPrompt);
          else atomicAdd(&s_cnt[at], 1u);
        }
      }
    }
    if (a.n_bias) sum_biases(a, b, c0, s_bias, s_id, s_val, s_base);
    __syncthreads();
    const float rep = a.repetition ? a.repetition[b] : 1.f;
    const float pres = a.presence ? a.presence[b] : 0.f;
    const float freq = a.frequency ? a.frequency[b] : 0.f;
    unsigned cnt[kPer];
    float bias[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      cnt[i] = s_cnt[(i / 4) * (NT * 4) + tid * 4 + i % 4];
      bias[i] = s_bias[(i / 4) * (NT * 4) + tid * 4 + i % 4];
    }
    for (int m = 0; m < a.K; ++m) {
      if (counts && a.prefix && m > 0) {
        const unsigned at = (unsigned)a.prefix[(size_t)b * a.K + m - 1] - (unsigned)c0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) cnt[i] += at == (unsigned)((i / 4) * (NT * 4) + tid * 4 + i % 4) ? 1u : 0u;
      }
      const uint32_t* words =
          a.masks ? a.allowed + ((size_t)b * a.masks + (a.masks > 1 ? m : 0)) * ((size_t)(a.V + 31) / 32) : nullptr;
      float y[kPer];
#pragma unroll
      for (int q = 0; q < kPer / 4; ++q) {
        const int c = c0 + q * (NT * 4) + tid * 4;
        const long at = (long)b * a.seq_stride + (long)m * a.slot_stride + c;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = -INFINITY;
          if (c + i < a.V) {
            if constexpr (BF16) x = __builtin_bit_cast(float, (unsigned)((const unsigned short*)a.logits)[at + i] << 16);
            else x = ((const float*)a.logits)[at + i];
          }
          const unsigned n = cnt[4 * q + i];
          if (counts && n) {
            x = x > 0.f ? x / rep : x * rep;
            const float times = (float)(n & ~kInPrompt);
            x -= freq * times;
            x -= times > 0.f ? pres : 0.f;
          }
          if (a.n_bias) x += bias[4 * q + i];
          x *= a.inv_tau;
          if (c + i >= a.V || (words && !((words[(c + i) >> 5] >> ((c + i) & 31)) & 1))) x = -INFINITY;
          if (c + i < a.V) a.out[(long)b * a.out_seq_stride + (long)m * a.out_slot_stride + c + i] = x;
          y[4 * q + i] = x;
        }
      }
      float mx = y[0];
#pragma unroll
      for (int i = 1; i < kPer; ++i) mx = fmaxf(mx, y[i]);
      mx = finite_max(wave_max(mx));
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) sum += exp_diff(y[i], mx);
      sum = wave_sum(sum);
      if (lane == 0) a.partials[((size_t)b * a.K + m) * (size_t)(chunks * NW) + chunk * NW + wave] = make_float2(mx, sum);
    }
  }
}

// A wavefront per row.
__global__ __launch_bounds__(NT) void edit_lse_kernel(EditArgs a, int nP) {
  const int lane = threadIdx.x & 63;
  const long r = (long)blockIdx.x * NW + (threadIdx.x >> 6);
  if (r >= (long)a.B * a.K) return;
  const float2* P = a.partials + (size_t)r * nP;
  float mx = -FLT_MAX, sm = 0.f;
  for (int t = lane; t < nP; t += kWave) {
    const float2 p = P[t];
    const float m = fmaxf(mx, p.x);
    sm = sm * exp_diff(mx, m) + p.y * exp_diff(p.x, m);
    mx = m;
  }
  const float m = wave_max(mx);
  sm = wave_sum(sm * exp_diff(mx, m));
  if (lane == 0) a.out_lse[r] = m + logf(sm);
}

}  // namespace

int edit_partials(int V) { return (V + kChunk - 1) / kChunk * NW; }

hipError_t launch_edit(const EditArgs& a) {
  const int chunks = (a.V + kChunk - 1) / kChunk;
  const long work = (long)chunks * a.B;
  const dim3 grid((unsigned)(work < (1L << 20) ? work : (1L << 20)));
  if (a.bf16) hipLaunchKernelGGL(edit_kernel<true>, grid, dim3(NT), 0, a.stream, a, chunks, work);
  else hipLaunchKernelGGL(edit_kernel<false>, grid, dim3(NT), 0, a.stream, a, chunks, work);
  if (a.out_lse) {
    const long rows = (long)a.B * a.K;
    hipLaunchKernelGGL(edit_lse_kernel, dim3((unsigned)((rows + NW - 1) / NW)), dim3(NT), 0, a.stream, a, chunks * NW);
  }
  return hipGetLastError();
}

}  // namespace fef
