// Edits of logits between a head and the token law: penalties for tokens that occurred, biases, grammar masks, and the row's
// log-sum-exp beside the edited logits.
//
//   edit_kernel      a workgroup takes a chunk of tokens of one sequence through some of its slots.  It counts the sequence's history and
//                    sums its biases for these tokens in LDS; from then on a thread reads and writes the entries of its own tokens only,
//                    so nothing waits: slot m + 1 differs from slot m by one token of the prefix, which that token's owner adds.  Per slot
//                    the logits are read once, written once, and leave a (max, sum exp) pair per wavefront.  A bit per token says
//                    whether it has an entry; the others see a multiplication and the mask.
//   edit_lse_kernel  a wavefront per row merges the pairs, where a row is more than one chunk.
//
// Counts are whole numbers, and a token's biases are added in the order of their list, so nothing depends on the order in which
// threads arrive.
//
// Bound: the read and the write of the logits (32 x 16 slots of V = 151936, 622 MB: 131 us without any edit, 4.7 TB/s, a plain copy of as
// much 121 to 130; with penalties, biases and masks 144 to 149, the edits' instructions), in small calls the way through the tables and the
// second launch (8 slots of V = 126464: 7.6 and 2 us).  Counting the history again for every chunk beats a table in memory, which would have to
// be cleared and needs atomics across XCDs.  Stores are non-temporal: grammar masks alone on 128 rows of V = 126464 37 -> 28 us.
//
// Log-sum-exp.  Maxima are clamped to the finite numbers, m in [-FLT_MAX, FLT_MAX], and differences x - m are taken before anything is
// multiplied: a row of nothing but -inf sums to 0 and ends at -inf, one of the type's lowest value keeps it, +inf gives +inf, NaN NaN.
#include <float.h>

#include "fef_device.hpp"
#include "wave_ops.hpp"

namespace fef {
namespace {

constexpr unsigned kInPrompt = 1u << 31;  // of a table entry; the other bits are the count
constexpr float kLog2e = 1.44269504088896340736f;

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short halfx4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef int intx4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float finite_max(float m) { return fminf(fmaxf(m, -FLT_MAX), FLT_MAX); }
__device__ __forceinline__ float exp_diff(float x, float m) { return __builtin_amdgcn_exp2f((x - m) * kLog2e); }

// Division by one y: x / y = (x / d) s with s a power of two such that r = 1 / d is a normal number; the quotient's remainder corrects it,
// so it is off by a step at most (what is infinite stays so).  y = 0 and an infinite y end as s.  32 x 16 slots of V = 151936 with every
// edit take 148.4 us so, with a plain division per logit 149.6 (8 x 65536 tokens of history 22.9 and 23.3).
struct Divisor {
  float d, r, s;
};
__device__ __forceinline__ Divisor divisor(float y) {
  const float m = fabsf(y);
  const float up = m < 0x1p-64f ? 0x1p64f : m > 0x1p64f ? 0x1p-64f : 1.f;
  const bool end = m == 0.f || m == INFINITY;
  const float d = end ? 1.f : y * up;
  return {d, 1.f / d, end ? copysignf(m == 0.f ? INFINITY : 0.f, y) : up};
}
__device__ __forceinline__ float divided(float x, const Divisor& y) {
  const float q = x * y.r, e = __builtin_fmaf(-q, y.d, x);
  return (fabsf(q) < INFINITY ? __builtin_fmaf(e, y.r, q) : q) * y.s;
}

// Biases of the chunk's tokens, summed per token in the order of the list (its first NT entries are given): the entries that name one of
// them are packed in order, and the first of each token adds up its like.
template <int NT, int kPer>
__device__ void sum_biases(const EditArgs& a, int b, int c0, int id0, float value0, float* s_bias, int* s_id, float* s_val, int* s_base) {
  constexpr int NW = NT / kWave, kChunk = NT * kPer;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t* ids = a.bias_ids + (size_t)b * a.n_bias;
  const float* vals = a.bias_values + (size_t)b * a.n_bias;
  for (int t0 = 0; t0 < a.n_bias; t0 += NT) {
    const int t = t0 + tid;
    const unsigned id = t0 == 0 ? (unsigned)id0 : t < a.n_bias ? (unsigned)ids[t] : 0xffffffffu;
    const float value = t0 == 0 ? value0 : t < a.n_bias ? vals[t] : 0.f;
    const bool mine = id < (unsigned)a.V && id - (unsigned)c0 < (unsigned)kChunk;
    const unsigned long long vote = __ballot(mine);
    if (lane == 0) s_base[wave] = __popcll(vote);
    __syncthreads();
    int before = __popcll(vote & ((1ull << lane) - 1)), total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const int n = s_base[w];
      before += w < wave ? n : 0;
      total += n;
    }
    if (mine) {
      s_id[before] = (int)id - c0;
      s_val[before] = value;
    }
    __syncthreads();
    if (tid < total) {
      const int own = s_id[tid];
      bool first = true;
      for (int j = 0; j < tid; ++j) first = first && s_id[j] != own;
      if (first) {
        float sum = s_bias[own];
        for (int j = tid; j < total; ++j) sum += s_id[j] == own ? s_val[j] : 0.f;
        s_bias[own] = sum;
      }
    }
    if (t0 + NT < a.n_bias) __syncthreads();
  }
}

// Workgroup: (sequence, chunk, group of `slots` slots), slots innermost; sequences from b0 on.  WHOLE: the chunk is the vocabulary.
template <int NT, int kPer, bool BF16, bool WHOLE>
__global__ __launch_bounds__(NT) void edit_kernel(EditArgs a, int b0, int chunks, int slots, int groups) {
  constexpr int NW = NT / kWave, kChunk = NT * kPer;
  __shared__ __attribute__((aligned(16))) unsigned s_cnt[kChunk];
  __shared__ __attribute__((aligned(16))) float s_bias[kChunk];
  __shared__ int s_id[NT];
  __shared__ float s_val[NT];
  __shared__ int s_base[NW];
  __shared__ float2 s_pair[WHOLE ? 2 : 1][NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned per_chunk = blockIdx.x / (unsigned)groups;
  const int m0 = (int)(blockIdx.x - per_chunk * (unsigned)groups) * slots, m1 = min(m0 + slots, a.K);
  const int chunk = (int)(per_chunk % (unsigned)chunks), b = b0 + (int)(per_chunk / (unsigned)chunks), c0 = chunk * kChunk;
  const bool counts = a.repetition || a.presence || a.frequency;
  const bool whole = c0 + kChunk <= a.V;
  const unsigned here = whole ? kChunk : a.V - c0;  // tokens of the chunk: ids behind them stand for none
  const int left = a.V - c0 - tid * 4;  // tokens from this thread's first on

  float x[kPer];
  uint32_t word[kPer / 4];
  auto fetch = [&](int m) {
    const size_t row = (size_t)b * a.seq_stride + (size_t)m * a.slot_stride + c0;
    const uint32_t* words =
        a.masks ? a.allowed + ((size_t)b * a.masks + (a.masks > 1 ? m : 0)) * ((size_t)(a.V + 31) / 32) + c0 / 32 : nullptr;
#pragma unroll
    for (int q = 0; q < kPer / 4; ++q) {
      const unsigned c = q * (NT * 4) + tid * 4;
      word[q] = ~0u;
      if (words && (whole || left > q * (NT * 4))) word[q] = words[c >> 5] >> (c & 31);
      if (whole) {
        if constexpr (BF16) {
          const halfx4_any v = *reinterpret_cast<const halfx4_any*>((const unsigned short*)a.logits + row + c);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[4 * q + i] = __builtin_bit_cast(float, (unsigned)v[i] << 16);
        } else {
          const floatx4_any v = *reinterpret_cast<const floatx4_any*>((const float*)a.logits + row + c);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[4 * q + i] = v[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[4 * q + i] = -INFINITY;
          if (left > q * (NT * 4) + i) {
            if constexpr (BF16) x[4 * q + i] = __builtin_bit_cast(float, (unsigned)((const unsigned short*)a.logits)[row + c + i] << 16);
            else x[4 * q + i] = ((const float*)a.logits)[row + c + i];
          }
        }
      }
    }
  };
  // All that the table is made of is asked for at once, in front of the logits; a list's first part stays in registers.
  const bool history = counts && a.history_max, prefix = counts && a.prefix;
  const bool table = history || prefix || a.n_bias;
  const int32_t* h = a.history + (size_t)b * a.history_max;
  const int first = history && tid * 4 + 4 <= a.history_max ? 4 : 0;  // ids of the first NT * 4 that this thread holds
  intx4_any ids = {-1, -1, -1, -1};
  if (first) ids = *reinterpret_cast<const intx4_any*>(h + tid * 4);
  int bias_id = -1;
  float bias_value = 0.f;
  if (tid < a.n_bias) {
    bias_id = a.bias_ids[(size_t)b * a.n_bias + tid];
    bias_value = a.bias_values[(size_t)b * a.n_bias + tid];
  }
  const int len = !history ? 0 : a.history_len ? min(max(a.history_len[b], 0), a.history_max) : a.history_max;
  const int prompt = history && a.prompt_len ? min(max(a.prompt_len[b], 0), len) : 0;
  const float rep = a.repetition ? a.repetition[b] : 1.f;
  const Divisor by = divisor(rep);
  const float pres = a.presence ? a.presence[b] : 0.f;
  const float freq = a.frequency ? a.frequency[b] : 0.f;
  fetch(m0);

  unsigned touched = 0;  // bit i: token i of this thread has a count or a bias
  if (table) {
#pragma unroll
    for (int q = 0; q < kPer / 4; ++q) {
      reinterpret_cast<uint4*>(s_cnt)[q * NT + tid] = make_uint4(0, 0, 0, 0);
      reinterpret_cast<float4*>(s_bias)[q * NT + tid] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncthreads();
    if (history) {
      auto count = [&](int i, int id) {
        const unsigned at = (unsigned)id - (unsigned)c0;
        if (at < here) {
          if (i < prompt) atomicOr(&s_cnt[at], kInPrompt);
          else atomicAdd(&s_cnt[at], 1u);
        }
      };
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (tid * 4 + e < len && first) count(tid * 4 + e, ids[e]);
      int i0 = NT * 4;
      if (a.history_max < i0) i0 = a.history_max / 4 * 4;  // what no thread holds four of
      for (; i0 + 16 * NT <= len; i0 += 16 * NT) {
        intx4_any v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const intx4_any*>(h + i0 + (j * NT + tid) * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) count(i0 + (j * NT + tid) * 4 + e, v[j][e]);
      }
      for (int i = i0 + tid; i < len; i += NT) count(i, h[i]);
    }
    if (a.n_bias) sum_biases<NT, kPer>(a, b, c0, bias_id, bias_value, s_bias, s_id, s_val, s_base);
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kPer / 4; ++q) {
      const uint4 n = reinterpret_cast<const uint4*>(s_cnt)[q * NT + tid];
      const float4 v = reinterpret_cast<const float4*>(s_bias)[q * NT + tid];
      touched |= (n.x || v.x != 0.f ? 1u : 0u) << (4 * q) | (n.y || v.y != 0.f ? 2u : 0u) << (4 * q) |
                 (n.z || v.z != 0.f ? 4u : 0u) << (4 * q) | (n.w || v.w != 0.f ? 8u : 0u) << (4 * q);
    }
  }
  // From here on a thread reads and writes its own tokens' entries only.
  auto add_prefix = [&](int m) {
    const unsigned at = (unsigned)a.prefix[(size_t)b * a.K + m] - (unsigned)c0;
    if (at < here && ((at >> 2) & (NT - 1)) == (unsigned)tid) {
      ++s_cnt[at];
      touched |= 1u << (at / (NT * 4) * 4 + (at & 3));
    }
  };
  if (prefix)
    for (int m = 0; m < m0; ++m) add_prefix(m);

  for (int m = m0; m < m1; ++m) {
    if (__any(touched != 0)) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (touched >> i & 1) {
          const unsigned at = (i / 4) * (NT * 4) + tid * 4 + i % 4, n = s_cnt[at];
          float z = x[i];
          if (n) {
            const float times = (float)(n & ~kInPrompt);
            z = z > 0.f ? divided(z, by) : z * rep;
            z -= freq * times;
            z -= times > 0.f ? pres : 0.f;
          }
          x[i] = z + s_bias[at];
        }
    }
    float* out = a.out + (size_t)b * a.out_seq_stride + (size_t)m * a.out_slot_stride + c0;
    float y[kPer];
#pragma unroll
    for (int q = 0; q < kPer / 4; ++q) {
      const unsigned c = q * (NT * 4) + tid * 4;
      floatx4_any v;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[4 * q + i] = v[i] = word[q] >> i & 1 ? x[4 * q + i] * a.inv_tau : -INFINITY;
      if (whole) {
        __builtin_nontemporal_store(v, reinterpret_cast<floatx4_any*>(out + c));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (left > q * (NT * 4) + i) out[c + i] = v[i];
      }
    }
    if (m + 1 < m1) fetch(m + 1);
    float mx = y[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) mx = fmaxf(mx, y[i]);
    mx = finite_max(wave_max(mx));
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += exp_diff(y[i], mx);
    sum = wave_sum(sum);
    if constexpr (!WHOLE) {
      if (lane == 0) a.partials[((size_t)b * a.K + m) * (size_t)(chunks * NW) + chunk * NW + wave] = make_float2(mx, sum);
    } else if (a.out_lse) {  // the row's pairs are all here
      if (lane == 0) s_pair[m & 1][wave] = make_float2(mx, sum);
      __syncthreads();
      if (wave == 0) {
        const float2 pair = lane < NW ? s_pair[m & 1][lane] : make_float2(-FLT_MAX, 0.f);
        const float top = wave_max(pair.x), all = wave_sum(pair.y * exp_diff(pair.x, top));
        if (lane == 0) a.out_lse[(size_t)b * a.K + m] = top + logf(all);
      }
    }
    if (prefix) add_prefix(m);
  }
}

constexpr int kLseThreads = 256;

// A wavefront per row.
__global__ __launch_bounds__(kLseThreads) void edit_lse_kernel(EditArgs a, int nP) {
  const int lane = threadIdx.x & 63;
  const long r = (long)blockIdx.x * (kLseThreads / kWave) + (threadIdx.x >> 6);
  if (r >= (long)a.B * a.K) return;
  const float2* P = a.partials + (size_t)r * nP;
  float mx = -FLT_MAX, sm = 0.f;
  for (int t0 = lane; t0 < nP; t0 += 8 * kWave) {  // eight loads in flight
    float2 p[8];
    float m = mx;
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = t0 + j * kWave < nP ? P[t0 + j * kWave] : make_float2(-FLT_MAX, 0.f);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, p[j].x);
    sm *= exp_diff(mx, m);
#pragma unroll
    for (int j = 0; j < 8; ++j) sm += p[j].y * exp_diff(p[j].x, m);
    mx = m;
  }
  const float m = wave_max(mx);
  sm = wave_sum(sm * exp_diff(mx, m));
  if (lane == 0) a.out_lse[r] = m + logf(sm);
}

}  // namespace

// A pair per wavefront and chunk: per 256 tokens at most, chunks of up to 4096.
int edit_partials(int V) { return (V + 4095) / 4096 * 16; }

template <int NT, int kPer, bool WHOLE = false>
static void launch_edit_of(const EditArgs& a) {
  const int chunks = (a.V + NT * kPer - 1) / (NT * kPer);
  const long units = (long)chunks * a.B;
  // Slots of a chunk go to workgroups of their own until there are four per CU, as long as the history that each of them counts again is
  // short against its logits.
  int groups = 1;
  while (groups < a.K && units * groups < 1024 && a.history_max <= (long)((a.K + groups - 1) / groups) * (NT * kPer / 2)) groups *= 2;
  if (groups > a.K) groups = a.K;
  const int slots = (a.K + groups - 1) / groups;
  groups = (a.K + slots - 1) / slots;
  const long most = (1L << 32) / NT - 1;  // a launch holds fewer than 2^32 threads
  const long per = most / ((long)chunks * groups);
  for (long b0 = 0; b0 < a.B; b0 += per) {
    const dim3 grid((unsigned)((a.B - b0 < per ? a.B - b0 : per) * chunks * groups));
    if (a.bf16) hipLaunchKernelGGL((edit_kernel<NT, kPer, true, WHOLE>), grid, dim3(NT), 0, a.stream, a, (int)b0, chunks, slots, groups);
    else hipLaunchKernelGGL((edit_kernel<NT, kPer, false, WHOLE>), grid, dim3(NT), 0, a.stream, a, (int)b0, chunks, slots, groups);
  }
  if (a.out_lse && !WHOLE) {
    const long rows = (long)a.B * a.K;
    constexpr int kRows = kLseThreads / kWave;
    hipLaunchKernelGGL(edit_lse_kernel, dim3((unsigned)((rows + kRows - 1) / kRows)), dim3(kLseThreads), 0, a.stream, a, chunks * (NT / kWave));
  }
}

// Threads and tokens per thread.  Many threads per token where a long history has to be counted for every chunk (8 sequences of 65536, 4
// slots of V = 126464: 23 us, with 512 x 8 28, with 256 x 8 32; of 8192 20 in all three); of large calls 512 x 8 rather than 256 x 8 (32 x 16
// slots of V = 126464, histories of 8192: 131 against 142); else 256 x 8, which start earlier and fill the CUs more evenly (64 x 4 slots of
// V = 32000 24 us, with 512 x 8 30).  Where such a chunk holds the vocabulary it also finishes the row, without a second launch (one row of
// V = 2000 9.2 -> 7.9 us, 64 x 8 slots of it 12.6 -> 10.4; larger workgroups that hold 8000 tokens lose more by waiting for each
// other in every slot: 64 x 16 slots 25 -> 45).
hipError_t launch_edit(const EditArgs& a) {
  if (a.history_max >= 16384) launch_edit_of<512, 4>(a);
  else if ((long)a.B * a.K * a.V >= 1L << 25) launch_edit_of<512, 8>(a);
  else if (a.V <= 2048) launch_edit_of<256, 8, true>(a);
  else launch_edit_of<256, 8>(a);
  return hipGetLastError();
}

}  // namespace fef
