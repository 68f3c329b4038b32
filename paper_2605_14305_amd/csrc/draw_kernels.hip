// Truncated laws and draws from them (fef_draw_logits): top-k, top-p and min-p over the logits of a row, the truncated logits, their
// log-sum-exp, and a token by inverse CDF.
//
// The order of a row's tokens is (key descending, id ascending), key being the logit's bits mapped to an unsigned number of the same order.
// Whatever the limits, what is kept is a beginning of that order: tokens with key > T, and those with key == T up to an id I.
//
// One workgroup takes a row and finds (T, I) without sorting it:
//   1. read the row: its maximum, and how many tokens and how much mass lie in each of 4096 bins of 1/32 (y - ref, ref = 0; a row whose
//      maximum lies outside [-32, 62) is read again with ref = max - 62).  Tokens below the lowest bin are counted in it.
//   2. sums over the bins from the top: the bin where top-k ends, and the bins where top-p can end, given what top-k may leave.
//   3. read the row again: what lies above these bins is kept and written, what lies in them goes to a list in LDS, the rest is -inf.
//   4. the list is sorted; rank and mass before each of its tokens give (T, I); what it keeps is written.
//   5. the token: sums of the kept mass per tile of ids, then the ids of one tile.
// A list longer than kList (a vocabulary of equal logits) is narrowed down by its keys instead, 12 bits per reading.
//
// Masses decide which token is the last, so they are exact to 2^-44 or so: a weight is computed in 64 bits and added as a whole number of
// 2^-s, which no order of the atomics changes.  In step 1 weights are relative to their bin's middle, |y - middle| <= 1/64, where a
// polynomial of degree 5 is exact to 2^-45.
#include <math.h>

#include "fef_device.hpp"

namespace fef {
namespace {

typedef unsigned long long u64;

constexpr int T = 1024, kWaves = T / kWave;
constexpr int kBins = 4096, kList = 2048, kTiles = 512, kTile = 4 * T;
constexpr float kWidth = 32.f;  // bins per unit of y
constexpr double kReached = 1 - 0x1p-44;  // of a mass: sums that meet top_p exactly (equal logits) are not missed for their last bits
constexpr float kNone = -2e38f;  // smaller numbers stand for no token

__device__ __forceinline__ unsigned key_of(float y) {
  const unsigned u = __builtin_bit_cast(unsigned, y);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(unsigned k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

struct Shared {
  unsigned cnt[kBins];
  u64 mass[kBins];       // fixed point; after the sums: the mass above the bin, a double
  u64 list[kList];
  u64 tile[kTiles];
  u64 part[kWaves];
  unsigned list_n, kept;
  unsigned found[4];
  double value[2];
  u64 sum;
};

// Sum over the workgroup of everything up to and with this thread, and the total; D is u64 or double.  Fixed order.
template <class D>
__device__ __forceinline__ D block_scan(D x, D* part, D& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const D o = __shfl_up(x, d);
    if (lane >= d) x += o;
  }
  __syncthreads();
  if (lane == 63) part[wave] = x;
  __syncthreads();
  D before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) before = all;
    all += part[w];
  }
  total = all;
  return before + x;
}

template <bool BF16>
struct Row {
  const void* x;
  float* out;      // or NULL
  int V, head;     // vector j holds tokens 4 j - head ..
  float inv_tau;
  bool out_wide;

  __device__ __forceinline__ float at(int v) const {
    const float f = BF16 ? (float)((const __bf16*)x)[v] : ((const float*)x)[v];
    return f * inv_tau + 0.f;  // -0 is 0
  }
  __device__ __forceinline__ int vectors() const { return (V + head + 3) >> 2; }
  // Tokens 4 j - head + {0, 1, 2, 3}; those outside of the row as -inf.
  __device__ __forceinline__ void load(int j, float (&y)[4]) const {
    const int v = 4 * j - head;
    if (v >= 0 && v + 4 <= V) {
      if constexpr (BF16) {
        const uint2 u = *reinterpret_cast<const uint2*>((const __bf16*)x + v);
        y[0] = __builtin_bit_cast(float, u.x << 16); y[1] = __builtin_bit_cast(float, u.x & 0xffff0000u);
        y[2] = __builtin_bit_cast(float, u.y << 16); y[3] = __builtin_bit_cast(float, u.y & 0xffff0000u);
      } else {
        const float4 f = *reinterpret_cast<const float4*>((const float*)x + v);
        y[0] = f.x; y[1] = f.y; y[2] = f.z; y[3] = f.w;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = y[i] * inv_tau + 0.f;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = v + i >= 0 && v + i < V ? at(v + i) : -INFINITY;
    }
  }
  __device__ __forceinline__ void store(int v, const float (&y)[4]) const {
    if (out_wide && v >= 0 && v + 4 <= V) {
      *reinterpret_cast<float4*>(out + v) = make_float4(y[0], y[1], y[2], y[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (v + i >= 0 && v + i < V) out[v + i] = y[i];
    }
  }
};

// All tokens of a row, four at a time: f(first id, y[4]); ids outside of the row come as -inf.  Wavefronts stay whole.
template <bool BF16, class F>
__device__ __forceinline__ void each(const Row<BF16>& r, F f) {
  const int n = r.vectors(), lane = threadIdx.x & 63;
  for (int j0 = threadIdx.x - lane; j0 < n; j0 += 4 * T) {
    float y[4][4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (j0 + u * T < n) r.load(j0 + u * T + lane, y[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (j0 + u * T < n) f(4 * (j0 + u * T + lane) - r.head, y[u]);
  }
}

struct Bins {
  float ref;
  __device__ __forceinline__ int of(float y) const { return (int)fminf(fmaxf((y - ref) * kWidth + kBins / 2, 0.f), kBins - 1.f); }
  __device__ __forceinline__ double middle(int b) const { return (double)ref + ((b - kBins / 2) + 0.5) * (1.0 / kWidth); }
  // exp(y - middle of its bin)
  __device__ __forceinline__ double weight(float y, int b) const {
    const double t = (double)y - middle(b);
    if (fabs(t) > 1.0 / 63) return exp(t);  // the lowest bin has no lower end
    return 1.0 + t * (1.0 + t * (1.0 / 2 + t * (1.0 / 6 + t * (1.0 / 24 + t * (1.0 / 120)))));
  }
};

struct Limits {
  unsigned k;      // 0: none
  double p;        // >= 1: none
  unsigned least;  // smallest key that min-p keeps
};

// Which of the tokens that `in` admits is the last one: the need_n-th in the order, or, where by_mass, the first at which their mass
// (relative to exp(top)) reaches need_m.  Readings of the row narrow its key down; `ids` is how many of that key belong to it.
template <bool BF16, class In>
__device__ void narrow(Shared& s, const Row<BF16>& r, In in, bool by_mass, u64 need_n, double need_m, float top, double scale,
                       unsigned& last, unsigned& ids) {
  unsigned low = 0, bits = 32;
  while (bits) {
    const unsigned shift = bits > 12 ? bits - 12 : 0;
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += T) {
      s.cnt[b] = 0;
      s.mass[b] = 0;
    }
    __syncthreads();
    each(r, [&](int, const float(&y)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned k = key_of(y[i]);
        if (y[i] >= kNone && in(y[i]) && (bits == 32 || (k - low) >> bits == 0)) {
          const unsigned b = (k - low) >> shift;
          atomicAdd(&s.cnt[b], 1u);
          if (by_mass) atomicAdd(&s.mass[b], (u64)(exp((double)y[i] - (double)top) * scale + 0.5));
        }
      }
    });
    __syncthreads();
    // from the top: thread t has bins kBins - 1 - 4 t and the three below
    u64 c = 0, all;
    u64 m = 0, all_m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = kBins - 1 - 4 * (int)threadIdx.x - i;
      c += s.cnt[b];
      m += s.mass[b];
    }
    u64 c_at = block_scan(c, s.part, all) - c, m_at = block_scan(m, s.part, all_m) - m;
    if (threadIdx.x == 0) s.found[0] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = kBins - 1 - 4 * (int)threadIdx.x - i;
      const u64 m_next = m_at + s.mass[b], c_next = c_at + s.cnt[b];
      // exactly one bin; the last one with tokens where rounding leaves the mass short
      if (s.cnt[b] && (by_mass ? (double)m_at < need_m && ((double)m_next >= need_m || c_next == all) : c_at < need_n && c_next >= need_n)) {
        s.found[0] = b;
        s.found[1] = s.cnt[b];
        s.sum = by_mass ? m_at : c_at;
      }
      m_at = m_next;
      c_at = c_next;
    }
    __syncthreads();
    if (by_mass) need_m -= (double)s.sum;
    else need_n -= s.sum;
    low += s.found[0] << shift;
    bits = shift;
  }
  last = low;
  const unsigned ties = s.found[1];
  if (by_mass) {
    const double w = floor(exp((double)of_key(low) - (double)top) * scale + 0.5);
    const double n = w > 0 ? ceil(need_m / w) : 1.0;
    ids = n < 1 ? 1 : n > ties ? ties : (unsigned)n;
  } else {
    ids = (unsigned)need_n;
  }
  __syncthreads();
}

template <bool BF16>
__device__ void draw_row(const DrawArgs& a, int row, Shared& s) {
  const int b = row / a.K, m = row - b * a.K;
  const int tid = threadIdx.x;
  Row<BF16> r;
  r.V = a.V;
  const long at = (long)b * a.seq_stride + (long)m * a.slot_stride;
  r.x = BF16 ? (const void*)((const __bf16*)a.logits + at) : (const void*)((const float*)a.logits + at);
  r.head = (int)(((uintptr_t)r.x / (BF16 ? 2 : 4)) & 3);
  r.out = a.out ? a.out + (long)b * a.out_seq_stride + (long)m * a.out_slot_stride : nullptr;
  r.out_wide = (((uintptr_t)r.out - 4 * (uintptr_t)r.head) & 15) == 0;
  float tau_inv = a.inv_tau;
  Limits lim;
  lim.k = a.top_k && a.top_k[b] > 0 ? (unsigned)a.top_k[b] : 0;
  lim.p = a.top_p && a.top_p[b] < 1.f ? (double)a.top_p[b] : 2.0;
  const float min_p = a.min_p && a.min_p[b] > 0.f ? a.min_p[b] : 0.f;
  bool law = true;
  if (a.temperatures) {
    const float t = a.temperatures[b];
    law = t >= 0.f;
    tau_inv = 1.f / t;
    if (!(tau_inv < INFINITY)) {
      tau_inv = 1.f;
      lim.k = 1;
    }
  }
  r.inv_tau = tau_inv;
  if (lim.p <= 0 || min_p > 1.f) lim.k = 1;
  if (lim.k == 1 || lim.p <= 0) lim.p = 2.0;
  const bool by_k = lim.k > 0, by_p = lim.p < 1;

  // 1. maximum and bins
  Bins bins{0.f};
  float top = 0.f;
  const int log_v = 32 - __clz(a.V);  // V < 2^log_v
  const double scale = __builtin_ldexp(1.0, 61 - log_v);
  for (int turn = 0;; ++turn) {
    __syncthreads();
    if (by_k || by_p)
      for (int i = tid; i < kBins; i += T) {
        s.cnt[i] = 0;
        s.mass[i] = 0;
      }
    if (tid == 0) {
      s.found[0] = 0;
      s.found[1] = 0;
      s.list_n = 0;
      s.kept = 0;
    }
    for (int i = tid; i < kTiles; i += T) s.tile[i] = 0;
    __syncthreads();
    unsigned high = 0;
    bool bad = false;
    each(r, [&](int, const float(&y)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bad |= !(y[i] < INFINITY);
        if (y[i] >= kNone) {
          high = max(high, key_of(y[i]));
          if (y[i] < INFINITY) {
            if (by_k | by_p) {
              const int bin = bins.of(y[i]);
              if (by_k) atomicAdd(&s.cnt[bin], 1u);
              if (by_p) atomicAdd(&s.mass[bin], (u64)(bins.weight(y[i], bin) * scale + 0.5));
            }
          }
        }
      }
    });
    atomicMax(&s.found[0], high);
    if (bad) s.found[1] = 1;
    __syncthreads();
    const unsigned top_key = s.found[0];
    law = law && top_key && !s.found[1];
    if (!law) break;
    top = of_key(top_key);
    if (turn || !(by_k || by_p) || (top >= -32.f && top < 62.f)) break;
    bins.ref = top - 62.f;
  }
  if (!law) {  // nothing kept
    if (r.out) {
      const float none[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      const int n = r.vectors();
      for (int j = tid; j < n; j += T) r.store(4 * j - r.head, none);
    }
    if (tid == 0) {
      if (a.out_tokens) a.out_tokens[row] = -1;
      if (a.out_conf) a.out_conf[row] = 0.f;
      if (a.out_kept) a.out_kept[row] = 0;
      if (a.out_lse) a.out_lse[row] = -INFINITY;
    }
    return;
  }
  // min-p as a key: the smallest y with exp(y - top) >= min_p
  lim.least = 0;
  if (min_p > 0.f && min_p <= 1.f) {
    const auto keeps = [&](unsigned k) { return exp((double)of_key(k) - (double)top) >= (double)min_p; };
    const double near = (double)top + log((double)min_p);
    unsigned low = key_of((float)(near - 0.01)), k = key_of(fminf((float)(near + 0.01), top));
    if (!keeps(k)) ++k;  // (numbers so far apart that one step misses the border)
    if (keeps(low)) k = low;
    while (k - low > 1 && k != low) {
      const unsigned mid = low + (k - low) / 2;
      if (keeps(mid)) k = mid;
      else low = mid;
    }
    lim.least = k;
  }

  // 2. where top-k and top-p end.  Zone: bins whose tokens have to be looked at one by one.
  int bin_k = -1, p_low = kBins, p_high = -1;  // -1: all of the row; zone of top-p: p_low .. p_high
  double above_k = 0;
  if (by_k || by_p) {
    unsigned c = 0;
    double w = 0, wi[4];
    unsigned ci[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int bin = kBins - 1 - 4 * tid - i;
      ci[i] = s.cnt[bin];
      wi[i] = s.mass[bin] ? (double)s.mass[bin] * exp(bins.middle(bin) - (double)top) : 0;  // of 2^-s
      c += ci[i];
      w += wi[i];
    }
    u64 all;
    double total;
    u64 c_at = block_scan((u64)c, s.part, all) - c;
    const double w_to = block_scan(w, (double*)s.part, total);
    double w_at = w_to - w;
    if (tid == 0) {
      s.found[0] = 0xffffffffu;
      s.found[1] = s.found[2] = 0xffffffffu;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int bin = kBins - 1 - 4 * tid - i;
      if (by_k && c_at < lim.k && c_at + ci[i] >= lim.k && lim.k < all) {
        s.found[0] = bin;
        s.value[0] = w_at;
        s.value[1] = w_at + wi[i];
      }
      s.cnt[bin] = (unsigned)c_at;                          // from here on: above the bin
      s.mass[bin] = __builtin_bit_cast(u64, w_at);
      c_at += ci[i];
      w_at += wi[i];
    }
    __syncthreads();
    const bool ends = s.found[0] != 0xffffffffu;
    bin_k = ends ? (int)s.found[0] : -1;
    above_k = ends ? s.value[0] : total;
    if (by_p) {
      // with the mass top-k leaves somewhere in [lowest, highest], and a little room for the sums' rounding
      const double lowest = lim.p * (ends ? s.value[0] : total) * (1 - 1e-12), highest = lim.p * (ends ? s.value[1] : total) * (1 + 1e-12);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int bin = kBins - 1 - 4 * tid - i;
        const double before = __builtin_bit_cast(double, s.mass[bin]);
        if (wi[i] > 0) {
          if (before + wi[i] >= lowest) atomicMin(&s.found[1], (unsigned)(kBins - 1 - bin));  // the first bin that may reach it
          if (before < highest) atomicMin(&s.found[2], (unsigned)bin);                        // the last one that may be needed
        }
      }
      __syncthreads();
      p_high = kBins - 1 - (int)s.found[1];
      p_low = (int)s.found[2];
      if (ends && p_low < bin_k) p_low = bin_k;
      if (ends && p_high < bin_k) p_high = bin_k;
    }
  }
  const int sure = max(by_p ? p_high : -1, by_p ? -1 : bin_k);  // bins above it are kept whole
  const bool zone = by_p || bin_k >= 0;
  auto in_k = [&](float y) { return bin_k >= 0 && bins.of(y) == bin_k; };
  auto in_p = [&](float y) { const int bin = bins.of(y); return by_p && bin >= p_low && bin <= p_high; };
  __syncthreads();

  // 3. what is sure, and the list
  const int tile_log = max(12, log_v - 9);
  auto weight = [&](float y) { return (u64)(exp((double)y - (double)top) * scale + 0.5); };
  unsigned kept_here = 0;
  each(r, [&](int v, const float(&y)[4]) {
    float o[4];
    u64 w[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool is = y[i] >= kNone;
      const int bin = is ? bins.of(y[i]) : -1;
      const bool keep = is && (!zone || bin > sure) && key_of(y[i]) >= lim.least;
      o[i] = keep ? y[i] : -INFINITY;
      w[i] = 0;
      if (keep) {
        w[i] = weight(y[i]);
        ++kept_here;
      }
      sum += w[i];
      if (is && zone && (bin == bin_k || (by_p && bin >= p_low && bin <= p_high))) {
        const unsigned p = atomicAdd(&s.list_n, 1u);
        if (p < kList) s.list[p] = ((u64)key_of(y[i]) << 32) | (unsigned)~(v + i);
      }
    }
    if (__ballot(sum != 0)) {
      const int v0 = v - 4 * (int)(threadIdx.x & 63);  // of the wavefront
      if (v0 >= 0 && v0 >> tile_log == (v0 + 255) >> tile_log) {
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        if (v == v0) atomicAdd(&s.tile[v >> tile_log], sum);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (w[i]) atomicAdd(&s.tile[(v + i) >> tile_log], w[i]);
      }
    }
    if (r.out) r.store(v, o);
  });
  if (kept_here) atomicAdd(&s.kept, kept_here);
  __syncthreads();

  // 4. the last token kept: key `last`, id `last_id`
  unsigned last = 0, last_id = 0x7fffffffu;
  if (zone) {
    const unsigned n = s.list_n;
    if (n <= kList) {
      unsigned size = 2;
      while (size < n) size <<= 1;
      for (unsigned i = n + tid; i < size; i += T) s.list[i] = 0;
      __syncthreads();
      for (unsigned k = 2; k <= size; k <<= 1)
        for (unsigned d = k >> 1; d; d >>= 1) {
          for (unsigned i = tid; i < size / 2; i += T) {
            const unsigned x = 2 * i - (i & (d - 1)), y = x + d;
            const u64 p = s.list[x], q = s.list[y];
            if ((p < q) == ((x & k) == 0)) {  // descending
              s.list[x] = q;
              s.list[y] = p;
            }
          }
          __syncthreads();
        }
      // two neighbours per thread: rank, and mass before, from the sums above their bin and the list's tokens of that bin in front
      float y[2];
      int bin[2];
      u64 w[2], dummy;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const unsigned p = 2 * tid + i;
        const bool is = p < n;
        y[i] = is ? of_key((unsigned)(s.list[p] >> 32)) : 0.f;
        bin[i] = is ? bins.of(y[i]) : -1;
        w[i] = is && by_p ? (u64)(bins.weight(y[i], bin[i]) * scale + 0.5) : 0;
      }
      u64 w_to = block_scan(w[0] + w[1], s.part, dummy);
      const u64 w_before[2] = {w_to - w[1] - w[0], w_to - w[1]};
      // where each token's bin begins in the list, by binary search
      unsigned first[2];
      u64 of_bin[2];
      __syncthreads();
      // sums in front of each list entry, for the entries that begin a bin
      u64* const sums = s.mass;  // entries of bins outside of the zone are not needed any more: the zone's are read first
      double above[2];
      unsigned c_above[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        above[i] = bin[i] >= 0 ? __builtin_bit_cast(double, s.mass[bin[i]]) : 0;
        c_above[i] = bin[i] >= 0 ? s.cnt[bin[i]] : 0;
      }
      __syncthreads();
      sums[2 * tid] = w_before[0];
      sums[2 * tid + 1] = w_before[1];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        unsigned lo = 0, hi = 2 * tid + i;  // first entry of the same bin
        if (bin[i] >= 0)
          while (lo < hi) {
            const unsigned mid = (lo + hi) / 2;
            if (bins.of(of_key((unsigned)(s.list[mid] >> 32))) > bin[i]) lo = mid + 1;
            else hi = mid;
          }
        first[i] = lo;
        of_bin[i] = bin[i] >= 0 ? sums[lo] : 0;
      }
      // what top-k leaves
      double target = INFINITY;
      if (by_p) {
        u64 mine = 0, in_bin;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (bin[i] >= 0 && bin[i] == bin_k && c_above[i] + (2 * tid + i - first[i]) < lim.k) mine += w[i];
        block_scan(mine, s.part, in_bin);
        target = lim.p * kReached * (above_k + (bin_k >= 0 ? (double)in_bin * exp(bins.middle(bin_k) - (double)top) : 0));
      }
      unsigned mine = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (bin[i] < 0) continue;
        const unsigned rank = c_above[i] + (2 * tid + i - first[i]);
        const double before = above[i] + (double)(w_before[i] - of_bin[i]) * exp(bins.middle(bin[i]) - (double)top);
        const unsigned key = (unsigned)(s.list[2 * tid + i] >> 32);
        if ((bin_k < 0 || rank < lim.k) && (!by_p || before < target) && key >= lim.least) ++mine;
      }
      u64 kept;
      block_scan((u64)mine, s.part, kept);
      if (kept) {
        const u64 e = s.list[kept - 1];
        last = (unsigned)(e >> 32);
        last_id = ~(unsigned)e;
      } else {
        last = (unsigned)(s.list[0] >> 32) + 1;
        last_id = 0x7fffffffu;
      }
      for (unsigned i = tid; i < kept; i += T) {
        const float v = of_key((unsigned)(s.list[i] >> 32));
        const int id = (int)~(unsigned)s.list[i];
        atomicAdd(&s.tile[id >> tile_log], weight(v));
        if (r.out) r.out[id] = v;
      }
      if (tid == 0) s.kept += (unsigned)kept;
      __syncthreads();
    } else {
      // top-k, then top-p, by readings
      const double above_p = by_p ? __builtin_bit_cast(double, s.mass[p_high]) : 0;
      const unsigned c_k = bin_k >= 0 ? s.cnt[bin_k] : 0;
      __syncthreads();
      unsigned ids = 0xffffffffu;  // how many tokens of key `last` are kept
      double left = above_k;
      if (bin_k >= 0) {
        narrow(s, r, in_k, false, (u64)(lim.k - c_k), 0.0, top, scale, last, ids);
        if (by_p) {
          // mass of what top-k keeps of its bin
          u64 mine = 0, in_bin;
          each(r, [&](int, const float(&y)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (y[i] >= kNone && in_k(y[i]) && key_of(y[i]) > last) mine += (u64)(bins.weight(y[i], bin_k) * scale + 0.5);
          });
          block_scan(mine, s.part, in_bin);
          const u64 each_w = (u64)(bins.weight(of_key(last), bin_k) * scale + 0.5);
          left += ((double)in_bin + (double)ids * (double)each_w) * exp(bins.middle(bin_k) - (double)top);
        }
      }
      if (by_p) {
        unsigned last_p, ids_p;
        // relative to the zone's largest token, found as the first in its order
        unsigned high, one;
        narrow(s, r, in_p, false, (u64)1, 0.0, top, scale, high, one);
        const float high_y = of_key(high);
        const double need = (lim.p * kReached * left - above_p) * exp((double)top - (double)high_y);
        if (need > 0) narrow(s, r, in_p, true, (u64)0, need, high_y, scale, last_p, ids_p);
        else { last_p = high; ids_p = 0; }
        if (last_p > last || (last_p == last && ids_p < ids)) {
          last = last_p;
          ids = ids_p;
        }
      }
      // the id of the last of them
      __syncthreads();
      unsigned* const per_tile = s.cnt;
      for (int i = tid; i < kTiles; i += T) per_tile[i] = 0;
      __syncthreads();
      each(r, [&](int v, const float(&y)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (y[i] >= kNone && key_of(y[i]) == last) atomicAdd(&per_tile[(v + i) >> tile_log], 1u);
      });
      __syncthreads();
      if (tid == 0) {
        s.found[0] = 0xffffffffu;
        unsigned before = 0;
        for (int i = 0; i < kTiles; ++i) {
          if (before < ids && before + per_tile[i] >= ids) { s.found[0] = i; s.found[1] = before; }
          before += per_tile[i];
        }
        s.found[2] = ids ? 0x7fffffffu : 0xffffffffu;
      }
      __syncthreads();
      const unsigned in_tile = s.found[0];
      if (in_tile != 0xffffffffu) {
        u64 before = s.found[1];
        __syncthreads();
        for (int v0 = (int)in_tile << tile_log; v0 < min(a.V, (int)(in_tile + 1) << tile_log); v0 += T) {
          const int v = v0 + tid;
          float y = -INFINITY;
          if (v < a.V) y = r.at(v);
          const u64 is = y >= kNone && key_of(y) == last;
          u64 all;
          const u64 to = before + block_scan(is, s.part, all);
          if (is && to == ids) s.found[2] = (unsigned)v;
          before += all;
        }
        __syncthreads();
      }
      last_id = s.found[2];
      // what the zone keeps
      const int lowest = by_p ? p_low : bin_k;
      each(r, [&](int v, const float(&y)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (y[i] >= kNone) {
            const unsigned k = key_of(y[i]);
            const int bin = bins.of(y[i]);
            if (bin <= sure && bin >= lowest && k >= lim.least && (k > last || (k == last && v + i <= (int)last_id))) {
              atomicAdd(&s.tile[(v + i) >> tile_log], weight(y[i]));
              atomicAdd(&s.kept, 1u);
              if (r.out) r.out[v + i] = y[i];
            }
          }
        }
      });
      __syncthreads();
    }
  }

  // 5. the token
  u64 mine = 0, total;
  if (tid < kTiles) mine = s.tile[tid];
  const u64 to = block_scan(mine, s.part, total);
  const float u = a.uniforms ? fminf(fmaxf(a.uniforms[row], 0.f), 1.f) : 0.f;
  const double target = (double)u * (double)total;
  if (tid == 0) s.found[0] = 0xffffffffu;
  __syncthreads();
  if (mine && (double)to >= target && (double)(to - mine) < target + (target == 0 && to == mine)) s.found[0] = tid, s.sum = to - mine;
  __syncthreads();
  if (tid == 0) {
    if (a.out_lse) a.out_lse[row] = (float)((double)top + log((double)total / scale));
    if (a.out_kept) a.out_kept[row] = (int)s.kept;
    s.found[1] = 0x7fffffffu;
  }
  if (!a.out_tokens && !a.out_conf) return;
  const int tile = (int)s.found[0];
  u64 before = s.sum;
  __syncthreads();
  const int end = min(a.V, (tile + 1) << tile_log);
  for (int v0 = tile << tile_log; v0 < end; v0 += kTile) {
    u64 w[4], sum = 0, all;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int v = v0 + 4 * tid + i;
      w[i] = 0;
      if (v < end) {
        const float y = r.at(v);
        const unsigned k = key_of(y);
        if (y >= kNone && k >= lim.least && (k > last || (k == last && v <= (int)last_id))) w[i] = weight(y);
      }
      sum += w[i];
    }
    u64 to_here = before + block_scan(sum, s.part, all) - sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      to_here += w[i];
      if (w[i] && (double)to_here >= target) atomicMin(&s.found[1], (unsigned)(v0 + 4 * tid + i));
    }
    before += all;
    __syncthreads();
    if (s.found[1] != 0x7fffffffu) break;
  }
  if (tid == 0) {
    const int v = (int)s.found[1];
    if (a.out_tokens) a.out_tokens[row] = v;
    if (a.out_conf) a.out_conf[row] = (float)((double)weight(r.at(v)) / (double)total);
  }
}

template <bool BF16>
__global__ __launch_bounds__(T) void draw_rows_kernel(DrawArgs a) {
  __shared__ Shared s;
  draw_row<BF16>(a, blockIdx.x, s);
}

}  // namespace

size_t draw_workspace(int, int) { return 256; }

hipError_t launch_draw(const DrawArgs& a) {
  const dim3 grid(a.B * a.K), threads(T);
  if (a.bf16) hipLaunchKernelGGL(draw_rows_kernel<true>, grid, threads, 0, a.stream, a);
  else hipLaunchKernelGGL(draw_rows_kernel<false>, grid, threads, 0, a.stream, a);
  return hipGetLastError();
}

}  // namespace fef
