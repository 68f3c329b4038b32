// Truncated laws and draws from them (fef_draw_logits): top-k, top-p and min-p over the logits of a row, the truncated logits, their
// log-sum-exp, and a token by inverse CDF.
//
// The order of a row's tokens is (key descending, id ascending), key being the logit's bits mapped to an unsigned number of the same order.
// Whatever the limits, what is kept is a beginning of that order: tokens with key > T, and those with key == T up to an id I.  (T, I) is
// found without sorting the row:
//   1. read the row: its maximum, and how many tokens and how much mass lie in each of 4096 bins of width 1/32, which reach from 80 below the
//      largest of a sample of the row to 48 above it.  Tokens below all bins are counted in the lowest one; they have no mass (exp(-64) of the
//      largest weight and less).
//   2. sums over the topmost bins (64 below the maximum, or 32): the bin where top-k ends, and the bins where top-p can end, given what top-k may
//      leave.  After a top-k of at most kFew top-p needs no bins: all that top-k leaves goes to the list.
//   3. read the row again: what lies above these bins is kept and written, what lies in them goes to a list, the rest is -inf.
//   4. the list is sorted; rank and mass before each of its tokens give (T, I); what it keeps is written.
//   5. the token: sums of the kept mass per tile of ids, then the ids of one tile.
//
// Masses decide which token is the last: a weight is computed in 64 bits and added as a whole number of 2^-s, s = min(50, 61 - the bits of V), which no
// order of the atomics changes.  In step 1 weights are relative to their bin's middle, |y - middle| <= 1/64, where a polynomial of degree 5
// is exact to 2^-45, so a bin's mass is off by 2^-(s + 1) of itself at the most, and by 2^-45: s = 44 up to V = 131071, 43 at 151936, 38 at 2^22, 31 at
// 2^29.  A border nearer to a mass than that is decided by rounding.
//
// Two ways through these steps.  draw_rows_kernel: a workgroup per row.  Slices of a row, a workgroup each, in three launches:
// draw_bins_kernel (step 1), draw_keep_kernel (steps 2 and 3: every workgroup adds up its row's bins) and draw_finish_kernel (a workgroup per
// row: steps 4 and 5).  What this does not serve (a list longer than kList: equal logits; limits that end below step 2's bins; a maximum far
// above the sample) is left to left_row, which narrows down the last key by readings of the row, 12 bits each: slow, some 270 to 310 us for 8 rows whose
// grammar leaves 5 tokens with negative logits (none in the sample: ref is 0), 510 to 600 where a bin's list is too long (gaussian logits of
// deviation 0.7, p = 0.8), up to 1900 where all logits are equal (V = 126464 and 151936; 28 to 63 us where the row is not left).
// Which way, with k = 100 and p = 0.95 / p = 0.95 alone, a workgroup per row against slices:
//   8 rows of V = 12000 23.0 / 20.6 against 27.9 / 26.4 us, 16384 24.9 / 27.2 against 28.0 / 29.5, 24000 29.0 / 33.5 against 28.1 / 31.1: one launch
//   below kShort tokens;
//   64 rows of V = 126464 78 / 133 against 42 / 58 us, 128 rows 87 / 145 against 58 / 80 (V = 32000: 36 / 45 against 34 / 39), with no more slices
//   than the 256 CUs take at once (64 rows in 8 slices each: 57 / 73).  From kManyRows on a slice would be a row.
//
// What bounds it.  Many rows: 512 rows of V = 151936 with k = 200, p = 0.95 163 us, 70 of them step 1 (4.4 TB/s; without limits 57: the rest are the
// LDS atomics), 50 step 3 (the stores, 6.2 TB/s; of its reading, groups of tokens that nothing is kept of are left out), the others the steps
// between, in which both workgroups of a CU compute; without limits 218 us, the exponentials of all tokens.  Few rows: the way through three
// launches, 30 us for 8 rows of V = 126464 with p = 0.95 (9.6 + 11.8 + 8.4), 42 us for 35 rows of V = 100003 with k = 1000, p = 0.98; one row of V = 5000:
// 16 us, a third each for steps 1 to 3, the list, the token.
#include <math.h>

#include <type_traits>

#include "head_common.hpp"
#include "wave_ops.hpp"

namespace fef {
namespace {

typedef unsigned long long u64;

constexpr int kBins = 4096, kList = 2048, kTiles = 512;
constexpr int kManyRows = 129, kShort = 24576;
constexpr unsigned kFew = 512;  // no masses in step 1: 512 rows of V = 151936 with k = 200, p = 0.95 186 -> 163 us; lists up to 512 need no sorting
constexpr int kGroupLog = 6, kGroups = 2816;  // positions of a row in groups of 64, of which step 3 reads those with a token that may be kept
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
  unsigned cnt[kBins];   // tokens per bin; after step 2: above the bin
  u64 mass[kBins];       // fixed point; after step 2: the mass above the bin, a double
  u64 list[kList];
  u64 tile[kTiles];
  u64 part[32];
  double power[64];      // 2^(j / 64)
  unsigned list_n, kept;
  unsigned found[4];
  double value[2];
  u64 sum;
  unsigned above_k;      // tokens above the bin where top-k ends
  u64 last_sum;
};

// t p + c, c uniform (in scalar registers: left to itself the compiler moves every constant to vector registers first)
__device__ __forceinline__ double horner(double t, double p, double c) {
  double r;
  asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(t), "v"(p), "s"(c));
  return r;
}
// exp(x) for x <= 1, to 2^-51 or so; each step one rounding, so that the same x gives the same bits wherever this is compiled into.  x = (64 i + j) ln 2 / 64 + q:
// 2^i, 2^(j / 64) from a table and a Taylor polynomial in q, the table-driven way that P. T. P. Tang published (ACM TOMS 15, 1989).
__device__ __forceinline__ double exp64(double x, const double* power) {
  x = fmax(x, -800.0);  // 0
  const double k = rint(x * 92.332482616893657);  // 64 / ln 2
  const double r = fma(k, -1.0830424696249145e-02, x), q = fma(k, -3.623510646634843e-19, r);  // ln 2 / 64 in two parts
  const int j = (int)k;
  const double p = horner(q, horner(q, horner(q, horner(q, horner(q, 1.0 / 120, 1.0 / 24), 1.0 / 6), 1.0 / 2), 1.0), 1.0);
  return ldexp(power[j & 63] * p, j >> 6);
}

// Inclusive sums over the lanes of a wavefront, of u64 or double (0 is all bits clear in both).
template <class D>
__device__ __forceinline__ D wave_scan64(D x) {
  auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
    const u64 b = __builtin_bit_cast(u64, x);
    const unsigned lo = (unsigned)dpp_mov<decltype(ctrl)::value, decltype(rows)::value>(0, (int)(unsigned)b);
    const unsigned hi = (unsigned)dpp_mov<decltype(ctrl)::value, decltype(rows)::value>(0, (int)(unsigned)(b >> 32));
    x += __builtin_bit_cast(D, (u64)hi << 32 | lo);
  };
  using All = std::integral_constant<int, 0xf>;
  step(std::integral_constant<int, kDppRowShr + 1>{}, All{});
  step(std::integral_constant<int, kDppRowShr + 2>{}, All{});
  step(std::integral_constant<int, kDppRowShr + 4>{}, All{});
  step(std::integral_constant<int, kDppRowShr + 8>{}, All{});
  step(std::integral_constant<int, kDppBcast15>{}, std::integral_constant<int, 0xa>{});
  step(std::integral_constant<int, kDppBcast31>{}, std::integral_constant<int, 0xc>{});
  return x;
}

// Maximum over a row of 16 lanes, in its last lane.
__device__ __forceinline__ float row_max(float x) {
  const int none = (int)0xff800000;
  auto step = [&](auto ctrl) __attribute__((always_inline)) {
    x = fmaxf(x, __builtin_bit_cast(float, dpp_mov<decltype(ctrl)::value, 0xf>(none, __builtin_bit_cast(int, x))));
  };
  step(std::integral_constant<int, kDppRowShr + 1>{});
  step(std::integral_constant<int, kDppRowShr + 2>{});
  step(std::integral_constant<int, kDppRowShr + 4>{});
  step(std::integral_constant<int, kDppRowShr + 8>{});
  return x;
}

// Sum over the workgroup of everything up to and with this thread, and the total; D is u64 or double.  Fixed order.
template <int T, class D>
__device__ __forceinline__ D block_scan(D x, D* part, D& total) {
  constexpr int W = T / kWave;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = wave_scan64(x);
  lds_barrier();
  if (lane == 63) part[wave] = x;
  lds_barrier();
  const D sums = wave_scan64(lane < W ? part[lane < W ? lane : 0] : D(0));
  auto of_lane = [&](int l) __attribute__((always_inline)) -> D {
    const u64 b = __builtin_bit_cast(u64, sums);
    const unsigned lo = __builtin_amdgcn_readlane((int)(unsigned)b, l), hi = __builtin_amdgcn_readlane((int)(unsigned)(b >> 32), l);
    return __builtin_bit_cast(D, (u64)hi << 32 | lo);
  };
  total = of_lane(W - 1);
  const int w = __builtin_amdgcn_readfirstlane(wave);
  return w ? of_lane(w - 1) + x : x;
}

// Both at once.
template <int T>
__device__ __forceinline__ void block_scan2(u64& c, double& w, u64* part, u64& all, double& total) {
  constexpr int W = T / kWave;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  c = wave_scan64(c);
  w = wave_scan64(w);
  lds_barrier();
  if (lane == 63) {
    part[wave] = c;
    part[W + wave] = __builtin_bit_cast(u64, w);
  }
  lds_barrier();
  const u64 c_sums = wave_scan64(lane < W ? part[lane < W ? lane : 0] : 0);
  const double w_sums = wave_scan64(lane < W ? __builtin_bit_cast(double, part[lane < W ? W + lane : W]) : 0.0);
  auto of_lane = [&](u64 b, int l) __attribute__((always_inline)) {
    return (u64)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(b >> 32), l) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)b, l);
  };
  const u64 w_bits = __builtin_bit_cast(u64, w_sums);
  all = of_lane(c_sums, W - 1);
  total = __builtin_bit_cast(double, of_lane(w_bits, W - 1));
  const int before = __builtin_amdgcn_readfirstlane(wave);
  if (before) {
    c += of_lane(c_sums, before - 1);
    w += __builtin_bit_cast(double, of_lane(w_bits, before - 1));
  }
}

template <bool BF16>
struct Row {
  const void* x;
  float* out;      // or NULL
  int V, head;     // vector j holds tokens 4 j - head .. ; a token's position is its id + head
  float inv_tau;
  bool out_wide;

  __device__ __forceinline__ float at(int v) const {
    const float f = BF16 ? (float)((const __bf16*)x)[v] : ((const float*)x)[v];
    return f * inv_tau + 0.f;  // -0 is 0
  }
  __device__ __forceinline__ int vectors() const { return (V + head + 3) >> 2; }
  __device__ __forceinline__ int position(int v) const { return v + head; }
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
  // STREAM: many rows, whose outputs only push the logits out of the caches (512 rows of V = 151936 245 -> 228 us when this came in)
  template <bool STREAM>
  __device__ __forceinline__ void store(int v, const float (&y)[4]) const {
    if (out_wide && v >= 0 && v + 4 <= V) {
      const floatx4 x{y[0], y[1], y[2], y[3]};
      if constexpr (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<floatx4*>(out + v));
      else *reinterpret_cast<floatx4*>(out + v) = x;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (v + i >= 0 && v + i < V) out[v + i] = y[i];
    }
  }
};

// Tokens of vectors [begin, end) of a row, four at a time: f(first id, y[4]); ids outside of the row come as -inf.  Wavefronts stay whole.
template <int T, int U, bool BF16, class F>
__device__ __forceinline__ void each(const Row<BF16>& r, int begin, int end, F f) {
  const int lane = threadIdx.x & 63;
  for (int j0 = begin + (int)threadIdx.x - lane; j0 < end; j0 += U * T) {
    float y[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + u * T < end) r.load(j0 + u * T + lane, y[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + u * T < end) f(4 * (j0 + u * T + lane) - r.head, y[u]);
  }
}
template <int T, bool BF16, class F>
__device__ __forceinline__ void each(const Row<BF16>& r, F f) { each<T, 4>(r, 0, r.vectors(), f); }

// Bins of width 1/32, the middle one from `ref` on, which is at most the row's maximum.  place(y), in 64 bits: the bin and how far y lies in it.
struct Bins {
  double ref;
  __device__ __forceinline__ double place(float y) const { return fma((double)y - ref, (double)kWidth, kBins / 2.0); }
  // whether a maximum lies in them, and 64 above the lowest one
  __device__ __forceinline__ bool serve(float top) const { return place(top) >= kBins / 2 && place(top) < kBins - 1; }
  // (the conversion saturates, and gives 0 for NaN; as assembly because the language leaves that open)
  __device__ __forceinline__ static int of_place(double u) {
    int b;
    asm("v_cvt_i32_f64 %0, %1" : "=v"(b) : "v"(u));
    return min(max(b, 0), kBins - 1);
  }
  __device__ __forceinline__ int of(float y) const { return of_place(place(y)); }
  __device__ __forceinline__ double begin(int b) const { return ref + (b - kBins / 2) * (1.0 / kWidth); }
  __device__ __forceinline__ double middle(int b) const { return ref + ((b - kBins / 2) + 0.5) * (1.0 / kWidth); }
  // exp(y - middle of its bin), bins above the lowest: the Taylor polynomial about the middle, in the fraction of u
  __device__ __forceinline__ static double weight(double u) {
    const double t = __builtin_amdgcn_fract(u);
    return horner(t, horner(t, horner(t, horner(t, horner(t, 0x1.1111111111111p-32, 0x1.5p-25), 0x1.500aaaaaaaaabp-18), 0x1.f80feaaaaaaabp-12),
                            0x1.f80feacp-6), 0x1.f80feabfeeeefp-1);
  }
  __device__ __forceinline__ double weight(float y) const { return weight(place(y)); }
};

// Weights in [0, 4) as whole numbers of 2^-f: adding 2^(52 - f) leaves them in the low bits.
struct Fixed {
  double magic, unit;
  __device__ __forceinline__ explicit Fixed(int V) {
    const int f = min(50, 61 - (32 - __clz(V)));
    magic = ldexp(1.0, 52 - f);
    unit = ldexp(1.0, -f);
  }
  __device__ __forceinline__ u64 of(double w) const {
    return __builtin_bit_cast(u64, w + magic) & ((1ull << 52) - 1);
  }
};

// In front of stores to places of the row that other wavefronts have written already: behind it their stores have landed.  (A barrier alone does
// not wait for stores, __syncthreads() neither.)  The comment in the assembly is what a check of the order goes by.
__device__ __forceinline__ void written_again() {
  wait_newer<0>();
  lds_barrier();
  asm volatile("; places of the row are written again" ::: "memory");
}

struct Limits {
  unsigned k;      // 0: none
  double p;        // >= 1: none
  unsigned least;  // smallest key that min-p keeps
  float min_p;     // 0: none
  bool law;
  bool few;        // top-p after a small top-k: the whole list of top-k is sorted, and no bin's mass is needed
};

struct Zone {
  int bin_k;          // bin where top-k ends, -1: it does not
  int p_low, p_high;  // bins where top-p can end
  int sure;           // bins above are kept whole
  int zone;           // there are tokens to be looked at one by one
  double above_k;     // mass above bin_k, or all of it
  __device__ __forceinline__ bool in_k(int bin) const { return bin == bin_k; }
  __device__ __forceinline__ bool in_p(int bin) const { return bin >= p_low && bin <= p_high; }
};

// Which of the tokens that `in` admits is the last one: the need_n-th in the order, or, where by_mass, the first at which their mass
// (relative to exp(top)) reaches need_m.  Readings of the row narrow its key down; `ids` is how many of that key belong to it.
template <int T, bool BF16, class In>
__device__ void narrow(Shared& s, const Row<BF16>& r, In in, bool by_mass, u64 need_n, double need_m, float top, const Fixed& fixed,
                       unsigned& last, unsigned& ids) {
  constexpr int kPer = kBins / T;
  unsigned low = 0, bits = 32;
  while (bits) {
    const unsigned shift = bits > 12 ? bits - 12 : 0;
    lds_barrier();
    for (int b = threadIdx.x; b < kBins; b += T) {
      s.cnt[b] = 0;
      s.mass[b] = 0;
    }
    lds_barrier();
    each<T>(r, [&](int, const float(&y)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned k = key_of(y[i]);
        if (y[i] >= kNone && in(y[i]) && (bits == 32 || (k - low) >> bits == 0)) {
          const unsigned b = (k - low) >> shift;
          atomicAdd(&s.cnt[b], 1u);
          if (by_mass) atomicAdd(&s.mass[b], fixed.of(exp64((double)y[i] - (double)top, s.power)));
        }
      }
    });
    lds_barrier();
    // from the top: thread t has bins kBins - 1 - kPer t and the next below
    u64 c = 0, all;
    u64 m = 0, all_m;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int b = kBins - 1 - kPer * (int)threadIdx.x - i;
      c += s.cnt[b];
      m += s.mass[b];
    }
    u64 c_at = block_scan<T>(c, s.part, all) - c, m_at = block_scan<T>(m, s.part, all_m) - m;
    if (threadIdx.x == 0) s.found[0] = 0;
    lds_barrier();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int b = kBins - 1 - kPer * (int)threadIdx.x - i;
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
    lds_barrier();
    if (by_mass) need_m -= (double)s.sum;
    else need_n -= s.sum;
    low += s.found[0] << shift;
    bits = shift;
  }
  last = low;
  const unsigned ties = s.found[1];
  if (by_mass) {
    const double w = (double)fixed.of(exp64((double)of_key(low) - (double)top, s.power));
    const double n = w > 0 ? ceil(need_m / w) : 1.0;
    ids = n < 1 ? 1 : n > ties ? ties : (unsigned)n;
  } else {
    ids = (unsigned)need_n;
  }
  lds_barrier();
}

// What a row asks for.
template <bool BF16>
__device__ __forceinline__ void set_up(const DrawArgs& a, int row, Row<BF16>& r, Limits& lim) {
  const int b = row / a.K, m = row - b * a.K;
  r.V = a.V;
  const long at = (long)b * a.seq_stride + (long)m * a.slot_stride;
  r.x = BF16 ? (const void*)((const __bf16*)a.logits + at) : (const void*)((const float*)a.logits + at);
  r.head = (int)(((uintptr_t)r.x / (BF16 ? 2 : 4)) & 3);
  r.out = a.out ? a.out + (long)b * a.out_seq_stride + (long)m * a.out_slot_stride : nullptr;
  r.out_wide = (((uintptr_t)r.out - 4 * (uintptr_t)r.head) & 15) == 0;
  lim.k = a.top_k && a.top_k[b] > 0 ? (unsigned)a.top_k[b] : 0;
  lim.p = a.top_p && a.top_p[b] < 1.f ? (double)a.top_p[b] : 2.0;
  lim.min_p = a.min_p && a.min_p[b] > 0.f ? a.min_p[b] : 0.f;
  lim.least = 0;
  lim.law = true;
  r.inv_tau = a.inv_tau;
  if (a.temperatures) {
    const float t = a.temperatures[b];
    lim.law = t >= 0.f;
    r.inv_tau = 1.f / t;
    if (!(r.inv_tau < INFINITY)) {
      r.inv_tau = 1.f;
      lim.k = 1;
    }
  }
  if (lim.p <= 0 || lim.min_p > 1.f) lim.k = 1;
  if (lim.k == 1) lim.p = 2.0;
  lim.few = lim.p < 1 && lim.k > 0 && lim.k <= kFew;
}
__device__ __forceinline__ bool by_k(const Limits& l) { return l.k > 0; }
__device__ __forceinline__ bool by_p(const Limits& l) { return l.p < 1; }
__device__ __forceinline__ bool by_mass(const Limits& l) { return by_p(l) && !l.few; }

__device__ __forceinline__ void set_powers(Shared& s) {
  if (threadIdx.x < 64) s.power[threadIdx.x] = exp2(threadIdx.x * (1.0 / 64));
}

// Step 1 over vectors [begin, end): s.cnt, s.mass (zero before), in each thread its largest y, NaN if there is one, and the largest of each group of
// 64 positions.
template <int T, bool GROUPS = false, bool BF16>
__device__ __forceinline__ void count(Shared& s, const Row<BF16>& r, int begin, int end, const Limits& lim, const Bins& bins, const Fixed& fixed,
                                      float& high, float* groups = nullptr) {
  unsigned low = 0;
  auto run = [&](auto k_tag, auto p_tag) __attribute__((always_inline)) {
    each<T, GROUPS ? 4 : 8>(r, begin, end, [&](int v, const float(&y)[4]) __attribute__((always_inline)) {
      const float four = __builtin_elementwise_maximum(__builtin_elementwise_maximum(y[0], y[1]), __builtin_elementwise_maximum(y[2], y[3]));
      high = __builtin_elementwise_maximum(high, four);
      if constexpr (GROUPS) {
        const float of_row = row_max(four);
        const int group = r.position(v) >> kGroupLog;
        if ((threadIdx.x & 15) == 15 && group < kGroups) groups[group] = of_row;
      }
      if constexpr (decltype(k_tag)::value || decltype(p_tag)::value) {
        double u[4];
        int bin[4];
        u64 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = bins.place(y[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) bin[i] = Bins::of_place(u[i]);
        if constexpr (decltype(p_tag)::value)
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = fixed.of(Bins::weight(u[i]));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (bin[i] > 0) {
            if constexpr (decltype(k_tag)::value) atomicAdd(&s.cnt[bin[i]], 1u);
            if constexpr (decltype(p_tag)::value) atomicAdd(&s.mass[bin[i]], w[i]);
          } else if constexpr (decltype(k_tag)::value) {
            low += y[i] >= kNone;
          }
        }
      }
    });
  };
  using Yes = std::true_type;
  using No = std::false_type;
  if (by_k(lim) && by_mass(lim)) run(Yes{}, Yes{});
  else if (by_k(lim)) run(Yes{}, No{});
  else if (by_mass(lim)) run(No{}, Yes{});
  else run(No{}, No{});
  if (low) atomicAdd(&s.cnt[0], low);
}

// min-p as a key: the smallest y with exp(y - top) >= min_p.
__device__ __forceinline__ void set_least(Limits& lim, float top) {
  if (!(lim.min_p > 0.f && lim.min_p <= 1.f)) return;
  const auto keeps = [&](unsigned k) { return exp((double)of_key(k) - (double)top) >= (double)lim.min_p; };
  const double near = (double)top + log((double)lim.min_p);
  const unsigned guess = key_of((float)near);
  unsigned low = guess - 2, k = min(guess + 2, key_of(top));
  if (!keeps(k) || keeps(low)) {  // sums near 0 may be further off; and numbers may be so far apart that one step misses the border
    low = key_of((float)(near - 0.01));
    k = key_of(fminf((float)(near + 0.01), top));
    if (!keeps(k)) ++k;
    if (keeps(low)) k = low;
  }
  while (k - low > 1 && k != low) {
    const unsigned mid = low + (k - low) / 2;
    if (keeps(mid)) k = mid;
    else low = mid;
  }
  lim.least = k;
}

// Step 2 over the PER T bins from b0 down: s.cnt and s.mass become what lies above each of them.  all, total: tokens and mass of the row, or
// (BELOW) of its bins further down; FULL: there are none.  False: the limits end below these bins.
template <int T, int PER, bool FULL, bool BELOW>
__device__ __forceinline__ bool find_zone(Shared& s, const Limits& lim, const Bins& bins, float top, int b0, u64 all, double total, Zone& z) {
  z = Zone{-1, kBins, -1, -1, 0, 0};
  const int tid = threadIdx.x;
  if (!by_k(lim) && !by_mass(lim)) return true;
  unsigned c = 0, ci[PER];
  double w = 0, wi[PER];
  u64 mi[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int bin = b0 - PER * tid - i;
    ci[i] = by_k(lim) && bin >= 0 ? s.cnt[bin] : 0;
    mi[i] = by_mass(lim) && bin > 0 ? s.mass[bin] : 0;
    c += ci[i];
  }
  u64 any = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    any |= mi[i];
    wi[i] = 0;
  }
  if (__ballot(any != 0)) {
    constexpr double kDown[8] = {1.0, 0x1.f03f56a88b5d8p-1, 0x1.e0fabfbc702a4p-1, 0x1.d22e6a0197c03p-1, 0x1.c3d6a24ed8222p-1, 0x1.b5efd29f24c26p-1, 0x1.a876812c0877cp-1, 0x1.9b674f8f2f3d8p-1};  // exp(-i / 32)
    static_assert(PER <= 8, "");
    const double first = exp64(bins.middle(b0 - PER * tid) - (double)top, s.power);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      wi[i] = (double)mi[i] * (first * kDown[i]);  // of 2^-f
      w += wi[i];
    }
  }
  u64 c_here = 0, c_at = 0;
  double w_here = 0, w_at = 0;
  if (by_k(lim) && by_mass(lim)) {
    c_at = c;
    w_at = w;
    block_scan2<T>(c_at, w_at, s.part, c_here, w_here);
    c_at -= c;
    w_at -= w;
  } else if (by_k(lim)) {
    c_at = block_scan<T>((u64)c, s.part, c_here) - c;
  } else {
    w_at = block_scan<T>(w, (double*)s.part, w_here) - w;
  }
  if (FULL || BELOW) {
    all += c_here;
    total += w_here;
  }
  if (tid == 0) s.found[0] = s.found[1] = s.found[2] = 0xffffffffu;
  lds_barrier();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int bin = b0 - PER * tid - i;
    if (by_k(lim) && c_at < lim.k && c_at + ci[i] >= lim.k && lim.k < all) {
      s.found[0] = bin;
      s.value[0] = w_at;
      s.value[1] = w_at + wi[i];
    }
    if (bin >= 0) {
      s.cnt[bin] = (unsigned)c_at;
      s.mass[bin] = __builtin_bit_cast(u64, w_at);
    }
    c_at += ci[i];
    w_at += wi[i];
  }
  lds_barrier();
  const bool ends = s.found[0] != 0xffffffffu;
  bool here = ends || !by_k(lim) || lim.k >= all;
  z.bin_k = ends ? (int)s.found[0] : -1;
  z.above_k = ends ? s.value[0] : total;
  if (by_mass(lim)) {
    // with the mass top-k leaves somewhere in [lowest, highest], and a little room for the sums' rounding
    const double lowest = lim.p * z.above_k * (1 - 1e-12), highest = lim.p * (ends ? s.value[1] : total) * (1 + 1e-12);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int bin = b0 - PER * tid - i;
      if (!(wi[i] > 0)) continue;
      const double before = __builtin_bit_cast(double, s.mass[bin]);
      if ((before < lowest || before == 0) && before + wi[i] >= lowest) atomicMin(&s.found[1], (unsigned)(kBins - 1 - bin));  // may be the first to reach it
      if (before < highest && before + wi[i] >= highest) atomicMin(&s.found[2], (unsigned)bin);                               // the last that may be needed
    }
    lds_barrier();
    here = here && (FULL || (s.found[1] != 0xffffffffu && s.found[2] != 0xffffffffu));
    z.p_high = s.found[1] == 0xffffffffu ? kBins - 1 : kBins - 1 - (int)s.found[1];
    z.p_low = s.found[2] == 0xffffffffu ? 0 : (int)s.found[2];
    if (ends && z.p_low < z.bin_k) z.p_low = z.bin_k;
    if (ends && z.p_high < z.bin_k) z.p_high = z.bin_k;
  }
  z.sure = lim.few ? kBins : by_mass(lim) ? z.p_high : z.bin_k;
  z.zone = by_p(lim) || z.bin_k >= 0;
  if (tid == 0 && z.bin_k >= 0) s.above_k = s.cnt[z.bin_k];
  return here;
}

// Step 3 over vectors [begin, end): out, s.tile, s.list, s.list_n (which counts on where the list is full).  Returns the tokens kept (of this
// thread).
template <int T, bool NEAR, bool GROUPS = false, bool BF16>
__device__ __forceinline__ unsigned keep(Shared& s, const Row<BF16>& r, int begin, int end, const Limits& lim, const Bins& bins, const Fixed& fixed,
                                         const Zone& z, float top, int tile_log, const float* groups = nullptr) {
  // y from `sure` on is kept, y below `maybe` is not; in between the bins say (and a little beside the zone, whose borders are numbers of 64 bits)
  const float least = fmaxf(kNone, lim.least ? of_key(lim.least) : kNone);
  const int low_bin = by_mass(lim) ? (z.bin_k >= 0 ? min(z.bin_k, z.p_low) : z.p_low) : z.bin_k;
  const double up = z.zone ? bins.begin(z.sure + 1) : 0, down = z.zone ? bins.begin(low_bin) : 0;
  const float sure = z.zone ? (z.sure < kBins - 1 ? fmaxf((float)(up + (1e-6 + 1e-6 * fabs(up))), least) : INFINITY) : least;
  const float maybe = z.zone ? (low_bin > 0 ? (float)(down - (1e-6 + 1e-6 * fabs(down))) : kNone) : INFINITY;
  const float least_wanted = fminf(sure, maybe);
  unsigned kept = 0;
  auto one = [&](int v, const float(&y)[4], u64& sum) __attribute__((always_inline)) {
    float o[4];
    unsigned mine = 0;
    bool listed = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool keep = y[i] >= sure;
      o[i] = keep ? y[i] : -INFINITY;
      mine |= (unsigned)keep << i;
      listed |= y[i] >= maybe && !keep;
    }
    if (listed) {
      bool is[4];
      unsigned n = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int bin = bins.of(y[i]);
        const bool token = y[i] >= maybe && y[i] >= kNone && !(y[i] >= sure);
        is[i] = token && (lim.few ? bin >= z.bin_k : z.in_k(bin) || (by_mass(lim) && z.in_p(bin)));
        n += is[i];
        if (token && bin > z.sure && y[i] >= least) {
          o[i] = y[i];
          mine |= 1u << i;
        }
      }
      if (n) {
        unsigned p = atomicAdd(&s.list_n, n);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (is[i]) {
            if (p < kList) s.list[p] = ((u64)key_of(y[i]) << 32) | (unsigned)~(v + i);
            ++p;
          }
      }
    }
    if (r.out) r.template store<GROUPS>(v, o);
    kept += __popc(mine);
    if (__ballot(mine == 15)) {  // much is kept: four at a time
      u64 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = fixed.of(exp64((double)y[i] - (double)top, s.power));
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += mine >> i & 1 ? w[i] : 0;
      mine = 0;
    }
    for (; mine; mine &= mine - 1) {  // few lanes have more than one
      const float x = mine & 1 ? y[0] : mine & 2 ? y[1] : mine & 4 ? y[2] : y[3];
      sum += fixed.of(exp64((double)x - (double)top, s.power));
    }
  };
  // NEAR: a wavefront takes 1024 neighbouring positions at a time, which lie in one tile; else, for short rows, 256, so that all have work.
  constexpr int U = 4, kApart = NEAR ? 64 : T;
  const int lane = threadIdx.x & 63;
  for (int j0 = begin + (NEAR ? U : 1) * ((int)threadIdx.x - lane); j0 < end; j0 += U * T) {
    float y[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + kApart * u + lane;
      bool wanted = j0 + kApart * u < end;
      if constexpr (GROUPS) wanted = wanted && ((4 * j) >> kGroupLog >= kGroups || groups[(4 * j) >> kGroupLog] >= least_wanted);
      if (wanted) r.load(j, y[u]);
      else y[u][0] = y[u][1] = y[u][2] = y[u][3] = -INFINITY;
    }
    u64 sum = 0;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + kApart * u < end) {
        one(4 * (j0 + kApart * u + lane) - r.head, y[u], sum);
        if constexpr (!NEAR) {
          if (sum) atomicAdd(&s.tile[(4 * (j0 + kApart * u + lane)) >> tile_log], sum);
          sum = 0;
        }
      }
    if (NEAR && __ballot(sum != 0)) {
      sum = wave_scan64(sum);
      if (lane == 63) atomicAdd(&s.tile[(4 * j0) >> tile_log], sum);
    }
  }
  return kept;
}

// Step 4: the last token kept, from n <= kList entries of s.list.  Adds what the list keeps to s.tile and s.kept, and writes it.
template <int T, bool BF16>
__device__ __forceinline__ void resolve(Shared& s, const Row<BF16>& r, const Limits& lim, const Bins& bins, const Fixed& fixed, const Zone& z,
                                        float top, int tile_log, unsigned n, unsigned& last, int& last_id) {
  const int tid = threadIdx.x;
  if (n <= T) {  // an entry's place is how many are larger (no two are equal): `parts` threads of different wavefronts count for each (some 60 entries: 2.3 us less than sorting them)
    unsigned size = 64;
    while (size < n) size <<= 1;
    const unsigned parts = T / size, part = tid / size, e = tid & (size - 1);
    const unsigned each = ((n + parts - 1) / parts + 7) & ~7u;  // entries that a part looks at, in eights: zeros behind the last
    static_assert(kList >= 2 * T, "");
    unsigned* const place = reinterpret_cast<unsigned*>(s.cnt);
    if (tid < (int)size) place[tid] = 0;
    const u64 mine = e < n ? s.list[e] : 0;
    for (unsigned j = n + tid; j < parts * each; j += T) s.list[j] = 0;
    lds_barrier();
    unsigned larger = 0;
    for (unsigned j = part * each; j < (part + 1) * each; j += 8) {
      u64 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s.list[j + i];
#pragma unroll
      for (int i = 0; i < 8; ++i) larger += x[i] > mine;
    }
    if (e < n && larger) atomicAdd(&place[e], larger);
    lds_barrier();
    if (part == 0 && e < n) s.list[place[e]] = mine;
    lds_barrier();
  } else {
    unsigned size = T;
    while (size < n) size <<= 1;
    for (unsigned i = n + tid; i < size; i += T) s.list[i] = 0;
    lds_barrier();
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
        lds_barrier();
      }
  }
  auto y_of = [&](unsigned i) __attribute__((always_inline)) { return of_key((unsigned)(s.list[i] >> 32)); };
  // sums[i]: weights of the entries in front of entry i, each relative to its own bin's middle (few: to the maximum); thread t has `per` neighbours
  u64* const sums = reinterpret_cast<u64*>(s.cnt);
  static_assert(sizeof s.cnt >= kList * sizeof(u64), "");
  const unsigned per = (n + T - 1) / T, i0 = min(n, tid * per), i1 = min(n, i0 + per);
  const Fixed fine(kList);  // fewer weights than a row has, in smaller units
  auto weight_of = [&](unsigned i) __attribute__((always_inline)) {
    return lim.few ? fine.of(exp64((double)y_of(i) - (double)top, s.power)) : fixed.of(bins.weight(y_of(i)));
  };
  if (by_p(lim)) {
    u64 mine = 0, all;
    for (unsigned i = i0; i < i1; ++i) {
      mine += weight_of(i);
    }
    u64 before = block_scan<T>(mine, s.part, all) - mine;
    for (unsigned i = i0; i < i1; ++i) {
      sums[i] = before;
      before += weight_of(i);
    }
    if (tid == 0) s.last_sum = all;
    lds_barrier();
  }
  // first entry of a bin or a lower one
  auto begin_of = [&](int bin) __attribute__((always_inline)) {
    unsigned lo = 0, hi = n;
    while (lo < hi) {
      const unsigned mid = (lo + hi) / 2;
      if (bins.of(y_of(mid)) > bin) lo = mid + 1;
      else hi = mid;
    }
    return lo;
  };
  double target = INFINITY;
  unsigned k_first = 0, k_end = n;  // entries of bin_k that top-k leaves end at k_end
  if (lim.few) {
    k_end = min(n, lim.k);
    target = lim.p * kReached * (double)(k_end < n ? sums[k_end] : s.last_sum);
  } else if (z.bin_k >= 0) {
    k_first = begin_of(z.bin_k);
    k_end = min(n, k_first + (lim.k - s.above_k));
  }
  if (by_mass(lim)) {
    double left = z.above_k;
    if (z.bin_k >= 0) left += (double)((k_end < n ? sums[k_end] : s.last_sum) - sums[k_first]) * exp64(bins.middle(z.bin_k) - (double)top, s.power);
    target = lim.p * kReached * left;
  }
  unsigned mine = 0;
  for (unsigned i = i0; i < min(i1, k_end); ++i) {
    const float y = y_of(i);
    bool is = key_of(y) >= lim.least;
    if (lim.few) {
      is = is && (double)sums[i] < target;
    } else if (by_p(lim)) {
      const int bin = bins.of(y);
      is = is && __builtin_bit_cast(double, s.mass[bin]) + (double)(sums[i] - sums[begin_of(bin)]) * exp64(bins.middle(bin) - (double)top, s.power) < target;
    }
    mine += is;
  }
  u64 kept;
  block_scan<T>((u64)mine, s.part, kept);
  last_id = 0x7fffffff;
  if (kept) {
    const u64 e = s.list[kept - 1];
    last = (unsigned)(e >> 32);
    last_id = (int)~(unsigned)e;
  } else {
    last = (unsigned)(s.list[0] >> 32) + 1;  // (a zone has tokens)
  }
  written_again();  // -inf of step 3
  for (unsigned i = tid; i < kept; i += T) {
    const float y = y_of(i);
    const int id = (int)~(unsigned)s.list[i];
    const u64 e = fixed.of(exp64((double)y - (double)top, s.power));
    if (e) atomicAdd(&s.tile[r.position(id) >> tile_log], e);
    if (r.out) r.out[id] = y;
  }
  if (tid == 0) s.kept += (unsigned)kept;
  lds_barrier();
}

// Step 4 by readings of the row, from step 2 over all bins.
template <int T, bool BF16>
__device__ __forceinline__ void resolve_by_reading(Shared& s, const Row<BF16>& r, const Limits& lim, const Bins& bins, const Fixed& fixed, const Zone& z, float top,
                                   int tile_log, unsigned& last, int& last_id) {
  const int tid = threadIdx.x;
  const double above_p = by_p(lim) ? __builtin_bit_cast(double, s.mass[z.p_high]) : 0;
  const unsigned c_k = z.bin_k >= 0 ? s.cnt[z.bin_k] : 0;
  lds_barrier();
  unsigned ids = 0xffffffffu;  // how many tokens of key `last` are kept
  double left = z.above_k;
  last = 0;
  auto in_k = [&](float y) { return z.in_k(bins.of(y)); };
  auto in_p = [&](float y) { return z.in_p(bins.of(y)); };
  if (z.bin_k >= 0) {
    narrow<T>(s, r, in_k, false, (u64)(lim.k - c_k), 0.0, top, fixed, last, ids);
    if (by_p(lim) && z.bin_k > 0) {
      // mass of what top-k keeps of its bin
      u64 mine = 0, in_bin;
      each<T>(r, [&](int, const float(&y)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (y[i] >= kNone && in_k(y[i]) && key_of(y[i]) > last) mine += fixed.of(bins.weight(y[i]));
      });
      block_scan<T>(mine, s.part, in_bin);
      const u64 each_w = fixed.of(bins.weight(of_key(last)));
      left += ((double)in_bin + (double)ids * (double)each_w) * exp64(bins.middle(z.bin_k) - (double)top, s.power);
    }
  }
  if (by_p(lim)) {
    unsigned last_p, ids_p, high, one;
    // relative to the zone's largest token, found as the first in its order
    narrow<T>(s, r, in_p, false, (u64)1, 0.0, top, fixed, high, one);
    const float high_y = of_key(high);
    const double need = (lim.p * kReached * left - above_p) / exp64((double)high_y - (double)top, s.power);
    last_p = high;
    ids_p = 0;
    if (need > 0) narrow<T>(s, r, in_p, true, (u64)0, need, high_y, fixed, last_p, ids_p);
    if (last_p > last || (last_p == last && ids_p < ids)) {
      last = last_p;
      ids = ids_p;
    }
  }
  // the id of the last of them
  lds_barrier();
  unsigned* const per_tile = s.cnt;
  for (int i = tid; i < kTiles; i += T) per_tile[i] = 0;
  lds_barrier();
  each<T>(r, [&](int v, const float(&y)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (y[i] >= kNone && key_of(y[i]) == last) atomicAdd(&per_tile[r.position(v + i) >> tile_log], 1u);
  });
  lds_barrier();
  if (tid == 0) {
    s.found[0] = 0xffffffffu;
    unsigned before = 0;
    for (int i = 0; i < kTiles; ++i) {
      if (before < ids && before + per_tile[i] >= ids) { s.found[0] = i; s.found[1] = before; }
      before += per_tile[i];
    }
    s.found[2] = ids ? 0x7fffffffu : 0xffffffffu;
  }
  lds_barrier();
  const unsigned in_tile = s.found[0];
  if (in_tile != 0xffffffffu) {
    u64 before = s.found[1];
    lds_barrier();
    const int end = min(r.position(r.V), (int)(in_tile + 1) << tile_log);
    for (int p0 = (int)in_tile << tile_log; p0 < end; p0 += T) {
      const int v = p0 + tid - r.head;
      float y = -INFINITY;
      if (v >= 0 && p0 + tid < end) y = r.at(v);
      const u64 is = y >= kNone && key_of(y) == last;
      u64 all;
      const u64 to = before + block_scan<T>(is, s.part, all);
      if (is && to == ids) s.found[2] = (unsigned)v;
      before += all;
    }
    lds_barrier();
  }
  last_id = (int)s.found[2];
  written_again();
  // what the zone keeps
  const int lowest = by_p(lim) ? z.p_low : z.bin_k;
  unsigned kept = 0;
  each<T>(r, [&](int v, const float(&y)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (y[i] >= kNone) {
        const unsigned k = key_of(y[i]);
        const int bin = bins.of(y[i]);
        if (bin <= z.sure && bin >= lowest && k >= lim.least && (k > last || (k == last && v + i <= last_id))) {
          const u64 e = fixed.of(exp64((double)y[i] - (double)top, s.power));
          if (e) atomicAdd(&s.tile[r.position(v + i) >> tile_log], e);
          ++kept;
          if (r.out) r.out[v + i] = y[i];
        }
      }
    }
  });
  if (kept) atomicAdd(&s.kept, kept);
  lds_barrier();
}

__device__ __forceinline__ void no_token(const DrawArgs& a, int row) {
  if (threadIdx.x == 0) {
    if (a.out_tokens) a.out_tokens[row] = -1;
    if (a.out_conf) a.out_conf[row] = 0.f;
    if (a.out_kept) a.out_kept[row] = 0;
    if (a.out_lse) a.out_lse[row] = -INFINITY;
  }
}
// Step 5, from s.tile and s.kept.
template <int T, bool BF16>
__device__ __forceinline__ void token(Shared& s, const DrawArgs& a, int row, const Row<BF16>& r, const Limits& lim, const Fixed& fixed, float top,
                                      int tile_log, unsigned last, int last_id) {
  constexpr int kPer = (kTiles + T - 1) / T;  // neighbouring tiles per thread
  const int tid = threadIdx.x;
  u64 mine = 0, total;
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (kPer * tid + i < kTiles) mine += s.tile[kPer * tid + i];
  u64 to = block_scan<T>(mine, s.part, total) - mine;
  if (!total) {  // (the row's maximum has the largest weight there is)
    no_token(a, row);
    return;
  }
  const float u = a.uniforms ? fminf(fmaxf(a.uniforms[row], 0.f), 1.f) : 0.f;
  const double target = (double)u * (double)total;
  // the first tile at whose end the mass reaches the target
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const u64 t = kPer * tid + i < kTiles ? s.tile[kPer * tid + i] : 0;
    if (t && (double)(to + t) >= target && ((double)to < target || to == 0)) {
      s.found[0] = kPer * tid + i;
      s.sum = to;
    }
    to += t;
  }
  if (tid == 0) {
    s.found[1] = 0x7fffffffu;
    if (a.out_kept) a.out_kept[row] = (int)s.kept;
  }
  lds_barrier();
  const int tile = (int)s.found[0];
  u64 before = s.sum;
  const int end = min(r.position(r.V), (tile + 1) << tile_log);
  const float y_last = of_key(last);
  const float least = fmaxf(kNone, lim.least ? of_key(lim.least) : kNone);
  for (int p0 = tile << tile_log; p0 < end; p0 += 4 * T) {
    u64 w[4], sum = 0, all;
    float y[4];
    const int v = p0 + 4 * tid - r.head;
    r.load((p0 >> 2) + tid, y);
    // by a wavefront that has none of the tile's first tokens, while the others wait for theirs
    if (p0 == tile << tile_log && tid == T - 1 && a.out_lse) a.out_lse[row] = (float)((double)top + log((double)total * fixed.unit));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = 0;
      if (y[i] >= least && r.position(v + i) < end && (last == 0 || key_of(y[i]) > last || (y[i] == y_last && v + i <= last_id)))
        w[i] = fixed.of(exp64((double)y[i] - (double)top, s.power));
      sum += w[i];
    }
    u64 to_here = before + block_scan<T>(sum, s.part, all) - sum;
    // the first token at which the mass reaches the target: what lies in front of it does not
    bool mine = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool is = w[i] && (double)(to_here + w[i]) >= target && ((double)to_here < target || to_here == 0);
      if (is) {
        if (a.out_tokens) a.out_tokens[row] = v + i;
        if (a.out_conf) a.out_conf[row] = (float)((double)w[i] / (double)total);
      }
      mine |= is;
      to_here += w[i];
    }
    if (mine) s.found[1] = 0;
    before += all;
    if (p0 + 4 * T >= end) break;
    lds_barrier();
    if (s.found[1] == 0) break;
  }
}

template <int T, bool BF16>
__device__ __forceinline__ void no_logits(const Row<BF16>& r, int begin, int end) {
  if (!r.out) return;
  const float none[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  for (int j = begin + (int)threadIdx.x; j < end; j += T) r.template store<false>(4 * j - r.head, none);
}

// The largest y of the workgroup, through s.found[0]; s.found[1]: whether there is a NaN or +inf.  Both 0 before.
__device__ __forceinline__ float top_of(Shared& s, float high) {
  if (!(high < INFINITY)) s.found[1] = 1;
#pragma unroll
  for (int d = 32; d; d >>= 1) high = fmaxf(high, __shfl_xor(high, d));
  if ((threadIdx.x & 63) == 0) atomicMax(&s.found[0], key_of(high));
  lds_barrier();
  return of_key(s.found[0]);
}

// Bins of a row by the largest of a sample, a vector per thread in T / 64 places; through s.found[2], which is 0 before.
template <int T, bool BF16>
__device__ __forceinline__ Bins bins_of(Shared& s, const Row<BF16>& r) {
  const int n = r.vectors(), wave = threadIdx.x >> 6;
  float y[4], high = -INFINITY;
  r.load((int)((long)n * wave / (T / 64)) + (int)(threadIdx.x & 63), y);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (y[i] < INFINITY) high = fmaxf(high, y[i]);
#pragma unroll
  for (int d = 32; d; d >>= 1) high = fmaxf(high, __shfl_xor(high, d));
  if ((threadIdx.x & 63) == 0) atomicMax(&s.found[2], key_of(high));
  lds_barrier();
  const float top = of_key(s.found[2]);
  return Bins{top >= kNone ? (double)top - 16.0 : 0.0};
}

template <int T>
__device__ __forceinline__ void clear(Shared& s) {
  uint4* const c = reinterpret_cast<uint4*>(s.cnt);
  uint4* const m = reinterpret_cast<uint4*>(s.mass);
  const uint4 zero{0, 0, 0, 0};
  for (int i = threadIdx.x; i < kBins / 4; i += T) c[i] = zero;
  for (int i = threadIdx.x; i < kBins / 2; i += T) m[i] = zero;
  for (int i = threadIdx.x; i < kTiles; i += T) s.tile[i] = 0;
  if (threadIdx.x == 0) s.found[0] = s.found[1] = s.found[2] = s.found[3] = s.list_n = s.kept = 0;
}

// Tokens and mass (relative to y) of the bins below `end`.
template <int T>
__device__ __forceinline__ void totals(Shared& s, const Limits& lim, const Bins& bins, double y, int end, u64& all, double& total) {
  constexpr int U = 4;
  unsigned c = 0;
  double w = 0;
  for (int b = threadIdx.x; b < end; b += U * T) {
    unsigned ci[U];
    u64 wi[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      ci[u] = by_k(lim) && b + u * T < end ? s.cnt[b + u * T] : 0;
      wi[u] = by_mass(lim) && b + u * T < end ? s.mass[b + u * T] : 0;
    }
    u64 any = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      c += ci[u];
      any |= wi[u];
    }
    if (__ballot(any != 0)) {
      constexpr double kUp[7] = {1.0, 0x1.0f2ebd0a80020p+23, 0x1.1f43fcc4b662cp+46, 0x1.304d6aeca254bp+69, 0x1.425982cf597cdp+92, 0x1.55779b984f3ebp+115, 0x1.69b7f55b808bap+138};  // exp(16 u)
      constexpr int kStep = T / (16 * 32);
      static_assert(T % (16 * 32) == 0 && (U - 1) * kStep < 7, "");
      const double first = exp64(bins.middle(b) - y, s.power);
#pragma unroll
      for (int u = 0; u < U; ++u) w += (double)wi[u] * (first * kUp[u * kStep]);
    }
  }
  all = 0;
  total = 0;
  u64 tokens = c;
  block_scan2<T>(tokens, w, s.part, all, total);
}

__host__ __device__ inline int tile_log_of(int V) {  // tiles of 2^this positions: at least 1024, at most kTiles of them
  int log = 10;
  while ((long)V + 3 > (long)kTiles << log) ++log;
  return log;
}

// A row that is left: all bins, the middle one 31 below the maximum, and step 4 by readings.
template <int T, bool BF16>
__device__ __forceinline__ void left_row(const DrawArgs& a, int row, Shared& s) {
  written_again();  // what was kept before the row was left
  Row<BF16> r;
  Limits lim;
  set_up(a, row, r, lim);
  lim.few = false;
  set_powers(s);
  const Fixed fixed(a.V);
  const int tile_log = tile_log_of(a.V);
  clear<T>(s);
  lds_barrier();
  float high = -INFINITY;
  each<T>(r, [&](int, const float(&y)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) high = fmaxf(high, y[i]);
  });
  const float top = top_of(s, high);
  const Bins bins{(double)top - 31.0};
  count<T>(s, r, 0, r.vectors(), lim, bins, fixed, high);
  lds_barrier();
  set_least(lim, top);
  Zone z;
  find_zone<T, kBins / T, true, false>(s, lim, bins, top, kBins - 1, 0, 0.0, z);
  const unsigned kept = keep<T, true>(s, r, 0, r.vectors(), lim, bins, fixed, z, top, tile_log);
  if (kept) atomicAdd(&s.kept, kept);
  lds_barrier();
  unsigned last = 0;
  int last_id = 0x7fffffff;
  if (z.zone) resolve_by_reading<T>(s, r, lim, bins, fixed, z, top, tile_log, last, last_id);
  token<T>(s, a, row, r, lim, fixed, top, tile_log, last, last_id);
}

// All steps for one row.  HERE: also where it is left; else left[row] says whether it is (the registers of what that takes would cost
// the second workgroup of a CU).
template <int T, bool BF16, bool HERE>
__global__ __launch_bounds__(T, HERE ? 1 : 4) void draw_rows_kernel(DrawArgs a, int* left) {
  constexpr int kWindow = 2048;
  constexpr bool GROUPS = !HERE;
  __shared__ Shared s;
  __shared__ float groups[GROUPS ? kGroups : 1];
  const int tid = threadIdx.x, row = blockIdx.x;
  Row<BF16> r;
  Limits lim;
  set_up(a, row, r, lim);
  set_powers(s);
  const Fixed fixed(a.V);
  const int tile_log = tile_log_of(a.V);
  clear<T>(s);
  lds_barrier();
  const Bins bins = bins_of<T>(s, r);
  float high = -INFINITY;
  count<T, GROUPS>(s, r, 0, r.vectors(), lim, bins, fixed, high, groups);
  const float top = top_of(s, high);
  if (!lim.law || !(top >= kNone) || s.found[1]) {
    no_logits<T>(r, 0, r.vectors());
    no_token(a, row);
    if (!HERE && tid == 0) left[row] = 0;
    return;
  }
  set_least(lim, top);
  Zone z{-1, kBins, -1, -1, 0, 0};
  bool here = true;
  if (by_k(lim) || by_p(lim)) {
    u64 all;
    double total;
    const int b0 = bins.of(top);
    totals<T>(s, lim, bins, top, b0 - kWindow + 1, all, total);
    here = find_zone<T, kWindow / T, false, true>(s, lim, bins, top, b0, all, total, z) && bins.serve(top);
    lds_barrier();
  }
  if (here) {
    const unsigned kept = keep<T, !HERE, GROUPS>(s, r, 0, r.vectors(), lim, bins, fixed, z, top, tile_log, groups);
    if (kept) atomicAdd(&s.kept, kept);
    lds_barrier();
  }
  here = here && s.list_n <= kList;
  if (!HERE && tid == 0) left[row] = !here;
  if (!here) {
    if constexpr (HERE) left_row<T, BF16>(a, row, s);
    return;
  }
  unsigned last = 0;
  int last_id = 0x7fffffff;
  if (z.zone) resolve<T>(s, r, lim, bins, fixed, z, top, tile_log, s.list_n, last, last_id);
  token<T>(s, a, row, r, lim, fixed, top, tile_log, last, last_id);
}

template <int T, bool BF16>
__global__ __launch_bounds__(T) void draw_left_kernel(DrawArgs a, const int* left) {
  __shared__ Shared s;
  if (left[blockIdx.x]) left_row<T, BF16>(a, blockIdx.x, s);
}

// ---- slices ------------------------------------------------------------------------------------------
constexpr int kSliceT = 1024, kFinishT = 512;   // threads (slices of 35 rows of V = 100003 with 512: 48.2 us, with 1024: 45.5)
constexpr int kMostSlices = 8, kCus = 256;     // of a row (16 for 8 rows: bins 10.7 -> 8.5 us, adding them up and the list 12.0 -> 13.0); of the card
constexpr int kWindow = 1024;                  // bins that a slice leaves: 32 below its maximum

// What a slice leaves of step 1: the topmost kWindow of its bins with tokens, which reach as far down as those of the row.
struct Slice {
  unsigned top_key, bad;
  double ref;
  int high, pad;       // its topmost bin
  u64 all;             // its tokens
  double total;        // and their mass times exp(-ref), of 2^-f
  struct {
    u64 mass;
    unsigned cnt, pad;
  } bin[kWindow];      // bins high, high - 1, ...
};
// What a row's slices leave of steps 2 and 3.
struct RowZone {
  unsigned n;          // entries of the list; more than kList: the list is not whole
  int law, left;
  float top;
  unsigned least;
  double ref;
  Zone z;
  int high;            // topmost bin
  unsigned above_k;
  double mass[kWindow];  // above bins high, high - 1, ...
  u64 list[kList];
};
struct Slices {
  Slice* slice;     // [rows, n]
  RowZone* row;     // [rows]
  u64* tile;        // [rows, tiles] kept mass
  unsigned* kept;   // [rows, n]
  int n, log, tiles;  // slices per row, of 2^log positions; tiles per row
};

// What a workgroup does of `all` pieces of work: neighbours on one XCD, whose L2 holds a row and its bins from one launch to the next (35 rows of
// V = 100003 45.5 -> 39.5 us).  Not less than `all`: nothing.
__device__ __forceinline__ int of_xcd(int all) {
  const int per = (all + 7) / 8, at = (int)(blockIdx.x >> 3);
  return at < per ? (int)(blockIdx.x & 7) * per + at : all;
}

template <bool BF16>
__global__ __launch_bounds__(kSliceT) void draw_bins_kernel(DrawArgs a, Slices sl) {
  constexpr int T = kSliceT;
  __shared__ Shared s;
  const int id = of_xcd(a.B * a.K * sl.n);
  if (id >= a.B * a.K * sl.n) return;
  const int tid = threadIdx.x, row = id / sl.n, i = id % sl.n;
  Row<BF16> r;
  Limits lim;
  set_up(a, row, r, lim);
  set_powers(s);
  const Fixed fixed(a.V);
  clear<T>(s);
  if (tid == 0 && i == 0) sl.row[row].n = 0;
  lds_barrier();
  const Bins bins = bins_of<T>(s, r);
  float high = -INFINITY;
  const int begin = i << (sl.log - 2), end = min(r.vectors(), (i + 1) << (sl.log - 2));
  count<T>(s, r, begin, end, lim, bins, fixed, high);
  const float top = top_of(s, high);
  Slice& o = sl.slice[id];
  const int b0 = top >= kNone ? bins.of(top) : 0;
  if (by_k(lim) || by_mass(lim)) {
    for (int j = tid; j < kWindow; j += T) {
      const int bin = b0 - j;
      o.bin[j] = {by_mass(lim) && bin >= 0 ? s.mass[bin] : 0, by_k(lim) && bin >= 0 ? s.cnt[bin] : 0, 0};
    }
    u64 all;
    double total;
    totals<T>(s, lim, bins, bins.ref, kBins, all, total);  // (at most 48 above the sample: no overflow)
    if (tid == 0) {
      o.all = all;
      o.total = total;
    }
  }
  if (tid == 0) {
    o.top_key = key_of(top);
    o.bad = s.found[1];
    o.ref = bins.ref;
    o.high = b0;
  }
}

template <bool BF16>
__global__ __launch_bounds__(kSliceT) void draw_keep_kernel(DrawArgs a, Slices sl) {
  constexpr int T = kSliceT, kPer = kWindow / T;
  __shared__ Shared s;
  const int id = of_xcd(a.B * a.K * sl.n);
  if (id >= a.B * a.K * sl.n) return;
  const int tid = threadIdx.x, row = id / sl.n, at = id % sl.n, n = sl.n;
  const Slice* const slice = sl.slice + (size_t)row * n;
  RowZone& o = sl.row[row];
  Row<BF16> r;
  Limits lim;
  set_up(a, row, r, lim);
  set_powers(s);
  for (int i = tid; i < kTiles; i += T) s.tile[i] = 0;
  if (tid == 0) s.found[0] = s.found[1] = s.found[3] = s.kept = s.list_n = 0;
  const Bins bins{slice[0].ref};
  u64 all = 0;
  double total = 0;
  lds_barrier();
  if (tid < n) {
    atomicMax(&s.found[0], slice[tid].top_key);
    atomicMax(&s.found[3], (unsigned)slice[tid].high);
    if (slice[tid].bad) s.found[1] = 1;
    s.list[tid] = (u64)slice[tid].high;
    s.list[64 + tid] = slice[tid].all;
    s.list[128 + tid] = __builtin_bit_cast(u64, slice[tid].total);
  }
  lds_barrier();
  const float top = of_key(s.found[0]);
  const bool law = lim.law && top >= kNone && !s.found[1];
  const int b0 = (int)s.found[3];
  const int begin = at << (sl.log - 2), end = min(r.vectors(), (at + 1) << (sl.log - 2));
  Zone z{-1, kBins, -1, -1, 0, 0};
  bool here = true;
  if (law) {
    set_least(lim, top);
    if (by_k(lim) || by_mass(lim)) {
      for (int i = 0; i < n; ++i) {
        all += s.list[64 + i];
        total += __builtin_bit_cast(double, s.list[128 + i]);
      }
      total *= exp(bins.ref - (double)top);
      unsigned c[kPer] = {};
      u64 w[kPer] = {};
      {
        unsigned ci[kMostSlices][kPer];
        u64 wi[kMostSlices][kPer];
#pragma unroll
        for (int i = 0; i < kMostSlices; ++i)
#pragma unroll
          for (int q = 0; q < kPer; ++q) {
            const int k = min(i, n - 1), j = (int)s.list[k] - (b0 - kPer * tid - q);
            const bool is = i < n && j >= 0;
            ci[i][q] = is ? slice[k].bin[j].cnt : 0;
            wi[i][q] = is ? slice[k].bin[j].mass : 0;
          }
#pragma unroll
        for (int i = 0; i < kMostSlices; ++i)
#pragma unroll
          for (int q = 0; q < kPer; ++q) {
            c[q] += ci[i][q];
            w[q] += wi[i][q];
          }
      }
#pragma unroll
      for (int q = 0; q < kPer; ++q) {
        const int bin = b0 - kPer * tid - q;
        if (bin >= 0) {
          s.cnt[bin] = c[q];
          s.mass[bin] = w[q];
        }
      }
      lds_barrier();
      here = find_zone<T, kPer, false, false>(s, lim, bins, top, b0, all, total, z) && bins.serve(top);
      lds_barrier();
    }
  }
  if (at == 0) {
    if (tid == 0) {
      o.law = law;
      o.left = !here;
      o.top = top;
      o.ref = bins.ref;
      o.least = lim.least;
      o.high = b0;
      o.above_k = s.above_k;
      o.z = z;
    }
    if (z.zone && by_mass(lim))
#pragma unroll
      for (int q = 0; q < kPer; ++q) o.mass[kPer * tid + q] = b0 >= kPer * tid + q ? __builtin_bit_cast(double, s.mass[b0 - kPer * tid - q]) : 0;
  }
  if (!law) no_logits<T>(r, begin, end);
  if (!law || !here) return;
  const int tile_log = tile_log_of(a.V);
  const unsigned kept = keep<T, true>(s, r, begin, end, lim, bins, Fixed(a.V), z, top, tile_log);
  if (kept) atomicAdd(&s.kept, kept);
  lds_barrier();
  const unsigned mine = s.list_n;
  if (tid == 0 && mine) s.found[2] = atomicAdd(&o.n, mine);
  lds_barrier();
  for (unsigned i = tid; i < min(mine, (unsigned)kList); i += T)
    if (s.found[2] + i < kList) o.list[s.found[2] + i] = s.list[i];
  const int t0 = at << (sl.log - tile_log), t1 = min(sl.tiles, (at + 1) << (sl.log - tile_log));
  for (int t = t0 + tid; t < t1; t += T) sl.tile[(size_t)row * sl.tiles + t] = s.tile[t];
  if (tid == 0) sl.kept[id] = s.kept;
}

template <bool BF16>
__global__ __launch_bounds__(kFinishT) void draw_finish_kernel(DrawArgs a, Slices sl) {
  constexpr int T = kFinishT;
  __shared__ Shared s;
  const int tid = threadIdx.x, row = of_xcd(a.B * a.K);
  if (row >= a.B * a.K) return;
  const RowZone& o = sl.row[row];
  Row<BF16> r;
  Limits lim;
  set_up(a, row, r, lim);
  set_powers(s);
  // everything that may be needed at once, one latency for all of it: a list behind its end, and what a row without a law or one that is
  // left did not write, is not looked at
  u64 list[kList / T];
  double mass[kWindow / T];
#pragma unroll
  for (int i = 0; i < kList / T; ++i) list[i] = o.list[tid + i * T];
#pragma unroll
  for (int i = 0; i < kWindow / T; ++i) mass[i] = o.mass[tid + i * T];
  static_assert(kTiles <= T, "");
  const u64 tile = tid < sl.tiles ? sl.tile[(size_t)row * sl.tiles + tid] : 0;
  const unsigned kept = tid < sl.n ? sl.kept[(size_t)row * sl.n + tid] : 0;
  const unsigned n = o.n;
  const int high = o.high;
  if (tid < kTiles) s.tile[tid] = tile;
#pragma unroll
  for (int i = 0; i < kList / T; ++i) s.list[tid + i * T] = list[i];
#pragma unroll
  for (int i = 0; i < kWindow / T; ++i)
    if (high >= tid + i * T) s.mass[high - tid - i * T] = __builtin_bit_cast(u64, mass[i]);
  if (tid == 0) {
    s.kept = 0;
    s.above_k = o.above_k;
  }
  lds_barrier();
  if (tid < sl.n) atomicAdd(&s.kept, kept);
  if (!o.law) {
    no_token(a, row);
    return;
  }
  if (o.left || n > kList) {
    left_row<T, BF16>(a, row, s);
    return;
  }
  const Zone z = o.z;
  const float top = o.top;
  const Bins bins{o.ref};
  lim.least = o.least;
  lds_barrier();
  const Fixed fixed(a.V);
  const int tile_log = tile_log_of(a.V);
  unsigned last = 0;
  int last_id = 0x7fffffff;
  if (z.zone) resolve<T>(s, r, lim, bins, fixed, z, top, tile_log, n, last, last_id);
  token<T>(s, a, row, r, lim, fixed, top, tile_log, last, last_id);
}

// Slices of a call: 0, or their number for each row, of 2^*log positions each.
int slices_of(int rows, int V, int* log) {
  *log = 12 > tile_log_of(V) ? 12 : tile_log_of(V);
  if (rows >= kManyRows || V < kShort) return 0;
  const int most = kCus / rows < kMostSlices ? kCus / rows : kMostSlices;
  while (((long)V + 3 + (1L << *log) - 1) >> *log > most) ++*log;
  return (int)(((long)V + 3 + (1L << *log) - 1) >> *log);
}
int tiles_of(int V) { return (int)(((long)V + 3 + (1L << tile_log_of(V)) - 1) >> tile_log_of(V)); }

}  // namespace

size_t draw_workspace(int rows, int V) {
  int log;
  const size_t n = (size_t)slices_of(rows, V, &log) * rows;
  return n ? n * (sizeof(Slice) + sizeof(unsigned)) + rows * (sizeof(RowZone) + tiles_of(V) * sizeof(u64)) : (size_t)rows * sizeof(int);
}

hipError_t launch_draw(const DrawArgs& a) {
  const int rows = a.B * a.K;
  Slices sl;
  sl.n = slices_of(rows, a.V, &sl.log);
  sl.tiles = tiles_of(a.V);
  const size_t n = (size_t)sl.n * rows;
  sl.slice = (Slice*)a.workspace;
  sl.row = (RowZone*)(sl.slice + n);
  sl.tile = (u64*)(sl.row + rows);
  sl.kept = (unsigned*)(sl.tile + (size_t)rows * sl.tiles);
  int* const left = (int*)a.workspace;
  auto run = [&](auto bf16) {
    constexpr bool B16 = decltype(bf16)::value;
    if (n) {
      hipLaunchKernelGGL(draw_bins_kernel<B16>, dim3((unsigned)((n + 7) / 8 * 8)), dim3(kSliceT), 0, a.stream, a, sl);
      hipLaunchKernelGGL(draw_keep_kernel<B16>, dim3((unsigned)((n + 7) / 8 * 8)), dim3(kSliceT), 0, a.stream, a, sl);
      hipLaunchKernelGGL(draw_finish_kernel<B16>, dim3((rows + 7) / 8 * 8), dim3(kFinishT), 0, a.stream, a, sl);
    } else if (a.V < kShort) {
      hipLaunchKernelGGL((draw_rows_kernel<512, B16, true>), dim3(rows), dim3(512), 0, a.stream, a, left);
    } else {
      hipLaunchKernelGGL((draw_rows_kernel<512, B16, false>), dim3(rows), dim3(512), 0, a.stream, a, left);
      hipLaunchKernelGGL((draw_left_kernel<512, B16>), dim3(rows), dim3(512), 0, a.stream, a, left);
    }
  };
  if (a.bf16) run(std::true_type{});
  else run(std::false_type{});
  return hipGetLastError();
}

}  // namespace fef
