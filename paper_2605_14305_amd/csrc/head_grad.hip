// Gradients of the head's cross-entropy (fef_head_cross_entropy_grad), bf16: with z = H W^T / tau, and G[r, v] =
// g_r (exp(z[r, v] - lse_r) - [v = label_r]) / tau, grad_H = G W and grad_W = G^T H.
//
// z comes from the head kernels, G is made from it in one pass (rounded to bf16: it is an operand of the matrix cores, whose products
// are summed in 32 bits), and two products of 2 R d V operations follow, each on the same kernel: C[m, n] = sum_k A[m, k] B[k, n].  B (W, or
// H) has n contiguous, so its fragments are read from LDS transposed (ds_read_b64_tr_b16).  A is G, with k (the tokens, for grad_H)
// or m (the tokens, for grad_W: read transposed too) contiguous.  No transposed copy of anything is made.
#include <type_traits>

#include "head_common.hpp"
#include "wave_ops.hpp"

namespace fef {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------------
// G from z
// ---------------------------------------------------------------------------------------------
constexpr int NT = 256, kQuads = 4, kChunk = NT * 4 * kQuads;  // tokens per workgroup

// Log-sum-exp of a row from its partials, in every thread; fixed order.
__device__ __forceinline__ float row_lse(const float2* P, int n) {
  __shared__ float2 part[NT / kWave];
  const int tid = threadIdx.x;
  float mx = kLowest, sm = 0.f;
  for (int t0 = tid; t0 < n; t0 += 4 * NT) {  // four loads in flight
    float2 p[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = t0 + j * NT < n ? P[t0 + j * NT] : make_float2(kLowest, 0.f);
    const float m = fmaxf(fmaxf(fmaxf(p[0].x, p[1].x), fmaxf(p[2].x, p[3].x)), mx);
    sm *= expf(mx - m);
#pragma unroll
    for (int j = 0; j < 4; ++j) sm += p[j].y * expf(p[j].x - m);
    mx = m;
  }
  const float top = wave_max(mx);
  sm = wave_sum(sm * expf(mx - top));
  if ((tid & 63) == 0) part[tid >> 6] = make_float2(top, sm);
  __syncthreads();
  mx = fmaxf(fmaxf(part[0].x, part[1].x), fmaxf(part[2].x, part[3].x));
  static_assert(NT / kWave == 4, "");
  sm = 0.f;
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) sm += part[w].y * expf(part[w].x - mx);
  return mx + logf(sm);
}

template <class T>
__device__ __forceinline__ void store_quad(T* p, const T (&o)[4]) {
  if constexpr (sizeof(T) == 2) {
    uint2 u;
    __builtin_memcpy(&u, o, 8);
    *reinterpret_cast<uint2*>(p) = u;
  } else {
    *reinterpret_cast<float4*>(p) = make_float4(o[0], o[1], o[2], o[3]);
  }
}

// A row of G (zeros behind the vocabulary, in rows that do not count and in the rows that fill up a block of 64), the row's loss, and its row
// of H.  G may be z itself (float).
//
// What bounds it: z read and G written, 1.55 GB at 2048 rows of V = 126464 in 257 us (6.0 TB/s; with a quad per thread and turn 327); a few rows: the way from the partials to the
// log-sum-exp, in whose shade the logits are read.
template <class T>
__global__ __launch_bounds__(NT) void grad_rows_kernel(GradArgs a) {
  const int r = blockIdx.y, tid = threadIdx.x;
  const int v0 = blockIdx.x * kChunk + 4 * tid;  // the thread's quads: every 4 NT tokens; a.ldl is a multiple of 64
  T* G = (T*)a.G + (size_t)r * a.ldl;
  const int label = r < a.rows ? a.labels[r] : -1;
  if (blockIdx.x == 0 && a.H) {  // (of grad_W) what a row that does not count holds is not looked at
    const T* from = (const T*)a.h + (size_t)r * a.d;
    T* to = (T*)a.H + (size_t)r * a.d;
    if (a.d % 4 == 0) {
      for (int k = 4 * tid; k < a.d; k += 4 * NT) {
        T x[4] = {(T)0.f, (T)0.f, (T)0.f, (T)0.f};
        if (label >= 0) __builtin_memcpy(x, from + k, sizeof x);
        store_quad(to + k, x);
      }
    } else {
      for (int k = tid; k < a.d; k += NT) to[k] = label >= 0 ? from[k] : (T)0.f;
    }
  }
  if (label < 0) {  // workgroup-uniform
    const T zero[4] = {(T)0.f, (T)0.f, (T)0.f, (T)0.f};
#pragma unroll
    for (int q = 0; q < kQuads; ++q)
      if (v0 + q * 4 * NT < a.ldl) store_quad(G + v0 + q * 4 * NT, zero);
    if (blockIdx.x == 0 && r < a.rows && tid == 0) {
      a.out_ce[r] = 0.f;
      if (a.rest) a.rest[r] = 0.f;
    }
    return;
  }
  const float* z = a.z + (size_t)r * a.ldl;
  floatx4 x[kQuads];
#pragma unroll
  for (int q = 0; q < kQuads; ++q)
    x[q] = v0 + q * 4 * NT < a.ldl ? *reinterpret_cast<const floatx4*>(z + v0 + q * 4 * NT) : floatx4{0.f, 0.f, 0.f, 0.f};
  const float lse = row_lse(a.partials + (size_t)r * a.nT, a.nT);
  const bool known = label < a.V;
  if (!known && blockIdx.x == 0 && tid == 0) {
    a.out_ce[r] = __builtin_nanf("");
    if (a.rest) a.rest[r] = 0.f;
  }
  const float g = known ? (a.weights ? a.weights[r] : 1.f) * a.inv_tau : __builtin_nanf("");
#pragma unroll
  for (int q = 0; q < kQuads; ++q) {
    const int v = v0 + q * 4 * NT;
    if (v >= a.ldl) break;
    T o[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float p = expf(x[q][c] - lse);
      if (known && v + c == label) {  // an unknown label may be a place of the padding
        p -= 1.f;
        a.out_ce[r] = lse - x[q][c];
        const float rest = p * g - (float)(T)(p * g);
        if (a.rest) a.rest[r] = fabsf(rest) < INFINITY ? rest : 0.f;
      }
      o[c] = (T)(v + c < a.V ? p * g : 0.f);
    }
    store_quad(G + v, o);
  }
}

// ---------------------------------------------------------------------------------------------
// C = A B, bf16 operands
// ---------------------------------------------------------------------------------------------
constexpr int BN = 256, BK = 64, HK = 32, WM = 2, kStrip = 4;

// Rows of `cols` columns in LDS, a row per k, 32 bytes (16 columns) at chunk c ^ turn_of(k): the 32 lanes of half a transposed read, which take
// 32 bytes of rows 8 g + {0, 1, 2, 3} of two lane groups g, fall on different banks.
template <int COLS>
__device__ __forceinline__ int turn_of(int k) {
  if constexpr (COLS >= 128) return (k & 3) | ((k >> 3) & 1) << 2;
  else return ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
}

// Four 16-bit values of a column of 4 rows x 16 columns whose row r lies in lanes 4 r .. 4 r + 3 of each group of 16.
__device__ __forceinline__ bf16x4 read_turned(const char* p) {
  typedef __attribute__((address_space(3))) shortx4* P;
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(shortx4*)p));
}
__device__ __forceinline__ bf16x8 both(bf16x4 a, bf16x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// Four columns of row m of grad_h, to which its sum is added what rounding took from G at the label, times the label's row of W.  A row that
// does not count is 0, also where W holds a NaN or an infinity, which its zeros of G have been multiplied by.
__device__ __forceinline__ floatx4 with_rest(floatx4 sum, const float* rest, const int* labels, int m, const __bf16* W, long ldw, int c) {
  const int label = labels[m];
  if (label < 0) return floatx4{0.f, 0.f, 0.f, 0.f};
  const float x = rest[m];
  if (x != 0.f) {  // (then the label is one of the vocabulary)
    const bf16x4 w = *reinterpret_cast<const bf16x4*>(W + (size_t)label * ldw + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += x * (float)w[i];
  }
  return sum;
}

// Tile of 32 NR rows x 256 columns, 2 x WN wavefronts of 16 NR rows.  AT: A is [K][M] (m contiguous), else [M][K].  OUT: __bf16 for C itself,
// float for the partial sums of a share of k.
//
// k goes in halves of 32 columns.  While a half is multiplied out of registers, the fragments of the next one are read from LDS, and the
// halves behind that are on their way from memory to LDS: B in a ring of halves, A likewise (AT), or in a ring of stages of 64 columns (rows
// of 128 bytes: 64-byte pieces move at 60 % of the rate out of L2).  One barrier per half.
//
// What bounds it: LDS and the matrix units alike.  A half of 256 x 256 x 32 takes 1024 cycles of multiplies, and with eight wavefronts of
// 128 x 64 96 KB of fragments and 32 KB on their way in, 1024 cycles of LDS.  Four wavefronts of 128 x 128 read 64 KB, but with one wavefront per
// SIMD every other instruction holds the multiplies: grad_h of 2048 rows of d = 4096, V = 126464 1655 -> 1931 us, grad_w 1963 -> 2092.
//   grad_h (WN = 4): few long tiles.  1655 to 1760 us = 1.21 to 1.28 PFLOP/s, with the card's clock (fragments read where they are multiplied, one
//     step ahead: 1816).
//   grad_w (WN = 2, 128 x 256): K is the number of rows, so a tile is short, and filling the rings and writing 64 KB weigh as much as the
//     multiplies.  Two workgroups per CU, in 72 KB each, work under each other's ends: 1903 us, against 1963 with
//     one of 256 x 256; 48 rows 290 -> 273, 333 rows of d = 2048, V = 50257 128 -> 112 (with stores past the caches 263 and 102).  An XCD walks
//     down a strip of kStrip tiles, whose columns of H (4 MB at 2048 rows) stay in its L2: 1740 us = 1.22 PFLOP/s, 4.3 GB read (strips of 8 tiles
//     1785 us, 6.2 GB; rows of all 16 1898 us, 12.0 GB).  With the labels' rounding made good, which takes the
//     gradients' error against 64 bits from 0.0024 to 0.0018 of their norm, 30 registers are spilled and the kernel takes 1976 us (1.07 PFLOP/s, 4.7 GB
//     read, 1.5 GB written, a third of it spills), 373 at 48 rows, 143 at 333.
template <int NR, int WN, bool AT, class OUT>
__global__ __launch_bounds__(128 * WN, WN == 2 ? 2 : 1) void grad_product_kernel(ProductArgs a) {
  constexpr int BM = 16 * NR * WM, kWaves = WM * WN, kThreads = kWave * kWaves, kColumns = BN / WN / 16;
  constexpr int RA = WN == 2 ? 3 : NR == 8 ? 3 : 4, RB = WN == 2 ? 3 : NR == 8 ? 4 : 6;
  static_assert(AT == (WN == 2) && (AT ? RA == RB : RB % 2 == 0 && RB <= 2 * RA - 1), "the waits count on B being the younger one");
  constexpr bool ROLL = WN == 4;  // a fragment of A goes into the registers of the one that has had its last use, else into a second set
  constexpr int kStageA = BM * (AT ? HK : BK) * 2, kStageB = BN * HK * 2;
  constexpr int kLoadsA = kStageA / 1024, LA = (kLoadsA + kWaves - 1) / kWaves, LB = kStageB / 1024 / kWaves;
  static_assert(kLoadsA >= LA && LA <= 4 && LB <= 4, "");
  // loads younger than those that a half waits for
  constexpr int kYounger = AT ? (RB - 2) * (LA + LB) : (RB - 2) * LB + (RB - 2) / 2 * LA;
  constexpr int kPitch = BN + 8;  // of the tile in LDS on its way out: a wavefront stores whole rows of 512 bytes
  constexpr int kOut = sizeof(OUT) == 2 ? BM * kPitch * 2 : 0;
  constexpr int kRings = RA * kStageA + RB * kStageB;
  __shared__ __align__(16) char lds[kRings > kOut ? kRings : kOut];
  __shared__ uint64_t hits[AT ? kGradRows / 64 : 1];
  char* const ringA = lds;
  char* const ringB = lds + RA * kStageA;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int i16 = lane & 15, g = lane >> 4;

  // consecutive tiles on one XCD
  const int mt = (a.M + BM - 1) / BM, nt = (a.N + BN - 1) / BN;
  const long tiles = (long)mt * nt * a.shares, per = (tiles + 7) / 8;
  const long id = (long)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((long)(blockIdx.x >> 3) >= per || id >= tiles) return;
  const int share = (int)(id / ((long)mt * nt)), at = (int)(id % ((long)mt * nt));
  int tm = at % mt, tn = at / mt;
  if (a.n_first) {
    const int strip = at / (mt * kStrip), first = strip * kStrip, wide = min(kStrip, nt - first), in = at - mt * first;
    tm = in / wide;
    tn = first + in % wide;
  }
  const int m0 = tm * BM, n0 = tn * BN;
  const int nk_all = a.K / BK;
  const int k0 = (int)((long)share * nk_all / a.shares), nk = (int)((long)(share + 1) * nk_all / a.shares) - k0, nh = 2 * nk;

  // Direct-to-LDS loads of 1 KB: lane l fills slot (instruction, l) of 16 bytes.
  const __bf16* ga[LA];
  const __bf16* gb[LB];
  const int ia0 = min(wave * LA, kLoadsA - LA);  // where the rows do not divide, the last wavefronts repeat some
#pragma unroll
  for (int q = 0; q < LA; ++q) {
    const int s = (ia0 + q) * 64 + lane;
    if constexpr (AT) {
      const int k = s / (BM / 8), p = s % (BM / 8);
      const int m = m0 + (((p >> 1) ^ turn_of<BM>(k)) * 16 + (p & 1) * 8);
      ga[q] = a.A + (size_t)(k0 * BK + k) * a.lda + min(m, (a.M - 1) & ~7) - q * 512;
    } else {
      const int m = s / 8, c = (s & 7) ^ ((m >> 1) & 7);
      ga[q] = a.A + (size_t)min(m0 + m, a.M - 1) * a.lda + k0 * BK + c * 8 - q * 512;
    }
  }
  int b_in[LB], b_end = k0 * BK;  // row of a load within its half; end of the half that is loaded next
#pragma unroll
  for (int q = 0; q < LB; ++q) {
    const int s = (wave * LB + q) * 64 + lane;
    const int k = s / (BN / 8), p = s % (BN / 8);
    const int n = n0 + (((p >> 1) ^ turn_of<BN>(k)) * 16 + (p & 1) * 8);
    b_in[q] = k;
    gb[q] = a.B + (size_t)(k0 * BK + k) * a.ldb + min(n, a.N - 8) - q * 512;
  }
  const uint32_t slotA = lds_offset(ringA) + ia0 * 1024, slotB = lds_offset(ringB) + wave * LB * 1024;
  int put_a = 0, put_b = 0;  // ring positions of the next loads
  auto load_a = [&]() __attribute__((always_inline)) {
    load_group_to_lds<false>(ga, __builtin_amdgcn_readfirstlane(slotA + put_a * kStageA));
#pragma unroll
    for (int q = 0; q < LA; ++q) ga[q] += AT ? (long)HK * a.lda : (long)BK;
    put_a = put_a == RA - 1 ? 0 : put_a + 1;
  };
  auto load_b = [&]() __attribute__((always_inline)) {
    const uint32_t lds_off = __builtin_amdgcn_readfirstlane(slotB + put_b * kStageB);
    b_end += HK;
    if (b_end <= a.b_rows) {
      load_group_to_lds<false>(gb, lds_off);
    } else {  // rows past the last: the last once more, which meets zeros of A
      const __bf16* p[LB];
#pragma unroll
      for (int q = 0; q < LB; ++q) p[q] = gb[q] - (long)max(0, b_end - HK + b_in[q] - (a.b_rows - 1)) * a.ldb;
      load_group_to_lds<false>(p, lds_off);
    }
#pragma unroll
    for (int q = 0; q < LB; ++q) gb[q] += HK * a.ldb;
    put_b = put_b == RB - 1 ? 0 : put_b + 1;
  };
  // What half h brings on its way, in this order: A of half h + RB, or of stage (h - 1) / 2 + RA where h is odd; B of half h + RB.
  auto load = [&](int h, bool odd) __attribute__((always_inline)) {
    if constexpr (AT) {
      if (h + RB < nh) load_a();
    } else {
      if (odd && (h - 1) / 2 + RA < nk) load_a();
    }
    if (h + RB >= 0 && h + RB < nh) load_b();
  };

  floatx4 acc[NR][kColumns];
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int t = 0; t < kColumns; ++t) acc[n][t] = floatx4{0.f, 0.f, 0.f, 0.f};

  // byte offsets of a lane's fragments in a half, or stage
  const int kr = 8 * g + (i16 >> 2), cc = (i16 & 3) * 8;
  int ob[kColumns], oa[AT ? NR : 2];
#pragma unroll
  for (int t = 0; t < kColumns; ++t) ob[t] = kr * (BN * 2) + ((wn * kColumns + t) ^ turn_of<BN>(kr)) * 32 + cc;
  if constexpr (AT) {
#pragma unroll
    for (int n = 0; n < NR; ++n) oa[n] = kr * (BM * 2) + ((wm * NR + n) ^ turn_of<BM>(kr)) * 32 + cc;
  } else {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) oa[ks] = (wm * NR * 16 + i16) * 128 + (((ks * 4 + g) ^ ((i16 >> 1) & 7)) * 16);
  }

  bf16x8 nf[2][kColumns], mf[ROLL ? 1 : 2][NR];
  int get_a = 0, get_b = 0;  // ring positions of the half that is read next
  // Half h (ODD) is multiplied, half h + 1 is read.
  auto half = [&](int h, auto odd_tag, auto mul_tag, auto read_tag) __attribute__((always_inline)) {
    constexpr bool ODD = decltype(odd_tag)::value, MUL = decltype(mul_tag)::value, READ = decltype(read_tag)::value;
    constexpr int cur = ODD ? 1 : 0, next = cur ^ 1;
    if constexpr (READ) {
      if (h + (AT ? RB - 1 : 2 * RA - 2 > RB - 1 ? 2 * RA - 2 : RB - 1) < nh) wait_newer<kYounger>();  // all of these exist
      else wait_newer<0>();
    }
    lds_barrier();
    load(h, ODD);
    __builtin_amdgcn_sched_barrier(0);
    const char* sA = ringA + get_a * kStageA;
    const char* sB = ringB + get_b * kStageB;
    auto read_n = [&](int t) __attribute__((always_inline)) {
      nf[next][t] = both(read_turned(sB + ob[t]), read_turned(sB + ob[t] + 4 * BN * 2));
    };
    auto read_m = [&](int n) __attribute__((always_inline)) {
      bf16x8& f = mf[ROLL ? 0 : next][n];
      if constexpr (AT) f = both(read_turned(sA + oa[n]), read_turned(sA + oa[n] + 4 * BM * 2));
      else f = *reinterpret_cast<const bf16x8*>(sA + oa[ODD ? 0 : 1] + n * 2048);
    };
    // ROLL: behind a row's multiplies, its own and some of the columns' fragments; else one behind every second multiply or so
    constexpr int kReads = NR + kColumns, kEvery = NR * kColumns * 3 / 4 / kReads < 1 ? 1 : NR * kColumns * 3 / 4 / kReads;
    static_assert(ROLL || kReads * kEvery <= NR * kColumns, "");
#pragma unroll
    for (int x = 0; x < NR * kColumns; ++x) {
      const int n = x / kColumns, t = x % kColumns;
      if constexpr (MUL) acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(nf[cur][t], mf[ROLL ? 0 : cur][n], acc[n][t], 0, 0, 0);
      if constexpr (READ && ROLL) {
        if (t == kColumns - 1) {
          constexpr int kRows = NR < kColumns ? NR : kColumns;
          for (int q = n * kColumns / kRows; q < (n + 1) * kColumns / kRows && q < kColumns; ++q) read_n(q);
          read_m(n);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else if constexpr (READ) {
        if (x % kEvery == 0 && x / kEvery < kReads) {
          if (x / kEvery < kColumns) read_n(x / kEvery);
          else read_m(x / kEvery - kColumns);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (READ) {
      get_b = get_b == RB - 1 ? 0 : get_b + 1;
      if (AT || !ODD) get_a = get_a == RA - 1 ? 0 : get_a + 1;  // (the stage of the half read behind an odd one is read on)
    }
  };
  using Yes = std::true_type;
  using No = std::false_type;
  if (nk > 0) {
    for (int h = AT ? -RB : -2 * RA; h < -1; ++h) load(h, h & 1);
    if constexpr (AT) {  // which rows' labels lie in the tile, while the first halves are on their way
      constexpr int U = 2;
#pragma unroll 1
      for (int r0 = 64 * wave; r0 < a.rows; r0 += 64 * kWaves * U) {
        int label[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int r = r0 + 64 * kWaves * u + lane;
          label[u] = r < a.rows ? a.labels[r] : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int r = r0 + 64 * kWaves * u;
          const uint64_t is = __ballot(label[u] >= m0 && label[u] < m0 + BM);
          if (lane == 0 && r < a.rows) hits[r / 64] = is;
        }
      }
    }
    half(-1, Yes{}, No{}, Yes{});
    for (int p = 0; p < nk - 1; ++p) {
      half(2 * p, No{}, Yes{}, Yes{});
      half(2 * p + 1, Yes{}, Yes{}, Yes{});
    }
    half(nh - 2, No{}, Yes{}, Yes{});
    half(nh - 1, Yes{}, Yes{}, No{});
  }
  // acc[n][t]: columns 16 t + 4 g .. + 3 of row 16 n + i16 of the wavefront's tile
  if constexpr (AT) {
    // What rounding took from G at a row's label: that element is as large as all others of its row together, so its one rounding is most of the row's
    // error, while theirs are many and independent.  (In a row that is sure of another token that token's element is as large, and its rounding
    // stays.)  A multiply with one k for each of the tile's labels; its time hardly depends on how they lie: 2048 rows of d = 4096, V = 126464 5.53 ms
    // with labels drawn uniformly, 5.56 by 1 / rank, 5.49 with one label for all; 8192 rows 24.8, 25.7, 25.1.
    for (int q0 = 0; q0 < a.rows; q0 += 64 * 64) {
      const uint64_t here = q0 + 64 * lane < a.rows ? hits[q0 / 64 + lane] : 0;
      for (uint64_t some = __ballot(here != 0); some; some &= some - 1) {
        const int q = __builtin_ctzll(some);
        uint64_t mine = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(here >> 32), q) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)here, q);
        for (; mine; mine &= mine - 1) {
          const int r = q0 + 64 * q + __builtin_ctzll(mine), row = a.labels[r] - (m0 + wm * NR * 16);
          const __bf16 rest = (__bf16)a.rest[r];
#pragma unroll
          for (int t = 0; t < kColumns; ++t) {
            bf16x8 x{};
            x[0] = a.B[(size_t)r * a.ldb + min(n0 + (wn * kColumns + t) * 16 + i16, a.N - 1)];
            if (g != 0) x[0] = (__bf16)0.f;
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              bf16x8 y{};
              if (g == 0 && row == n * 16 + i16) y[0] = rest;
              acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, acc[n][t], 0, 0, 0);
            }
          }
        }
      }
    }
  }
  if constexpr (sizeof(OUT) == 4) {
    float* C = (float*)a.C + (size_t)share * a.stride;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int m = m0 + (wm * NR + n) * 16 + i16;
#pragma unroll
      for (int t = 0; t < kColumns; ++t) {
        const int c = n0 + (wn * kColumns + t) * 16 + 4 * g;
        if (m < a.M && c < a.N) {
          floatx4* p = reinterpret_cast<floatx4*>(C + (size_t)m * a.N + c);
          *p = a.add ? *p + acc[n][t] : acc[n][t];
        }
      }
    }
  } else {
    lds_barrier();  // nobody reads the rings any more
    __bf16* tile = reinterpret_cast<__bf16*>(lds);
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int t = 0; t < kColumns; ++t) {
        floatx4 x = acc[n][t];
        if constexpr (!AT) {
          const int m = m0 + (wm * NR + n) * 16 + i16, c = n0 + (wn * kColumns + t) * 16 + 4 * g;
          if (m < a.M && c < a.N) x = with_rest(x, a.rest, a.labels, m, a.B, a.ldb, c);
        }
        bf16x4 o;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = (__bf16)x[c];
        *reinterpret_cast<bf16x4*>(tile + ((wm * NR + n) * 16 + i16) * kPitch + (wn * kColumns + t) * 16 + 4 * g) = o;
      }
    lds_barrier();
    __bf16* C = (__bf16*)a.C;  // stored past the caches, which keep H, G and W: 48 rows of d = 4096, V = 126464 285 -> 263 us, their whole call 663 -> 593
    for (int s = tid; s < BM * (BN / 8); s += kThreads) {
      const int m = s / (BN / 8), c = (s % (BN / 8)) * 8;
      if (m0 + m < a.M && n0 + c < a.N)
        __builtin_nontemporal_store(*reinterpret_cast<const bf16x8*>(tile + m * kPitch + c), reinterpret_cast<bf16x8*>(C + (size_t)(m0 + m) * a.N + n0 + c));
    }
  }
}

// Sum of the shares' partial sums, in their order.  With labels: of grad_h, whose rows that do not count are 0; rest: and bf16.
template <class OUT>
__global__ __launch_bounds__(256) void grad_sum_kernel(const float* part, int shares, size_t stride, size_t n, OUT* out, const int* labels, int d, const float* rest,
                                                       const __bf16* W) {
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  floatx4 s = *reinterpret_cast<const floatx4*>(part + i);
  for (int j0 = 1; j0 < shares; j0 += 8) {  // eight loads in flight
    floatx4 x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = *reinterpret_cast<const floatx4*>(part + (size_t)min(j0 + j, shares - 1) * stride + i);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j0 + j < shares) s += x[j];
  }
  if (rest) {
    s = with_rest(s, rest, labels, (int)(i / d), W, d, (int)(i % d));  // (bf16: d is a multiple of 64)
  } else if (labels) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (i + c < n && labels[(i + c) / d] < 0) s[c] = 0.f;
  }
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (i + c < n) out[i + c] = (OUT)s[c];
}

template <int NR, int WN, bool AT>
hipError_t launch_rows(const ProductArgs& a, bool partial, hipStream_t stream) {
  constexpr int BM = 16 * NR * WM;
  const long tiles = (long)((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN) * a.shares;
  if (tiles >= 1L << 23) return hipErrorInvalidValue;  // 2^32 threads
  const dim3 grid((unsigned)(8 * ((tiles + 7) / 8))), threads(128 * WN);
  if (partial) hipLaunchKernelGGL((grad_product_kernel<NR, WN, AT, float>), grid, threads, 0, stream, a);
  else hipLaunchKernelGGL((grad_product_kernel<NR, WN, AT, __bf16>), grid, threads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_grad_rows(const GradArgs& a, bool bf16, hipStream_t stream) {
  const dim3 grid((unsigned)((a.ldl + kChunk - 1) / kChunk), (unsigned)a.padded), threads(NT);
  if (bf16) hipLaunchKernelGGL(grad_rows_kernel<__bf16>, grid, threads, 0, stream, a);
  else hipLaunchKernelGGL(grad_rows_kernel<float>, grid, threads, 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_grad_sum(const float* part, int shares, size_t stride, size_t n, void* out, bool bf16, const int* labels, int d, const float* rest,
                           const __bf16* W, hipStream_t stream) {
  const dim3 grid((unsigned)((n + 1023) / 1024)), threads(256);
  if (bf16) hipLaunchKernelGGL(grad_sum_kernel<__bf16>, grid, threads, 0, stream, part, shares, stride, n, (__bf16*)out, labels, d, rest, W);
  else hipLaunchKernelGGL(grad_sum_kernel<float>, grid, threads, 0, stream, part, shares, stride, n, (float*)out, labels, d, rest, W);
  return hipGetLastError();
}

// grad_H: rows of H to a tile (rows that do not exist are multiplied all the same: 48 rows of V = 126464 in tiles of 64 176 us, W read at 5.9 TB/s),
// and into how many shares k (the tokens) is cut so that the CUs have work.
static int grad_h_rows(int rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256; }
int grad_h_shares(int rows, int d, int V) {
  const int bm = grad_h_rows(rows);
  const long tiles = (long)((rows + bm - 1) / bm) * ((d + BN - 1) / BN);
  const long steps = (V + BK - 1) / BK, want = tiles >= 256 ? 1 : 256 / tiles;
  return (int)(want < steps ? want : steps);
}

hipError_t launch_grad_h(const ProductArgs& a, hipStream_t stream) {
  const bool partial = a.shares > 1;
  switch (grad_h_rows(a.M)) {
    case 32: return launch_rows<1, 4, false>(a, partial, stream);
    case 64: return launch_rows<2, 4, false>(a, partial, stream);
    case 128: return launch_rows<4, 4, false>(a, partial, stream);
    default: return launch_rows<8, 4, false>(a, partial, stream);
  }
}
hipError_t launch_grad_w(const ProductArgs& a, bool partial, hipStream_t stream) { return launch_rows<4, 2, true>(a, partial, stream); }

}  // namespace fef
