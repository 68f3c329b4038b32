// Logits of the vocabulary head from weights in 4 bits (OCP MX, MXFP4): logits[r, v] = inv_tau sum_k h[r, k] w[v, k],
// w[v, k] = e2m1(code) 2^(scale - 127) with a scale per 32 codes.
//
// Numbers.  A code times its scale has two significant bits, so below 2^128 it is exact in bf16 (from there on infinite), and v_cvt_scalef32_pk_bf16_fp4 makes two of
// them with their scale in one instruction (checked over all codes and scales: exact, subnormals too, scale 255 gives NaN).  The
// products run on v_mfma_f32_16x16x32_bf16 with float32 sums.  The scaled 8-bit multiplies would take the codes as they are, but add
// with 13 to 15 bits only (measured: error 2^-13.5 of the sum of magnitudes), and two of them per bf16 value cost as much time.
// Hidden states in float32 are cut into three bf16 parts, 8 bits each, whose sum is the value itself.
//
// Layout.  The multiply adds over k in any order as long as both operands agree on it.  Lane l = (token or row l % 16, group g = l / 16)
// takes the 32 codes of block 4 u + g (16 bytes and one scale), which feed four multiplies of 8 codes per lane; of h it takes the same
// columns.  Tokens are the rows of D, so a lane ends with four consecutive tokens of one row of h.
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "head_common.hpp"

namespace fef {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int intx4 __attribute__((ext_vector_type(4)));

struct __attribute__((packed, aligned(4))) Float4 { float v[4]; };

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

constexpr int kWaves = 8, kThreads = kWaves * kWave;

// 16 or 4 bytes per lane from base + offset straight to LDS, lane after lane from lds_off on; counted by hand (wait_newer).
__device__ __forceinline__ void request_16(const void* base, uint32_t offset, uint32_t lds_off) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(offset), "s"(base), "s"(lds_off) : "memory");
}
__device__ __forceinline__ void request_4(const void* base, uint32_t offset, uint32_t lds_off) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" :: "v"(offset), "s"(base), "s"(lds_off) : "memory");
}

typedef float floatx4_any __attribute__((ext_vector_type(4), aligned(4)));

// Rows whose h fits the registers, 16 MT at a time.  A workgroup per CU takes a run of 16-token tiles in stages of TG of them, up to 32 KB
// of codes and 2 KB of scales, which come in the order of memory straight into LDS, RING - 1 stages ahead.  Its eight wavefronts are KS
// slices of k times TG = 8 / KS tiles: a wavefront holds its slice of h as operands for the whole kernel (UPW units of 128 columns) and
// multiplies its codes of each stage with it; the KS partial sums of a tile meet in LDS and are added in the order of the slices by one
// thread per sum while the next stage is multiplied.  One barrier per stage.
// LDS holds a stage's rows one behind another, their 16-byte chunks exchanged within 256 bytes (chunk ^ row, as far as the row length
// allows) so that 16 rows meet all banks.
// Bound: the read of the codes.  8 rows of d = 4096, V = 126464 (279 MB) 51.6 us, 5.4 TB/s; a plain read of as much takes 45 to 46.  Stages of
// 32 KB in the order of memory are what carries it: codes loaded from memory into registers by the wavefronts that
// use them took 70.  With 32 rows 63 to 67 us.  Of a short head the start (launch, h, the first stage's way from memory: 4 of the 5
// us at d = 512, V = 5000) and a barrier per stage count (16 float32 rows of d = 1024, V = 32000, eight stages of 8 KB: 11.6 us against 3.2
// of bytes); a ring of five or six such stages changes nothing (12.1, 12.4).
template <int UPW, int MT, bool F32>
__global__ __launch_bounds__(kThreads, 2) void mx4_stages_kernel(Mx4Args a, int KS, int runs, int row_blocks) {
  constexpr int P = F32 ? 3 : 1, ROWS = 16 * MT;
  constexpr int RING = 3;
  constexpr int kCodes = UPW * kThreads;                       // chunks of 16 bytes per stage
  constexpr int kOut = MT == 1 ? 32 : 12, kOutLd = kOut * 16 + 4;  // tiles of logits that wait in LDS
  __shared__ intx4 s_codes[RING][kCodes];
  __shared__ int s_scales[RING][kThreads];
  __shared__ floatx4 s_sum[2][MT][kWaves][kWave];
  __shared__ __attribute__((aligned(16))) float s_out[ROWS][kOutLd];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g = lane >> 4;
  const int TG = kWaves / KS, slice = wave % KS, tg = wave / KS;
  const int nb = a.d / 32, nu = (nb + 3) / 4;
  const int u0 = slice * nu / KS, count = (slice + 1) * nu / KS - u0;  // UPW or UPW - 1
  const int swap = min(nb & -nb, 16) - 1;
  const int tiles = (a.V + 15) / 16;
  // Row blocks of a run go to one XCD one behind another: its codes come from memory once.
  const int q8 = blockIdx.x >> 3, by = q8 % row_blocks, bx = q8 / row_blocks * 8 + (blockIdx.x & 7);
  if (bx >= runs) return;
  const int run0 = (int)((long)bx * tiles / runs), run1 = (int)((long)(bx + 1) * tiles / runs);
  const int stages = (run1 - run0 + TG - 1) / TG;
  const int row0 = by * ROWS;

  // Where this lane's chunks and its word of scales come from, relative to the stage's first token; `last`: the last token there is.
  auto chunk_at = [&](int i, int last) {
    const int s = min((i * kWaves + wave) * kWave + lane, TG * 16 * nb - 1), row = s / nb;
    return (uint32_t)(min(row, last) * nb + ((s - row * nb) ^ (row & swap))) * 16;
  };
  uint32_t code_off[UPW];
#pragma unroll
  for (int i = 0; i < UPW; ++i) code_off[i] = chunk_at(i, TG * 16);
  const uint32_t scale_off = (uint32_t)min(tid, TG * 4 * nb - 1) * 4;
  auto request = [&](int stage) {
    const int tok0 = (run0 + stage * TG) * 16, slot = stage % RING;
    const uint8_t* codes = a.codes + (size_t)tok0 * (a.d / 2);
    const uint8_t* scales = a.scales + (size_t)tok0 * nb;
    const uint32_t c_lds = lds_offset(&s_codes[slot][wave * kWave]), s_lds = lds_offset(&s_scales[slot][wave * kWave]);
    if (tok0 + TG * 16 <= a.V) {
#pragma unroll
      for (int i = 0; i < UPW; ++i) request_16(codes, code_off[i], c_lds + i * (kThreads * 16));
      request_4(scales, scale_off, s_lds);
    } else {  // the vocabulary ends inside: its last token again; the last word of scales that lies inside
#pragma unroll
      for (int i = 0; i < UPW; ++i) request_16(codes, chunk_at(i, a.V - 1 - tok0), c_lds + i * (kThreads * 16));
      request_4(scales, min(scale_off, (uint32_t)((a.V - tok0) * nb / 4 - 1) * 4), s_lds);
    }
  };
#pragma unroll
  for (int s = 0; s < RING - 1; ++s)
    if (s < stages) request(s);

  bf16x8 h[UPW][4][P][MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const size_t row = min(row0 + 16 * m + i16, a.R - 1);
#pragma unroll
    for (int u = 0; u < UPW; ++u)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int k = (u0 + u) * 128 + g * 32 + q * 8;
        const bool in = u < count && k < a.d;
        if constexpr (F32) {
          float x[8] = {};
          if (in) {
            *reinterpret_cast<floatx4*>(x) = *reinterpret_cast<const floatx4*>((const float*)a.h + row * a.d + k);
            *reinterpret_cast<floatx4*>(x + 4) = *reinterpret_cast<const floatx4*>((const float*)a.h + row * a.d + k + 4);
          }
          bf16x8 part[3];
          split3(x, part);
#pragma unroll
          for (int p = 0; p < P; ++p) h[u][q][p][m] = part[p];
        } else {
          h[u][q][0][m] = bf16x8{};
          if (in) h[u][q][0][m] = *reinterpret_cast<const bf16x8*>((const __bf16*)a.h + row * a.d + k);
        }
      }
  }

  // waited for here: the compiler, which does not know the requests, would wait for all of them at h's first use in the loop
#pragma unroll
  for (int u = 0; u < UPW; ++u)
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int m = 0; m < MT; ++m) asm volatile("" : "+v"(h[u][q][p][m]));

  // Logits wait in LDS and leave in long pieces: flushes of up to per_flush stages.
  const int flushes = (stages + kOut / TG - 1) / (kOut / TG), per_flush = (stages + flushes - 1) / flushes;
  auto add_up = [&](int stage) {  // a thread per (tile, row, token), TG * MT * 256 of them
    const int at = stage % per_flush * TG;
#pragma unroll 1
    for (int j = tid; j < TG * MT * 256; j += kThreads) {
      const int l = (j >> 2) & 63, e = j & 3, x = j >> 8, m = x % MT, t = x / MT;
      const float* from = reinterpret_cast<const float*>(&s_sum[stage & 1][m][t * KS][l]) + e;
      float y = from[0];
      if (KS == 8) {
#pragma unroll
        for (int v = 1; v < 8; ++v) y += from[v * 256];
      } else {
        for (int v = 1; v < KS; ++v) y += from[v * 256];
      }
      s_out[16 * m + (l & 15)][(at + t) * 16 + 4 * (l >> 4) + e] = y * a.inv_tau;
    }
  };
  auto flush = [&](int first, int end) {  // stages
    lds_barrier();
    const int tok0 = (run0 + first * TG) * 16, width = min(min(run0 + end * TG, run1) * 16, a.V) - tok0, quads = (width + 3) / 4;
    const int rows = min(ROWS, a.R - row0);
    for (int j = tid; j < rows * quads; j += kThreads) {
      const int row = j / quads, c = (j - row * quads) * 4;
      float* out = a.logits + (size_t)(row0 + row) * a.ld + tok0 + c;
      const floatx4 y = *reinterpret_cast<const floatx4*>(&s_out[row][c]);
      if (c + 4 <= width) {
        __builtin_nontemporal_store(y, reinterpret_cast<floatx4_any*>(out));
      } else {
        for (int i = 0; i < width - c; ++i) out[i] = y[i];
      }
    }
    lds_barrier();
  };

  for (int n = 0; n < stages; ++n) {
    // this stage's requests are the oldest; stores that are still under way only make the wait a longer one
    const int ahead = min(RING - 2, stages - 1 - n);
    if (ahead == 1) wait_newer<UPW + 1>();
    else wait_newer<0>();
    const int tok0 = (run0 + n * TG) * 16;
    if (tok0 + TG * 16 > a.V && (((a.V - tok0) * nb) & 3)) {  // the vocabulary's last scales are no whole word
      const int at = (a.V - tok0) * nb & ~3, bytes = (a.V - tok0) * nb & 3;
      if (tid == at / 4) {  // the thread whose request filled this word
        const uint8_t* from = a.scales + (size_t)tok0 * nb + at;
        s_scales[n % RING][tid] = from[0] | (bytes > 1 ? from[1] << 8 : 0) | (bytes > 2 ? from[2] << 16 : 0);
      }
    }
    lds_barrier();
    if (n + RING - 1 < stages) request(n + RING - 1);
    const int slot = n % RING, row = tg * 16 + i16;
    intx4 w[UPW];
    int sc[UPW];
#pragma unroll
    for (int u = 0; u < UPW; ++u) {  // a unit that this slice lacks, and blocks past the row: some codes, times h = 0, with a scale of one
      const int kb = min(4 * (u0 + u) + g, nb - 1), in = u < count && 4 * (u0 + u) + g < nb ? -1 : 0;
      w[u] = s_codes[slot][row * nb + (kb ^ (row & swap))];
      sc[u] = (reinterpret_cast<const uint8_t*>(s_scales[slot])[row * nb + kb] & in) | (127 & ~in);
    }
    floatx4 acc[MT] = {};
#pragma unroll
    for (int u = 0; u < UPW; ++u) {
      const float scale = __builtin_bit_cast(float, sc[u] << 23);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bf16x8 v = unpack8(w[u][q], scale);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int p = P - 1; p >= 0; --p) acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, h[u][q][p][m], acc[m], 0, 0, 0);
      }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) asm volatile("" : "+v"(acc[m]));  // no multiply moves under a condition
    if (KS == 1) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
        *reinterpret_cast<floatx4*>(&s_out[16 * m + i16][(n % per_flush * TG + tg) * 16 + 4 * g]) = acc[m] * a.inv_tau;
      if ((n + 1) % per_flush == 0 || n + 1 == stages) flush(n / per_flush * per_flush, n + 1);
    } else {
#pragma unroll
      for (int m = 0; m < MT; ++m) s_sum[n & 1][m][wave][lane] = acc[m];
      if (n) add_up(n - 1);
      if (n && n % per_flush == 0) flush(n - per_flush, n);
    }
  }
  if (KS > 1) {
    lds_barrier();
    add_up(stages - 1);
    flush((stages - 1) / per_flush * per_flush, stages);
  }
}

// Few slices mean few barriers and few partial sums, but every tile of a stage brings its copy of h into registers before the first
// multiply: one slice wherever h fits (8 rows of d = 512, V = 126464: 11.1 us, in two slices 13.1, in four 16.0), and of more
// slices the fewest that leave a workgroup eight stages (8 rows of d = 2048, V = 50257 in four slices, six stages: 15.9, in eight 14.7;
// 16 float32 rows, whose h is three times as long, of d = 1024, V = 32000 in two slices, two stages: 18.1, in eight 11.7), but no more
// slices than units of 128 columns, rounded up to a power of two (8 rows of d = 256, V = 32000 in two slices 5.8, in eight, six of them
// empty, 8.7; five to seven units in eight slices leave up to three of them empty).
template <int MT, bool F32>
bool launch_stages(const Mx4Args& a) {
  const int tiles = (a.V + 15) / 16, nu = (a.d + 127) / 128;
  if (nu > 4 * kWaves || a.d < 128 || a.R > 1 << 20) return false;  // a launch holds fewer than 2^32 threads
  // Rounds of a workgroup per CU, 32 per XCD: more of them leave fewer CUs without work where row blocks do not divide 32; the start of a
  // run (h, the first stages) costs about 16 tiles.  272 float32 rows of d = 4096, V = 50257, 17 row blocks: 346 us, in one round 523.
  const int row_blocks = (a.R + 16 * MT - 1) / (16 * MT), first = (row_blocks + 31) / 32;
  int runs = 0;
  long least = LONG_MAX;
  for (int r = first; r < first + 8; ++r) {
    const int n = std::min(tiles, 32 * r / row_blocks * 8);
    const long cost = r * ((tiles + n - 1) / n + 16L);
    if (cost < least) least = cost, runs = n;
  }
  int KS = 1;
  while (nu > 4 * KS || (KS < kWaves && KS < nu && tiles < (KS == 1 && !F32 ? 1 : 8) * runs * (kWaves / KS))) KS *= 2;
  const dim3 grid((runs + 7) / 8 * 8 * row_blocks);
  switch ((nu + KS - 1) / KS) {
    case 1: FEF_LAUNCH_HEAD((mx4_stages_kernel<1, MT, F32>), grid, dim3(kThreads), a, a, KS, runs, row_blocks); break;
    case 2: FEF_LAUNCH_HEAD((mx4_stages_kernel<2, MT, F32>), grid, dim3(kThreads), a, a, KS, runs, row_blocks); break;
    case 3: FEF_LAUNCH_HEAD((mx4_stages_kernel<3, MT, F32>), grid, dim3(kThreads), a, a, KS, runs, row_blocks); break;
    default: FEF_LAUNCH_HEAD((mx4_stages_kernel<4, MT, F32>), grid, dim3(kThreads), a, a, KS, runs, row_blocks); break;
  }
  return true;
}

__device__ __forceinline__ void request_2(const void* base, uint32_t offset, uint32_t lds_off) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_ushort %0, %1" :: "v"(offset), "s"(base), "s"(lds_off) : "memory");
}

// More rows: a workgroup takes a run of up to WC TT tiles times 16 M WR rows through steps of 128 columns.  Its eight wavefronts are WR
// groups of 16 M rows times WC = 8 / WR columns of tiles, wavefront column c with the tiles c, c + WC, ... of the run: codes become bf16
// where they are used, once for 16 M rows, and a fragment of h serves TT tiles.  All of it is requested straight into LDS: h, which L2
// holds, one step ahead by wavefronts 0 to 3, and whole 128-byte lines of codes, two steps at a time, up to four steps ahead by the others
// (requests of one wavefront complete in order, so one that had asked for both would wait for the far ones with the near ones).
// Bound: the multiplies.  512 rows of d = 3584, V = 151936: 488 to 515 us, 1.08 to 1.14 PFLOP/s, a plain bf16 product of 8192^3 1.22; the
// transfers alone take 313, the multiplies alone 382.  With fewer rows neither covers the other well, since the wavefronts meet at
// a barrier per step: 64 rows of d = 4096, V = 126464 91 us, transfers alone 75 (59 without h), multiplies alone 63, bytes 51.  h two
// steps ahead (93 to 95) or four tiles of tokens per wavefront with a single step of h in LDS (96) are no better.
template <int M, int WR, int TT, bool F32>
__global__ __launch_bounds__(kThreads, 2) void mx4_tile_kernel(Mx4Args a, int runs, int row_blocks) {
  constexpr int P = F32 ? 3 : 1, WC = 8 / WR, ROWS = 16 * M * WR, TOK = 16 * WC * TT, kElem = F32 ? 4 : 2;
  constexpr int HI = (ROWS * 8 * kElem + 255) / 256, CI = TOK / 32, SI = TOK / 64;  // requests per wavefront: h per step, codes and scales per pair
  constexpr int kH = HI * 4096, kC = TOK * 128, kS = TOK * 16, kOutLd = TOK + 4;
  constexpr int kFit = ((160 << 10) - 2 * kH) / (kC + kS), CR = kFit < 3 ? kFit : 3;  // pairs of steps in LDS; of h: two steps
  constexpr int kBytes = 2 * kH + CR * (kC + kS);
  static_assert(ROWS * kOutLd * 4 <= kBytes && CR >= 2 && TOK % 64 == 0, "");
  __shared__ __attribute__((aligned(16))) char smem[kBytes];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g = lane >> 4, wc = wave % WC, wr = wave / WC;
  const int asks_codes = wave >> 2, quarter = wave & 3;
  // Row blocks of a run go to one XCD one behind another.
  const int q = blockIdx.x >> 3, by = q % row_blocks, bx = q / row_blocks * 8 + (blockIdx.x & 7);
  if (bx >= runs) return;
  const int nb = a.d / 32, steps = (nb + 3) / 4, pairs = (nb + 7) / 8;
  const int tiles = (a.V + 15) / 16;
  const int t0 = (int)((long)bx * tiles / runs), t1 = (int)((long)(bx + 1) * tiles / runs);
  const int row0 = by * ROWS;
  const int last = min(t1 * 16, a.V) - 1 - t0 * 16;                    // last token there is, from the run's first

  // Where this lane's 16-byte pieces come from: request i fills the pieces (4 i + quarter) 64 + lane of its step or pair.
  constexpr int NI = HI > CI ? HI : CI;
  uint32_t off[NI], s_off[SI];
  auto piece_of = [&](int i) { return (i * 4 + quarter) * kWave + lane; };
  // Where a row's 16-byte chunks lie: exchanged by fold(row), so that 16 lanes which are served together, eight rows of one group g and
  // the other eight of the next, meet all banks (rows 0-3 and 12-15, and 4-11 of the next group).  Exchanged by the row itself, every read
  // took twice its cycles (64 rows of d = 4096, V = 126464: 94.8 us, so 91.1).
  auto fold = [](int row) { return (row ^ (F32 ? row >> 1 & 4 : row << 1 & 8)) & 15; };
  auto h_column = [&](int i) { const int s = piece_of(i); return (s & (8 * kElem - 1)) ^ fold(s / (8 * kElem)); };
  auto c_chunk = [&](int i) { const int s = piece_of(i); return (s & 7) ^ (s >> 4 & 7); };
  if (!asks_codes) {
#pragma unroll
    for (int i = 0; i < HI; ++i) off[i] = (uint32_t)min(piece_of(i) / (8 * kElem), a.R - 1 - row0) * (uint32_t)a.d * kElem + h_column(i) * 16;
  } else {
#pragma unroll
    for (int i = 0; i < CI; ++i) off[i] = (uint32_t)min(piece_of(i) >> 3, last) * (uint32_t)(a.d / 2) + c_chunk(i) * 16;
  }
#pragma unroll
  for (int i = 0; i < SI; ++i)  // 64 words: two scales, number `quarter` of the pair's four, of 64 tokens
    s_off[i] = (uint32_t)min(i * kWave + lane, last) * (uint32_t)nb + 2 * quarter;
  const char* h0 = (const char*)a.h + (size_t)row0 * a.d * kElem;
  const uint8_t* codes = a.codes + (size_t)t0 * 16 * (a.d / 2);
  const uint8_t* scales = a.scales + (size_t)t0 * 16 * nb;
  const uint32_t lds = lds_offset(smem);
  // What lies past the row is taken from its end and not used.
  auto request_h = [&](int step) {
    const uint32_t at = lds + (step & 1) * kH + quarter * 1024;
    const char* from = h0 + (size_t)step * 128 * kElem;
    const bool half = 4 * step + 4 > nb;
#pragma unroll
    for (int i = 0; i < HI; ++i) request_16(from, off[i] - (half && h_column(i) >= 4 * kElem ? 64 * kElem : 0), at + i * 4096);
  };
  auto request_c = [&](int pair) {
    const uint32_t at = lds + 2 * kH + pair % CR * (kC + kS);
    const uint8_t *c = codes + (size_t)pair * 128, *s = scales + (size_t)pair * 8;
    const int left = nb - 8 * pair;  // blocks of the row from the pair's first on
    if (left >= 8) {
#pragma unroll
      for (int i = 0; i < CI; ++i) request_16(c, off[i], at + quarter * 1024 + i * 4096);
#pragma unroll
      for (int i = 0; i < SI; ++i) request_2(s, s_off[i], at + kC + quarter * (TOK * 4) + i * 256);
    } else {
#pragma unroll
      for (int i = 0; i < CI; ++i) request_16(c, off[i] - max(c_chunk(i) - (left - 1), 0) * 16, at + quarter * 1024 + i * 4096);
#pragma unroll
      for (int i = 0; i < SI; ++i) request_2(s, s_off[i] - max(2 * quarter - (left - 2), 0), at + kC + quarter * (TOK * 4) + i * 256);
    }
  };
  if (!asks_codes) {
    request_h(0);
  } else {
#pragma unroll
    for (int n = 0; n < CR - 1; ++n)
      if (n < pairs) request_c(n);
  }

  // Fragments of eight columns per lane are read and converted under the multiplies of the eight before, the first of a step under the
  // last of the step before: those are multiplied behind the barrier.
  floatx4 acc[TT][M] = {};
  bf16x8 x[2][P][M] = {}, v[2][TT] = {};
  auto multiply = [&](int j) {
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int p = P - 1; p >= 0; --p) acc[t][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[j & 1][t], x[j & 1][p][m], acc[t][m], 0, 0, 0);
  };
  auto step = [&](int n, auto half) {
    if (!asks_codes) {
      wait_newer<0>();
    } else if (!(n & 1)) {  // later pairs may still be under way
      if (CR > 2 && n / 2 + 1 < pairs) wait_newer<CI + SI>();
      else wait_newer<0>();
    }
    lds_barrier();
    const bf16x8* s_h = reinterpret_cast<const bf16x8*>(smem + (n & 1) * kH);
    const char* at = smem + 2 * kH + n / 2 % CR * (kC + kS);
    const intx4* s_c = reinterpret_cast<const intx4*>(at);
    const int* s_s = reinterpret_cast<const int*>(at + kC) + (2 * (n & 1) + (g >> 1)) * TOK;
    const int keep = g < 2 ? -1 : 0;  // half a step: what its last two blocks hold is masked, without a branch in front of a multiply
    intx4 w[TT];
    int b[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int tok = (WC * t + wc) * 16 + i16;
      w[t] = s_c[tok * 8 + ((4 * (n & 1) + g) ^ (tok >> 1 & 7))];
      b[t] = s_s[tok];
    }
    floatx4 f[2][F32 ? M : 1];
    auto read_h = [&](int j) {
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const int row = (wr * M + m) * 16 + i16;
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            f[e][m] = reinterpret_cast<const floatx4*>(s_h)[row * 32 + ((8 * g + 2 * j + e) ^ fold(i16))];
            if (half) f[e][m] = __builtin_bit_cast(floatx4, __builtin_bit_cast(intx4, f[e][m]) & keep);
          }
        } else {
          x[j & 1][0][m] = s_h[row * 16 + ((4 * g + j) ^ fold(i16))];
          if (half) x[j & 1][0][m] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(intx4, x[j & 1][0][m]) & keep);
        }
      }
    };
    auto convert = [&](int j) {
      if constexpr (F32) {
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const float xs[8] = {f[0][m][0], f[0][m][1], f[0][m][2], f[0][m][3], f[1][m][0], f[1][m][1], f[1][m][2], f[1][m][3]};
          bf16x8 part[3];
          split3(xs, part);
#pragma unroll
          for (int p = 0; p < P; ++p) x[j & 1][p][m] = part[p];
        }
      }
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        int s = (b[t] >> (8 * (g & 1))) & 255;
        if (half) {
          if (j == 0) w[t] &= keep;
          s = (s & keep) | (127 & ~keep);
        }
        v[j & 1][t] = unpack8(w[t][j], __builtin_bit_cast(float, s << 23));
      }
    };
    read_h(0);
    multiply(3);
    if (!asks_codes) {
      if (n + 1 < steps) request_h(n + 1);
    } else if (!(n & 1) && n / 2 + CR - 1 < pairs) {
      request_c(n / 2 + CR - 1);
    }
    convert(0);
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      read_h(j + 1);
      if constexpr (!F32) convert(j + 1);
      multiply(j);
      if constexpr (F32) convert(j + 1);
    }
  };
  const int whole = nb / 4;
  for (int n = 0; n < whole; ++n) step(n, std::false_type{});
  if (whole < steps) step(whole, std::true_type{});
  multiply(3);
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int m = 0; m < M; ++m) asm volatile("" : "+v"(acc[t][m]));  // the multiplies need all lanes: none may move under a condition

  // Logits change places in LDS and leave row by row.
  lds_barrier();
  float* s_out = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int m = 0; m < M; ++m)
      *reinterpret_cast<floatx4*>(s_out + ((wr * M + m) * 16 + i16) * kOutLd + (WC * t + wc) * 16 + 4 * g) = acc[t][m] * a.inv_tau;
  lds_barrier();
  const int rows = min(ROWS, a.R - row0);
  for (int row = wave; row < rows; row += kWaves) {
    for (int c = lane * 4; c <= last; c += 4 * kWave) {
      float* out = a.logits + (size_t)(row0 + row) * a.ld + t0 * 16 + c;
      const floatx4 y = *reinterpret_cast<const floatx4*>(s_out + row * kOutLd + c);
      if (c + 3 <= last) {
        __builtin_nontemporal_store(y, reinterpret_cast<floatx4_any*>(out));
      } else {
        for (int i = 0; c + i <= last; ++i) out[i] = y[i];
      }
    }
  }
}

template <int M, int WR, bool F32>
void launch_tile(const Mx4Args& a) {
  constexpr int ROWS = 16 * M * WR, WC = 8 / WR, kMostTT = WR == 1 ? 3 : 4;
  const int row_blocks = (a.R + ROWS - 1) / ROWS;
  const long tiles = (a.V + 15) / 16, least = (tiles + WC * kMostTT - 1) / (WC * kMostTT);
  // As many runs as fill whole rounds of one workgroup per CU.
  const long rounds = (least * row_blocks + 255) / 256;
  long runs = rounds * 256 / row_blocks;
  if (runs < least) runs = least;
  if (runs > tiles) runs = tiles;
  const dim3 grid((unsigned)((runs + 7) / 8 * 8 * row_blocks));
  const int tt = (int)((tiles + runs - 1) / runs + WC - 1) / WC;
#define MX4_TILE(n) case n: FEF_LAUNCH_HEAD((mx4_tile_kernel<M, WR, n, F32>), grid, dim3(kThreads), a, a, (int)runs, row_blocks); break
  switch (tt) {
    MX4_TILE(1);
    MX4_TILE(2);
    default:
      if constexpr (kMostTT > 2) {
        switch (tt) {
          MX4_TILE(3);
          default:
            if constexpr (kMostTT > 3) switch (tt) { MX4_TILE(4); }
        }
      }
  }
#undef MX4_TILE
}

constexpr int kRowsPerWave = 64;

// Rows of d = 32 (2 n + 1) below 128 or above 4096: a wavefront per 16 tokens and 64 rows, straight from memory; grid (groups of 64 tokens,
// groups of 64 rows).  Bound: the latency of its loads, a step of 128 columns after another: 8 rows of d = 4128, V = 126464
// 352 us (of d = 4160 in tiles 84).  Sizes of models are not among them.
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

// float32 rows go through stages, 16 at a time: there h is split once per workgroup, in tiles before every use (us, stages and tiles; d =
// 4096, V = 50257: 96 rows 118, 251, 512 rows 527, 869; 32 rows of V = 126464 112, 163), unless the head is small and the runs so short that
// starting them tells (64 rows of d = 256, V = 50257 19.6, 15.0; 32 of d = 768, V = 50257 22.2, 18.9; 40 of d = 896, V = 20000 16.2, 26.1).
// bf16 rows go through stages up to 32; above them only where the vocabulary makes too few tiles for all CUs, so that slices of k are
// needed (64 rows of d = 4096, V = 8000 17.7, 26; 300 of d = 2048, V = 1000 10.4, 18.2; but 64 of V = 126464 105, 94; 512 of d = 1024,
// V = 8000 27.7, 13.7), and where d is no whole number of 64, which tiles do not do (64 rows of d = 1056, V = 50257 25.2; of 1024 14.5).
hipError_t launch_mx4(const Mx4Args& a) {
  const long rv = (long)a.R * a.V;
  const bool lines = a.d % 64 == 0;  // whole pairs of blocks, which tiles need
  if (a.f32) {
    const bool tiles = lines && a.R > 16 && a.d < 896 && a.V >= 16384 && rv < 1L << 22;
    if (!tiles && launch_stages<1, true>(a)) return hipGetLastError();
  } else {
    if (a.R <= 16 && launch_stages<1, false>(a)) return hipGetLastError();
    if ((a.R <= 32 || !lines || (a.V <= 8192 && rv <= 1L << 20)) && launch_stages<2, false>(a)) return hipGetLastError();
  }
  if (lines) {
    const int blocks = (a.R + 127) / 128, rows = (a.R + blocks - 1) / blocks;
    if (a.f32) {
      if (a.R <= 32) launch_tile<1, 2, true>(a);
      else launch_tile<2, 2, true>(a);
    } else if (rows <= 32) {
      launch_tile<2, 1, false>(a);
    } else if (rows <= 48) {
      launch_tile<3, 1, false>(a);
    } else if (rows <= 64) {
      launch_tile<4, 1, false>(a);
    } else if (rows <= 96) {
      launch_tile<3, 2, false>(a);
    } else {
      launch_tile<4, 2, false>(a);
    }
    return hipGetLastError();
  }
  const int groups = (a.R + kRowsPerWave - 1) / kRowsPerWave;
  const dim3 grid((a.V + 63) / 64, groups < 1024 ? groups : 1024);
  if (a.f32) FEF_LAUNCH_HEAD(mx4_kernel<true>, grid, dim3(256), a, a);
  else FEF_LAUNCH_HEAD(mx4_kernel<false>, grid, dim3(256), a, a);
  return hipGetLastError();
}

}  // namespace fef
