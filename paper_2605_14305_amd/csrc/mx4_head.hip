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
constexpr int kUnit = 256;  // columns per stage of h; two of them share a load of 16 scales

// 16 or 4 bytes per lane from base + offset straight to LDS, lane after lane from lds_off on; counted by hand (wait_newer).
__device__ __forceinline__ void request_16(const void* base, uint32_t offset, uint32_t lds_off) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(offset), "s"(base), "s"(lds_off) : "memory");
}
__device__ __forceinline__ void request_4(const void* base, uint32_t offset, uint32_t lds_off) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" :: "v"(offset), "s"(base), "s"(lds_off) : "memory");
}

typedef float floatx4_any __attribute__((ext_vector_type(4), aligned(4)));
struct __attribute__((packed, aligned(1))) Bytes16 { int v[4]; };

// The walk: a workgroup per CU takes a run of 16-token tiles, wavefront w the tiles w, w + 8, ... of up to 8 TT of them at a time, and walks
// over k in stages of 256 columns.  Codes come from memory straight into the registers that the conversion reads, a ring of up to 4 KB
// per tile ahead (the whole wait for HBM is hidden behind it); 128 bytes of a row at a time, a whole line.  h, which all wavefronts share,
// comes through LDS in two stages, 16-byte pieces exchanged so that 16 rows meet all banks.
// grid (runs, row blocks of 16 MT).
template <int TT, int MT, bool F32>
__global__ __launch_bounds__(kThreads, 2) void mx4_walk_kernel(Mx4Args a, int passes) {
  constexpr int DS = TT >= 3 ? 1 : TT == 2 ? 2 : 4;  // pairs of stages in the ring
  constexpr int P = F32 ? 3 : 1, ROWS = 16 * MT;
  __shared__ bf16x8 s_h[2][P][ROWS * (kUnit / 8)];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g = lane >> 4;
  const int nb = a.d / 32, nu = (nb + 7) / 8;
  const int tiles = (a.V + 15) / 16;
  const int run0 = (int)((long)blockIdx.x * tiles / gridDim.x), run1 = (int)((long)(blockIdx.x + 1) * tiles / gridDim.x);
  const int row0 = blockIdx.y * ROWS;
  // Addresses are a scalar pointer that moves and a 32-bit offset per lane that does not, which keeps them out of the vector registers.
  constexpr int kElem = F32 ? 4 : 2;
  const char* h0 = (const char*)a.h + (size_t)row0 * a.d * kElem;

  // h, stage u: thread -> pieces of eight columns
  uint32_t h_off[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int item = tid + i * kThreads;
    h_off[i] = (uint32_t)min(item >> 5, a.R - 1 - row0) * (uint32_t)a.d * kElem + (item & 31) * 8 * kElem;
  }
  float xf[F32 ? MT : 1][8];
  bf16x8 xb[F32 ? 1 : MT];
  auto fetch_h = [&](int u) {
    const char* at = h0 + (size_t)u * kUnit * kElem;
    const bool in = u * kUnit + (tid & 31) * 8 < a.d;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      if constexpr (F32) {
        floatx4 lo = {}, hi = {};
        if (in) {
          lo = *reinterpret_cast<const floatx4*>(at + h_off[i]);
          hi = *reinterpret_cast<const floatx4*>(at + h_off[i] + 16);
        }
        *reinterpret_cast<floatx4*>(xf[i]) = lo;
        *reinterpret_cast<floatx4*>(xf[i] + 4) = hi;
      } else {
        xb[i] = bf16x8{};
        if (in) xb[i] = *reinterpret_cast<const bf16x8*>(at + h_off[i]);
      }
    }
  };
  auto store_h = [&](int buf) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int item = tid + i * kThreads, row = item >> 5, slot = row * 32 + ((item & 31) ^ (row & 15));
      if constexpr (F32) {
        bf16x8 part[3];
        split3(xf[i], part);
#pragma unroll
        for (int p = 0; p < 3; ++p) s_h[buf][p][slot] = part[p];
      } else {
        s_h[buf][0][slot] = xb[i];
      }
    }
  };

  for (int pass = 0; pass < passes; ++pass) {
    const int t0 = run0 + (int)((long)pass * (run1 - run0) / passes), t1 = run0 + (int)((long)(pass + 1) * (run1 - run0) / passes);
    intx4 w[DS][2][TT][2];
    intx4 sc[DS][TT];
    const uint8_t *codes[TT], *scales[TT];
    uint32_t code_off[TT], scale_off[TT];
    // the runs' lengths differ by one tile at most, so a wavefront has TT of them or TT - 1
    const bool full = t0 + wave + (TT - 1) * kWaves < t1;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int tok0 = min(t0 + wave + t * kWaves, t1 - 1) * 16;
      const uint32_t r = min(i16, a.V - 1 - tok0);
      codes[t] = a.codes + (size_t)tok0 * (a.d / 2);
      scales[t] = a.scales + (size_t)tok0 * nb;
      code_off[t] = r * (uint32_t)(a.d / 2);
      scale_off[t] = r * (uint32_t)nb;
    }
    // codes of half a pair of stages, scales of a whole one; blocks past the row: its last codes, times h = 0, with a scale of one
    auto fetch_codes = [&](int slot, int half, int pair) {
      const int kb = 16 * pair + 8 * half;
      if (kb + 8 <= nb) {
#pragma unroll
        for (int t = 0; t < TT; ++t)
          if (t < TT - 1 || full) {
            const uint8_t* at = codes[t] + (size_t)kb * 16;
            w[slot][half][t][0] = *reinterpret_cast<const intx4*>(at + (code_off[t] + g * 16));
            w[slot][half][t][1] = *reinterpret_cast<const intx4*>(at + (code_off[t] + g * 16) + 64);
          }
      } else {
#pragma unroll
        for (int t = 0; t < TT; ++t)
          if (t < TT - 1 || full) {
            w[slot][half][t][0] = *reinterpret_cast<const intx4*>(codes[t] + (code_off[t] + min(kb + g, nb - 1) * 16));
            w[slot][half][t][1] = *reinterpret_cast<const intx4*>(codes[t] + (code_off[t] + min(kb + 4 + g, nb - 1) * 16));
          }
      }
    };
    auto fetch_scales = [&](int slot, int pair) {
      if (16 * pair + 16 <= nb) {
#pragma unroll
        for (int t = 0; t < TT; ++t)
          if (t < TT - 1 || full) sc[slot][t] = __builtin_bit_cast(intx4, *reinterpret_cast<const Bytes16*>(scales[t] + 16 * pair + scale_off[t]));
      } else {
#pragma unroll
        for (int t = 0; t < TT; ++t)
          if (t < TT - 1 || full) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int kb = 16 * pair + 4 * q + g;
              sc[slot][t][q] = (kb < nb ? (int)scales[t][scale_off[t] + min(kb, nb - 1)] : 127) << (8 * g);
            }
          }
      }
    };

    floatx4 acc[TT][MT] = {};
    fetch_h(0);
#pragma unroll
    for (int s = 0; s < DS; ++s) {
      if (2 * s < nu) {
        fetch_scales(s, s);
        fetch_codes(s, 0, s);
      }
      if (2 * s + 1 < nu) fetch_codes(s, 1, s);
    }
    if (pass) lds_barrier();  // the last stage of the pass before has been read
    store_h(0);
    lds_barrier();
    for (int pair0 = 0; 2 * pair0 < nu; pair0 += DS) {
#pragma unroll
      for (int s = 0; s < DS; ++s) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int pair = pair0 + s, u = 2 * pair + half;
          if (u < nu) {
            if (u + 1 < nu) fetch_h(u + 1);
            // eight multiplies' worth of columns per lane and stage; fragments of h are read one step ahead
            bf16x8 x[2][P][MT];
            auto read_h = [&](int step) {
              const int piece = (16 * (step >> 2) + 4 * g + (step & 3)) ^ i16;
#pragma unroll
              for (int p = 0; p < P; ++p)
#pragma unroll
                for (int m = 0; m < MT; ++m) x[step & 1][p][m] = s_h[half][p][(16 * m + i16) * 32 + piece];
            };
            read_h(0);
            float scale[TT];
#pragma unroll
            for (int step = 0; step < 8; ++step) {
              if (step + 1 < 8) read_h(step + 1);
#pragma unroll
              for (int t = 0; t < TT; ++t)
                if (t < TT - 1 || full) {
                  if ((step & 3) == 0)
                    scale[t] = __builtin_bit_cast(float, __builtin_amdgcn_ubfe((unsigned)sc[s][t][2 * half + (step >> 2)], 8 * g, 8) << 23);
                  const bf16x8 v = unpack8(w[s][half][t][step >> 2][step & 3], scale[t]);
#pragma unroll
                  for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int p = P - 1; p >= 0; --p) acc[t][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, x[step & 1][p][m], acc[t][m], 0, 0, 0);
                }
              __builtin_amdgcn_sched_barrier(0);  // else all fragments of a stage are read at its start, into registers that the ring needs
            }
            if (u + 2 * DS < nu) {
              if (half == 0) fetch_codes(s, 0, pair + DS);
              else fetch_codes(s, 1, pair + DS);
            }
            if (half == 1 && u + 2 * DS - 1 < nu) fetch_scales(s, pair + DS);
            if (u + 1 < nu) store_h(half ^ 1);
            lds_barrier();
          }
        }
      }
    }
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        asm volatile("" : "+v"(acc[t][m]));  // the multiplies need all lanes: none may move under a condition
        const int row = row0 + 16 * m + i16, tok = (t0 + wave + t * kWaves) * 16 + 4 * g;
        if ((t < TT - 1 || full) && row < a.R) {
          float* out = a.logits + (size_t)row * a.ld + tok;
          const floatx4 y = acc[t][m] * a.inv_tau;
          if (tok + 4 <= a.V) {
            *reinterpret_cast<Float4*>(out) = Float4{{y[0], y[1], y[2], y[3]}};
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (tok + i < a.V) out[i] = y[i];
          }
        }
      }
  }
}

template <int TT, int MT, bool F32>
void launch_walk(const Mx4Args& a, int runs, int passes) {
  const dim3 grid(runs, (a.R + 16 * MT - 1) / (16 * MT));
  FEF_LAUNCH_HEAD((mx4_walk_kernel<TT, MT, F32>), grid, dim3(kThreads), a, a, passes);
}

template <int MT, bool F32>
void launch_walk_of(const Mx4Args& a) {
  const int tiles = (a.V + 15) / 16, runs = tiles < 256 ? tiles : 256;
  const int longest = (tiles + runs - 1) / runs;
  const int passes = (longest + 8 * 5 - 1) / (8 * 5);
  const int tt = ((longest + passes - 1) / passes + 7) / 8;
  switch (tt) {
    case 1: launch_walk<1, MT, F32>(a, runs, passes); break;
    case 2: launch_walk<2, MT, F32>(a, runs, passes); break;
    case 3: launch_walk<3, MT, F32>(a, runs, passes); break;
    case 4: launch_walk<4, MT, F32>(a, runs, passes); break;
    default: launch_walk<5, MT, F32>(a, runs, passes); break;
  }
}


// Up to 16 MT rows whose h fits the registers.  A workgroup per CU takes a run of 16-token tiles in stages of TG of them, up to 32 KB of
// codes and 2 KB of scales, which come in the order of memory straight into LDS, RING - 1 stages ahead.  Its eight wavefronts are KS slices of
// k times TG = 8 / KS tiles: a wavefront holds its slice of h as operands for the whole kernel (UPW units of 128 columns) and multiplies
// its codes of each stage with it; the KS partial sums of a tile meet in LDS and are added in the order of the slices by one
// wavefront, in turn, while the next stage is multiplied.  One barrier per stage.
// LDS holds a stage's rows one behind another, their 16-byte chunks exchanged within 256 bytes (chunk ^ row, as far as the row length allows) so that
// 16 rows meet all banks.
template <int UPW, int MT, bool F32>
__global__ __launch_bounds__(kThreads, 2) void mx4_stages_kernel(Mx4Args a, int KS) {
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
  const int run0 = (int)((long)blockIdx.x * tiles / gridDim.x), run1 = (int)((long)(blockIdx.x + 1) * tiles / gridDim.x);
  const int stages = (run1 - run0 + TG - 1) / TG;
  const int row0 = blockIdx.y * ROWS;

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
    if (tok0 + TG * 16 > a.V && (((a.V - tok0) * nb) & 3)) {  // an odd vocabulary, rows of 2 + 4 n scales: the last two
      const int at = (a.V - tok0) * nb - 2;
      if (tid == at / 4) {  // the thread whose request filled this word
        const uint8_t* from = a.scales + (size_t)tok0 * nb + at;
        s_scales[n % RING][tid] = from[0] | from[1] << 8;
      }
    }
    lds_barrier();
    if (n + RING - 1 < stages) request(n + RING - 1);
    const int slot = n % RING, row = tg * 16 + i16;
    intx4 w[UPW];
    int sc[UPW];
#pragma unroll
    for (int u = 0; u < UPW; ++u)
      if (u < UPW - 1 || count == UPW) {
        const int kb = min(4 * (u0 + u) + g, nb - 1);
        w[u] = s_codes[slot][row * nb + (kb ^ (row & swap))];
        sc[u] = 4 * (u0 + u) + g < nb ? reinterpret_cast<const uint8_t*>(s_scales[slot])[row * nb + kb] : 127;
      }
    floatx4 acc[MT] = {};
#pragma unroll
    for (int u = 0; u < UPW; ++u)
      if (u < UPW - 1 || count == UPW) {
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
// 16 float32 rows, whose h is three times as long, of d = 1024, V = 32000 in two slices, two stages: 18.1, in eight 11.7).
template <int MT, bool F32>
bool launch_stages(const Mx4Args& a) {
  const int tiles = (a.V + 15) / 16, nu = (a.d + 127) / 128;
  if (nu > 4 * kWaves || a.d % 64 || a.d < 128) return false;
  int KS = 1;
  while (nu > 4 * KS || (KS < kWaves && tiles < (KS == 1 && !F32 ? 1 : 8) * 256 * (kWaves / KS))) KS *= 2;
  const dim3 grid(tiles < 256 ? tiles : 256, (a.R + 16 * MT - 1) / (16 * MT));
  switch ((nu + KS - 1) / KS) {
    case 1: FEF_LAUNCH_HEAD((mx4_stages_kernel<1, MT, F32>), grid, dim3(kThreads), a, a, KS); break;
    case 2: FEF_LAUNCH_HEAD((mx4_stages_kernel<2, MT, F32>), grid, dim3(kThreads), a, a, KS); break;
    case 3: FEF_LAUNCH_HEAD((mx4_stages_kernel<3, MT, F32>), grid, dim3(kThreads), a, a, KS); break;
    default: FEF_LAUNCH_HEAD((mx4_stages_kernel<4, MT, F32>), grid, dim3(kThreads), a, a, KS); break;
  }
  return true;
}

}  // namespace

hipError_t launch_mx4(const Mx4Args& a) {
  if (a.f32) {
    if (a.R <= 16 && launch_stages<1, true>(a)) {}
    else if (a.R <= 16) launch_walk_of<1, true>(a);
    else launch_walk_of<2, true>(a);
  } else {
    if (a.R <= 16 && launch_stages<1, false>(a)) {}
    else if (a.R <= 32 && launch_stages<2, false>(a)) {}
    else if (a.R <= 16) launch_walk_of<1, false>(a);
    else if (a.R <= 32) launch_walk_of<2, false>(a);
    else if (a.R <= 48) launch_walk_of<3, false>(a);
    else launch_walk_of<4, false>(a);
  }
  return hipGetLastError();
}

}  // namespace fef
