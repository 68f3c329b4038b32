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

}  // namespace

hipError_t launch_mx4(const Mx4Args& a) {
  if (a.f32) {
    if (a.R <= 16) launch_walk_of<1, true>(a);
    else launch_walk_of<2, true>(a);
  } else {
    if (a.R <= 16) launch_walk_of<1, false>(a);
    else if (a.R <= 32) launch_walk_of<2, false>(a);
    else if (a.R <= 48) launch_walk_of<3, false>(a);
    else launch_walk_of<4, false>(a);
  }
  return hipGetLastError();
}

}  // namespace fef
