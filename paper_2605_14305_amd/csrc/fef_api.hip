// C ABI of the verify-step library: argument validation, workspace layout, kernel sequencing.
// Everything is validated on the host before the first launch; nothing is allocated.
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <memory>
#include <new>

#include "../../include/fef.h"
#include "fef_device.hpp"
#include "head_rules.hpp"

// Scratch of fef_verify_step_static: one copy per GPU the library runs on, held until the process
// ends.  In host code this name is only a handle for hipGetSymbolAddress; the device address it
// yields (one per device) is what kernels, memsets and copies must be given.
static __device__ __align__(256) unsigned char scratch[FEF_STATIC_SCRATCH_BYTES];

namespace {

thread_local char g_err[512] = "";

fef_status fail(fef_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return s;
}

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

struct Layout {
  int variant, nT, tile_unit, tile_T, nRC, all_slots;
  long ldl;
  size_t off_logits, off_partials, off_lse, off_xdraft, off_xtarget, off_slot_pos, off_window, off_seqstate,
      off_rmass, off_amass, total;
};

// Row counts and sizes of the two variants whose workgroups take runs of tokens.
bool stream_supports(long M, int d) { return M <= 128 && d % 64 == 0; }
bool rowstream_supports(long M, int d) { return M > 0 && M <= 128 && d % 512 == 0; }
int run_unit(int variant) { return variant == FEF_GEMM_STREAM ? 64 : variant == FEF_GEMM_ROWSTREAM ? 16 : 0; }

// Sizes only; no pointer checks.
fef_status check_sizes(const fef_params* p, int32_t K, int32_t block) {
  if (!p) return fail(FEF_ERR_INVALID_ARG, "params is NULL");
  if (p->struct_size != sizeof(fef_params))
    return fail(FEF_ERR_INVALID_ARG, "struct_size %u does not match this library's %zu",
                p->struct_size, sizeof(fef_params));
  if (p->B < 1 || p->d < 1 || p->V < 1)
    return fail(FEF_ERR_INVALID_ARG, "B, d, V must be >= 1 (got %d, %d, %d)", p->B, p->d, p->V);
  if (K < 1 || K > FEF_MAX_K || block < 1 || block > FEF_MAX_BLOCK || K > block)
    return fail(FEF_ERR_INVALID_ARG, "need 1 <= K <= min(block, %d) and block <= %d (got K=%d, block=%d)",
                FEF_MAX_K, FEF_MAX_BLOCK, K, block);
  if (p->dtype != FEF_BF16 && p->dtype != FEF_F32)
    return fail(FEF_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
  if (!(p->temperature > 0.f) || !(p->temperature < 1e30f))
    return fail(FEF_ERR_INVALID_ARG, "temperature must be a positive finite number");
  if (p->dtype == FEF_BF16 && p->d % 64 != 0)
    return fail(FEF_ERR_INVALID_ARG, "bf16 path needs d to be a multiple of 64 (got %d)", p->d);
  if ((long)p->B * K > (1L << 24))
    return fail(FEF_ERR_INVALID_ARG, "B*K = %ld exceeds 2^24 rows per call", (long)p->B * K);
  if (p->lowconf_scope != 0 && p->lowconf_scope != 1)
    return fail(FEF_ERR_INVALID_ARG, "lowconf_scope must be 0 or 1");
  if (p->greedy != 0 && p->greedy != 1) return fail(FEF_ERR_INVALID_ARG, "greedy must be 0 or 1");
  if (!(p->recorrupt_prob > 0.f && p->recorrupt_prob <= 1.f))
    return fail(FEF_ERR_INVALID_ARG, "recorrupt_prob must lie in (0, 1]");
  if (p->phase != FEF_PHASE_FUSED && p->phase != FEF_PHASE_DRAFT && p->phase != FEF_PHASE_TARGET)
    return fail(FEF_ERR_INVALID_ARG, "unknown phase %d", p->phase);
  if (p->seq_pass && p->n_pass < 1)
    return fail(FEF_ERR_INVALID_ARG, "seq_pass needs n_pass >= 1 (got %d)", p->n_pass);
  if (!p->conf && (p->pass_mask || p->lowconf_scope == 1))
    return fail(FEF_ERR_INVALID_ARG, "conf may be NULL only with pass_mask NULL and lowconf_scope 0");
  return FEF_OK;
}

fef_status select_variant(const fef_params* p, int32_t K, int* variant) {
  const long M = (p->phase == FEF_PHASE_FUSED ? 2L : 1L) * p->B * K;  // rows through the head in this call
  int v = p->gemm_variant;
  if (v == FEF_GEMM_AUTO) {
    if (p->dtype == FEF_F32) v = FEF_GEMM_F32;
    else if (fef::skinny_supports((int)(M > 1 << 20 ? 1 << 20 : M), p->d)) v = FEF_GEMM_SKINNY;
    else if (M > 128) v = FEF_GEMM_TILED256;
    else if (!rowstream_supports(M, p->d)) v = FEF_GEMM_STREAM;
    else if (M <= 48 || (M > 64 && M <= 96)) {
      v = FEF_GEMM_ROWSTREAM;  // two orders of the sums (see fef.h); which one AUTO gives is part of the interface
    } else {
      v = FEF_GEMM_STREAM;
    }
  }
  switch (v) {
    case FEF_GEMM_SKINNY:
      if (p->dtype != FEF_BF16 || !fef::skinny_supports((int)(M > 1 << 20 ? 1 << 20 : M), p->d))
        return fail(FEF_ERR_UNSUPPORTED, "skinny head kernel needs bf16, at most 32 rows through the head and d in {512, 1024, 2048, 2560, 3072, 3584, 4096}");
      break;
    case FEF_GEMM_TILED:
    case FEF_GEMM_TILED256:
      if (p->dtype != FEF_BF16) return fail(FEF_ERR_UNSUPPORTED, "tiled head kernels are bf16 only");
      break;
    case FEF_GEMM_STREAM:
      if (p->dtype != FEF_BF16 || !stream_supports(M, p->d))
        return fail(FEF_ERR_UNSUPPORTED, "the STREAM variant needs bf16 and at most 128 rows through the head");
      break;
    case FEF_GEMM_ROWSTREAM:
      if (p->dtype != FEF_BF16 || !rowstream_supports(M, p->d))
        return fail(FEF_ERR_UNSUPPORTED, "the ROWSTREAM variant needs bf16, at most 128 rows through the head and d a multiple of 512");
      break;
    case FEF_GEMM_F32:
      if (p->dtype != FEF_F32) return fail(FEF_ERR_UNSUPPORTED, "f32 head kernel needs dtype f32");
      if (M > 65535) return fail(FEF_ERR_UNSUPPORTED, "f32 head kernel serves at most 65535 rows");
      break;
    default:
      return fail(FEF_ERR_INVALID_ARG, "unknown gemm_variant %d", v);
  }
  *variant = v;
  return FEF_OK;
}

fef_status make_layout(const fef_params* p, int32_t K, int32_t block, Layout* L) {
  fef_status s = check_sizes(p, K, block);
  if (s != FEF_OK) return s;
  s = select_variant(p, K, &L->variant);
  if (s != FEF_OK) return s;
  const size_t BK = (size_t)p->B * K, M = 2 * BK;
  if (L->variant == FEF_GEMM_SKINNY) {
    // one partial per (row, workgroup); a workgroup's tokens are a contiguous run of 16-token tiles
    L->tile_unit = fef::kSkinnyUnit;
    L->tile_T = (p->V + fef::kSkinnyUnit - 1) / fef::kSkinnyUnit;
    L->nT = L->tile_T < fef::kSkinnyMaxGrid ? L->tile_T : fef::kSkinnyMaxGrid;
  } else if (const int unit = run_unit(L->variant)) {
    // one partial per (row, workgroup); a workgroup's tokens are a contiguous run of units
    L->tile_unit = unit;
    L->tile_T = (p->V + unit - 1) / unit;
    L->nT = fef::runs_grid(p->V, unit);
  } else if (L->variant == FEF_GEMM_TILED256) {
    // one partial per (row, workgroup tile of 256 tokens)
    L->tile_unit = fef::kTiled256Tn;
    L->tile_T = L->nT = (p->V + fef::kTiled256Tn - 1) / fef::kTiled256Tn;
  } else {
    L->tile_unit = fef::kTiledTn;
    L->tile_T = L->nT = (p->V + fef::kTiledTn - 1) / fef::kTiledTn;
  }
  L->nRC = (p->V + fef::kResidChunk - 1) / fef::kResidChunk;
  L->ldl = (long)align_up((size_t)p->V, 64);
  L->all_slots = (p->diag_alpha || p->diag_resid_mass) ? 1 : 0;
  const size_t nslots = L->all_slots ? BK : (size_t)p->B;
  size_t o = 0;
  auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, 256); return at; };
  L->off_logits = take(M * (size_t)L->ldl * sizeof(float));
  L->off_partials = take(M * (size_t)L->nT * sizeof(float2));
  L->off_lse = take(M * sizeof(float));
  L->off_xdraft = take(BK * sizeof(int32_t));
  L->off_xtarget = take(BK * sizeof(int32_t));
  L->off_slot_pos = take(BK * sizeof(int32_t));
  L->off_window = take((size_t)p->B * sizeof(int32_t));
  L->off_seqstate = take((size_t)p->B * sizeof(fef::SeqState));
  L->off_rmass = take(nslots * (size_t)L->nRC * sizeof(float));
  L->off_amass = take(L->all_slots ? nslots * (size_t)L->nRC * sizeof(float) : 0);
  L->total = o;
  return FEF_OK;
}

// The workspace of a call that brings its logits: all but the first area.
void drop_logits(Layout* L) {
  const size_t less = L->off_partials;
  for (size_t* o : {&L->off_partials, &L->off_lse, &L->off_xdraft, &L->off_xtarget, &L->off_slot_pos, &L->off_window, &L->off_seqstate,
                    &L->off_rmass, &L->off_amass, &L->total})
    *o -= less;
}

__global__ __launch_bounds__(256) void copy_probe_kernel(uint4* __restrict__ dst, const uint4* __restrict__ src,
                                                        size_t n16) {
  for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < n16; i += (size_t)gridDim.x * blockDim.x)
    dst[i] = src[i];
}

// The fastest read of a large buffer found on this machine, which is what the probe is for: the
// buffer as blocks of 16 rows of 8 KB (the shape of a 16-token tile of W at d = 4096); one workgroup
// per CU walks a contiguous run of blocks; its eight wavefronts split a row eight ways, and a
// wavefront fetches its 1 KB of each of the 16 rows in two bursts of eight 16-byte loads per lane
// (16 rows x 64 bytes per load), the last 64 bytes of a burst first, the next burst requested before
// the one in hand is consumed and waited for in full before anything else is asked for.  6.6 TB/s
// on 1 GB; a linear sweep with eight loads per thread in flight reaches 6.1 to 6.2.  What does not
// fill a block is swept linearly.
__global__ __launch_bounds__(512) void read_probe_kernel(const char* __restrict__ src, size_t nbytes, unsigned* sink) {
  constexpr size_t kBlock = 16 * 8192;
  const size_t nblocks = nbytes / kBlock;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i16 = lane & 15, g = lane >> 4;
  const size_t b0 = blockIdx.x * nblocks / gridDim.x, b1 = (blockIdx.x + 1) * nblocks / gridDim.x;
  const size_t nburst = 2 * (b1 - b0);
  uint4 acc = {0u, 0u, 0u, 0u};
  auto burst = [&](size_t j, uint4(&v)[8]) {
    const char* p = src + (b0 + (j >> 1)) * kBlock + (size_t)i16 * 8192 + wave * 1024 + g * 16 + (j & 1) * 512;
    v[7] = *reinterpret_cast<const uint4*>(p + 448);
    asm volatile("" ::: "memory");
#pragma unroll
    for (int u = 0; u < 7; ++u) {
      v[u] = *reinterpret_cast<const uint4*>(p + 64 * u);
      asm volatile("" ::: "memory");
    }
  };
  uint4 cur[8], nxt[8];
  if (nburst) burst(0, cur);
  for (size_t j = 0; j < nburst; ++j) {
    burst(j + 1 < nburst ? j + 1 : j, nxt);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      acc.x ^= cur[u].x; acc.y ^= cur[u].y; acc.z ^= cur[u].z; acc.w ^= cur[u].w;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) cur[u] = nxt[u];
  }
  const uint4* tail = reinterpret_cast<const uint4*>(src + nblocks * kBlock);
  const size_t ntail = (nbytes - nblocks * kBlock) / 16;
  for (size_t i = (size_t)blockIdx.x * 512 + threadIdx.x; i < ntail; i += (size_t)gridDim.x * 512) {
    const uint4 v = tail[i];
    acc.x ^= v.x; acc.y ^= v.y; acc.z ^= v.z; acc.w ^= v.w;
  }
  if ((acc.x ^ acc.y ^ acc.z ^ acc.w) == 0x9E3779B9u) *sink = 1u;
}

}  // namespace

extern "C" {

fef_status fef_read_probe(const void* src, size_t nbytes, void* sink, void* stream) {
  if (!src || !sink || nbytes == 0 || nbytes % 16 || ((uintptr_t)src & 15) || ((uintptr_t)sink & 3))
    return fail(FEF_ERR_INVALID_ARG, "read probe needs a non-NULL 16-byte aligned source, a size multiple of 16 and a sink");
  hipLaunchKernelGGL(read_probe_kernel, dim3(256), dim3(512), 0, (hipStream_t)stream, (const char*)src, nbytes,
                     (unsigned*)sink);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FEF_ERR_HIP, "read probe launch: %s", hipGetErrorString(e));
  return FEF_OK;
}

fef_status fef_copy_probe(void* dst, const void* src, size_t nbytes, void* stream) {
  if (!dst || !src || nbytes == 0 || nbytes % 16 || (((uintptr_t)dst | (uintptr_t)src) & 15))
    return fail(FEF_ERR_INVALID_ARG, "copy probe needs non-NULL 16-byte aligned pointers and a size multiple of 16");
  hipLaunchKernelGGL(copy_probe_kernel, dim3(2048), dim3(256), 0, (hipStream_t)stream, (uint4*)dst,
                     (const uint4*)src, nbytes / 16);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FEF_ERR_HIP, "copy probe launch: %s", hipGetErrorString(e));
  return FEF_OK;
}

size_t fef_workspace_bytes(const fef_params* prm, int32_t K, int32_t block) {
  Layout L;
  if (make_layout(prm, K, block, &L) != FEF_OK) return 0;
  // The halves of a split round share one workspace and may run another kernel than the whole round, with more partials
  // per row: the size serves them all.
  size_t need = L.total;
  fef_params p = *prm;
  for (p.phase = FEF_PHASE_FUSED; p.phase <= FEF_PHASE_TARGET; ++p.phase)
    if (make_layout(&p, K, block, &L) == FEF_OK && L.total > need) need = L.total;
  return need;
}

int32_t fef_select_gemm(const fef_params* prm, int32_t K) {
  fef_status s = check_sizes(prm, K, K > 0 ? (K > FEF_MAX_BLOCK ? FEF_MAX_BLOCK : K) : 1);
  if (s != FEF_OK) return s;
  int v = 0;
  s = select_variant(prm, K, &v);
  return s != FEF_OK ? (int32_t)s : v;
}

namespace {
constexpr int kPhaseTopN = 3;  // internal: draft rows only, then the baseline's top-n selection
fef_status run_step(const fef_params* prm, int phase, int n_transfer, const void* h_draft, const void* h_target,
                    const void* W_vocab, int32_t K, int32_t block, uint64_t seed, int32_t* out_tokens,
                    int32_t* out_accept_len, uint8_t* out_remask, void* workspace, size_t workspace_bytes,
                    const float* given = nullptr, long given_ld = 0);
}  // namespace

fef_status fef_verify_step(const fef_params* prm, const void* h_draft, const void* h_target,
                           const void* W_vocab, int32_t K, int32_t block, uint64_t seed,
                           int32_t* out_tokens, int32_t* out_accept_len, uint8_t* out_remask) {
  if (!prm) return fail(FEF_ERR_INVALID_ARG, "params is NULL");
  return run_step(prm, prm->phase, 0, h_draft, h_target, W_vocab, K, block, seed, out_tokens, out_accept_len,
                  out_remask, prm->workspace, prm->workspace_bytes);
}

namespace {
constexpr int kMaxDevices = 64;
std::atomic<void*> g_scratch_ptr[kMaxDevices];  // device address of `scratch` per device, NULL = not asked yet

// Address of this device's copy of `scratch`; resolved once per device with that device current.
fef_status static_scratch(void** out) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail(FEF_ERR_HIP, "hipGetDevice: %s", hipGetErrorString(e));
  if (dev < 0 || dev >= kMaxDevices) return fail(FEF_ERR_UNSUPPORTED, "device index %d out of range", dev);
  void* ptr = g_scratch_ptr[dev].load(std::memory_order_acquire);
  if (!ptr) {
    e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
    if (e != hipSuccess || !ptr)
      return fail(FEF_ERR_HIP, "hipGetSymbolAddress(scratch) on device %d: %s", dev, hipGetErrorString(e));
    g_scratch_ptr[dev].store(ptr, std::memory_order_release);  // concurrent first calls store the same address
  }
  *out = ptr;
  return FEF_OK;
}
}  // namespace

fef_status fef_verify_step_static(const fef_params* prm, const void* h_draft, const void* h_target,
                                  const void* W_vocab, int32_t K, int32_t block, uint64_t seed,
                                  int32_t* out_tokens, int32_t* out_accept_len, uint8_t* out_remask) {
  if (!prm) return fail(FEF_ERR_INVALID_ARG, "params is NULL");
  Layout L;
  fef_status s = make_layout(prm, K, block, &L);
  if (s != FEF_OK) return s;
  if (L.total > (size_t)FEF_STATIC_SCRATCH_BYTES)
    return fail(FEF_ERR_WORKSPACE, "this call needs %zu bytes of scratch, the built-in buffer has %zu: use fef_verify_step "
                "with a caller workspace", L.total, (size_t)FEF_STATIC_SCRATCH_BYTES);
  void* ptr = nullptr;
  s = static_scratch(&ptr);
  if (s != FEF_OK) return s;
  return run_step(prm, prm->phase, 0, h_draft, h_target, W_vocab, K, block, seed, out_tokens, out_accept_len,
                  out_remask, ptr, (size_t)FEF_STATIC_SCRATCH_BYTES);
}

fef_status fef_topn_step(const fef_params* prm, const void* h, const void* W_vocab, int32_t K, int32_t block,
                         uint64_t seed, int32_t n_transfer, int32_t* out_tokens, int32_t* out_committed,
                         uint8_t* out_remask) {
  if (!prm) return fail(FEF_ERR_INVALID_ARG, "params is NULL");
  if (n_transfer < 1) return fail(FEF_ERR_INVALID_ARG, "n_transfer must be at least 1 (got %d)", n_transfer);
  if (prm->phase != FEF_PHASE_FUSED) return fail(FEF_ERR_INVALID_ARG, "phase must be FUSED (0) in a baseline step");
  if (prm->draft_tokens || prm->pass_mask || prm->seq_pass || prm->seq_rounds)
    return fail(FEF_ERR_INVALID_ARG, "draft_tokens, pass_mask, seq_pass and seq_rounds have no meaning in a baseline step");
  fef_params p = *prm;
  p.phase = FEF_PHASE_DRAFT;  // sizes, kernel choice and workspace layout of a call over B*K rows
  return run_step(&p, kPhaseTopN, n_transfer, h, nullptr, W_vocab, K, block, seed, out_tokens, out_committed,
                  out_remask, p.workspace, p.workspace_bytes);
}

namespace {
fef_status run_step(const fef_params* prm, int phase, int n_transfer, const void* h_draft, const void* h_target,
                    const void* W_vocab, int32_t K, int32_t block, uint64_t seed, int32_t* out_tokens,
                    int32_t* out_accept_len, uint8_t* out_remask, void* workspace, size_t workspace_bytes,
                    const float* given, long given_ld) {
  Layout L;
  fef_status s = make_layout(prm, K, block, &L);
  if (s != FEF_OK) return s;
  if (given) {
    drop_logits(&L);
  } else if ((!h_draft && phase != FEF_PHASE_TARGET) || (!h_target && phase != FEF_PHASE_DRAFT && phase != kPhaseTopN) ||
      !W_vocab)
    return fail(FEF_ERR_INVALID_ARG, "h_draft, h_target and W_vocab must not be NULL");
  if (!out_tokens || ((!out_accept_len || !out_remask) && phase != FEF_PHASE_DRAFT))
    return fail(FEF_ERR_INVALID_ARG, "out_tokens, out_accept_len and out_remask must not be NULL");
  if (((uintptr_t)h_draft | (uintptr_t)h_target | (uintptr_t)W_vocab) & 15)
    return fail(FEF_ERR_INVALID_ARG, "h_draft, h_target and W_vocab must be 16-byte aligned");
  if (!prm->ev_head_begin != !prm->ev_head_end)
    return fail(FEF_ERR_INVALID_ARG, "ev_head_begin and ev_head_end must be given together");
  if (!workspace) return fail(FEF_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", L.total);
  if ((uintptr_t)workspace & 255) return fail(FEF_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (workspace_bytes < L.total)
    return fail(FEF_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, L.total);

  char* ws = (char*)workspace;
  hipStream_t stream = (hipStream_t)prm->stream;

  fef::HeadArgs h{};
  h.h_draft = h_draft; h.h_target = h_target; h.W = W_vocab;
  h.BK = prm->B * K; h.d = prm->d; h.V = prm->V;
  h.row0 = phase == FEF_PHASE_TARGET ? h.BK : 0;
  h.nrows = phase == FEF_PHASE_FUSED ? 2 * h.BK : h.BK;
  h.inv_tau = 1.0f / prm->temperature;
  h.logits = (float*)(ws + L.off_logits) + (size_t)h.row0 * L.ldl; h.ldl = L.ldl;
  h.partials = (float2*)(ws + L.off_partials) + (size_t)h.row0 * L.nT; h.nT = L.nT;
  h.stream = stream;
  h.ev_begin = (hipEvent_t)prm->ev_head_begin; h.ev_end = (hipEvent_t)prm->ev_head_end;
  fef::VerifyArgs v;
  memset(&v, 0, sizeof v);
  v.B = prm->B; v.K = K; v.block = block; v.V = prm->V;
  v.row0 = h.row0; v.nrows = h.nrows; v.phase = phase;
  v.ldl = given ? given_ld : L.ldl; v.logits = given ? given : (float*)(ws + L.off_logits); v.partials = (float2*)(ws + L.off_partials); v.nT = L.nT;
  v.tile_unit = L.tile_unit; v.tile_T = L.tile_T; v.tile_G = L.nT;
  v.seed = seed; v.step = prm->step; v.seq_base = prm->seq_base; v.pos_base = prm->pos_base;
  v.n_rm = prm->n_rm; v.final_pass = prm->final_pass; v.lowconf_scope = prm->lowconf_scope;
  v.recorrupt_prob = prm->recorrupt_prob;
  v.greedy = prm->greedy;
  v.mask_in = prm->mask_in; v.pass_mask = prm->pass_mask; v.conf = prm->conf;
  v.draft_tokens_in = prm->draft_tokens;
  v.n_pass = prm->n_pass; v.seq_pass = prm->seq_pass; v.seq_rounds = prm->seq_rounds;
  v.tokens_state = prm->tokens_state;
  v.lse = (float*)(ws + L.off_lse);
  v.xdraft = (int32_t*)(ws + L.off_xdraft);
  v.xtarget = (int32_t*)(ws + L.off_xtarget);
  v.slot_pos = (int32_t*)(ws + L.off_slot_pos);
  v.window = (int32_t*)(ws + L.off_window);
  v.seqstate = (fef::SeqState*)(ws + L.off_seqstate);
  v.rmass = (float*)(ws + L.off_rmass);
  v.amass = (float*)(ws + L.off_amass);
  v.nRC = L.nRC; v.all_slots = L.all_slots;
  v.out_tokens = out_tokens; v.out_accept_len = out_accept_len; v.out_remask = out_remask;
  v.diag_draft_tokens = prm->diag_draft_tokens; v.diag_alpha = prm->diag_alpha;
  v.diag_resid_mass = prm->diag_resid_mass; v.diag_lse = prm->diag_lse;
  v.diag_logits = prm->diag_logits; v.diag_conf_tok = prm->diag_conf_tok;
  v.stream = stream;
  v.n_transfer = n_transfer;
  // (events mark the head kernel alone; the masses of every slot and the logits come from kernels of their own)
  if (given) {
    hipError_t e = fef::launch_logit_partials(v);
    if (e != hipSuccess) return fail(FEF_ERR_HIP, "logit kernel launch: %s", hipGetErrorString(e));
    e = fef::launch_verify(v);
    if (e != hipSuccess) return fail(FEF_ERR_HIP, "verify kernel launch: %s", hipGetErrorString(e));
    return FEF_OK;
  }
  if (L.variant == FEF_GEMM_F32 && phase == FEF_PHASE_FUSED && !h.ev_begin && !v.all_slots && !v.diag_logits &&
      fef::toy_round_serves(v.B, K, h.d, h.V)) {
    const hipError_t e = fef::launch_toy_round(h, v);
    if (e != hipSuccess) return fail(FEF_ERR_HIP, "round kernel launch: %s", hipGetErrorString(e));
    return FEF_OK;
  }
  hipError_t e;
  const int unit = L.variant == FEF_GEMM_TILED256 ? fef::kTiled256Tn : run_unit(L.variant);  // of a partial's tokens; 0: other kernels
  const fef::PieceShape pieces = unit ? fef::piece_shape(h.nrows, h.V, h.d, h.nT, unit) : fef::PieceShape{0, 0, 0, 0};
  if (pieces.pieces) {
    v.row_sums = unit == 16 ? 16 : 64;
    e = fef::launch_head_pieces(h, unit, pieces);
  } else {
    switch (L.variant) {
      case FEF_GEMM_SKINNY: e = fef::launch_head_skinny(h); break;
      case FEF_GEMM_TILED: e = fef::launch_head_tiled(h); break;
      case FEF_GEMM_TILED256: e = fef::launch_head_tiled256(h); break;
      case FEF_GEMM_STREAM:
      case FEF_GEMM_ROWSTREAM: e = fef::launch_head_runs(h, run_unit(L.variant)); break;
      default: e = fef::launch_head_f32(h); break;
    }
  }
  if (e != hipSuccess) return fail(FEF_ERR_HIP, "head kernel launch: %s", hipGetErrorString(e));
  e = fef::launch_verify(v);
  if (e != hipSuccess) return fail(FEF_ERR_HIP, "verify kernel launch: %s", hipGetErrorString(e));
  return FEF_OK;
}
}  // namespace

namespace {
// workspace of a cross-entropy call: partials, label logits
size_t ce_bytes(int32_t R, int nT) {
  return align_up((size_t)R * (size_t)nT * sizeof(float2), 256) + align_up((size_t)R * sizeof(float), 256);
}

// sizes and kernel choice of a cross-entropy call; *variant receives the head kernel
fef_status ce_check(const fef_params* p, int32_t R, int* variant, int* nT, size_t* total) {
  if (!p) return fail(FEF_ERR_INVALID_ARG, "params is NULL");
  if (p->struct_size != sizeof(fef_params))
    return fail(FEF_ERR_INVALID_ARG, "struct_size %u does not match this library's %zu", p->struct_size,
                sizeof(fef_params));
  if (R < 1 || R > (1 << 24)) return fail(FEF_ERR_INVALID_ARG, "R = %d out of range [1, 2^24]", R);
  if (p->V < 1 || p->d < 1) return fail(FEF_ERR_INVALID_ARG, "V and d must be positive");
  if (p->dtype != FEF_BF16 && p->dtype != FEF_F32) return fail(FEF_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
  if (p->dtype == FEF_BF16 && p->d % 64 != 0)
    return fail(FEF_ERR_INVALID_ARG, "bf16 needs d to be a multiple of 64 (got %d)", p->d);
  if (!(p->temperature > 0.f) || !(p->temperature < INFINITY))
    return fail(FEF_ERR_INVALID_ARG, "temperature must be positive and finite");
  int v = p->gemm_variant;
  if (v == FEF_GEMM_AUTO)
    v = p->dtype == FEF_F32 ? FEF_GEMM_F32 : R <= 128 ? FEF_GEMM_STREAM : FEF_GEMM_TILED256;
  switch (v) {
    case FEF_GEMM_F32:
      if (p->dtype != FEF_F32) return fail(FEF_ERR_UNSUPPORTED, "f32 head kernel needs dtype f32");
      if (R > 65535) return fail(FEF_ERR_UNSUPPORTED, "f32 head kernel serves at most 65535 rows");
      break;
    case FEF_GEMM_STREAM:
      if (p->dtype != FEF_BF16 || !stream_supports(R, p->d))
        return fail(FEF_ERR_UNSUPPORTED, "the STREAM variant needs bf16 and at most 128 rows");
      break;
    case FEF_GEMM_TILED256:
      if (p->dtype != FEF_BF16) return fail(FEF_ERR_UNSUPPORTED, "tiled head kernels are bf16 only");
      break;
    default:
      return fail(FEF_ERR_UNSUPPORTED, "cross-entropy runs through the F32, STREAM or TILED256 head kernel");
  }
  *variant = v;
  *nT = v == FEF_GEMM_F32 ? (p->V + fef::kTiledTn - 1) / fef::kTiledTn : fef::tiled256_tiles(p->V, R);
  *total = ce_bytes(R, *nT);
  return FEF_OK;
}
}  // namespace

size_t fef_cross_entropy_workspace_bytes(const fef_params* prm, int32_t R) {
  int v, nT;
  size_t total;
  return ce_check(prm, R, &v, &nT, &total) == FEF_OK ? total : 0;
}

fef_status fef_head_cross_entropy(const fef_params* prm, const void* h, const void* W_vocab,
                                  const int32_t* labels, int32_t R, float* out_ce, float* out_loss) {
  int variant, nT;
  size_t total;
  fef_status s = ce_check(prm, R, &variant, &nT, &total);
  if (s != FEF_OK) return s;
  if (variant == FEF_GEMM_TILED256 && prm->workspace_bytes < total && fef::loss_wide_serves(R, prm->V)) {
    // a workspace of what such a call needs in two row tiles, which leave fewer partials: accepted, with the sums in their order (see fef.h)
    nT = (prm->V + fef::kTiled256Tn - 1) / fef::kTiled256Tn;
    total = ce_bytes(R, nT);
  }
  if (!h || !W_vocab || !labels || !out_ce)
    return fail(FEF_ERR_INVALID_ARG, "h, W_vocab, labels and out_ce must not be NULL");
  if (((uintptr_t)h | (uintptr_t)W_vocab) & 15)
    return fail(FEF_ERR_INVALID_ARG, "h and W_vocab must be 16-byte aligned");
  if (!prm->ev_head_begin != !prm->ev_head_end)
    return fail(FEF_ERR_INVALID_ARG, "ev_head_begin and ev_head_end must be given together");
  if (!prm->workspace) return fail(FEF_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", total);
  if ((uintptr_t)prm->workspace & 255) return fail(FEF_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (prm->workspace_bytes < total)
    return fail(FEF_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", prm->workspace_bytes, total);

  char* ws = (char*)prm->workspace;
  fef::HeadArgs a{};
  a.h_draft = h; a.h_target = h; a.W = W_vocab;
  a.BK = R; a.d = prm->d; a.V = prm->V; a.row0 = 0; a.nrows = R;
  a.inv_tau = 1.0f / prm->temperature;
  a.logits = nullptr; a.ldl = 0;
  a.partials = (float2*)ws; a.nT = nT;
  a.labels = labels;
  a.label_logit = (float*)(ws + align_up((size_t)R * (size_t)nT * sizeof(float2), 256));
  a.stream = (hipStream_t)prm->stream;
  a.ev_begin = (hipEvent_t)prm->ev_head_begin; a.ev_end = (hipEvent_t)prm->ev_head_end;
  hipError_t e;
  switch (variant) {
    case FEF_GEMM_TILED256:
    case FEF_GEMM_STREAM: e = fef::launch_head_tiled256(a); break;
    default: e = fef::launch_head_f32(a); break;
  }
  if (e != hipSuccess) return fail(FEF_ERR_HIP, "head kernel launch: %s", hipGetErrorString(e));
  fef::CeArgs c{};
  c.R = R; c.V = prm->V; c.nT = nT; c.partials = a.partials; c.labels = labels; c.label_logit = a.label_logit;
  c.out_ce = out_ce; c.out_loss = out_loss; c.stream = a.stream;
  e = fef::launch_ce_finish(c);
  if (e != hipSuccess) return fail(FEF_ERR_HIP, "cross-entropy kernel launch: %s", hipGetErrorString(e));
  return FEF_OK;
}

namespace {
// Largest vocabulary of the calls below and longest list of an edit: token and list indices of the kernels, rounded up to whole tiles and
// one step further, then stay in 32 bits with their sign, and a grid of 16-token tiles below 2^32 threads.
constexpr int kMaxGivenV = 1 << 29, kMaxList = 1 << 30;

// Logits are multiplied by 1 / tau, which is infinite for tau below 2^-128 (and a logit of 0 would become NaN).
bool scales_logits(float tau) { return tau > 0.f && tau < 1e30f && 1.f / tau < INFINITY; }

// A call on given logits as one of a 256-token head: a partial per tile, whatever made the logits.
fef_status logits_params(const fef_params* prm, fef_params* p) {
  if (!prm) return fail(FEF_ERR_INVALID_ARG, "params is NULL");
  if (prm->struct_size != sizeof(fef_params))
    return fail(FEF_ERR_INVALID_ARG, "struct_size %u does not match this library's %zu", prm->struct_size, sizeof(fef_params));
  if (prm->V > kMaxGivenV) return fail(FEF_ERR_INVALID_ARG, "V = %d exceeds 2^29", prm->V);
  *p = *prm;
  p->d = 64; p->dtype = FEF_BF16; p->gemm_variant = FEF_GEMM_TILED256; p->temperature = 1.f;
  return FEF_OK;
}
}  // namespace

size_t fef_verify_logits_workspace_bytes(const fef_params* prm, int32_t K, int32_t block) {
  fef_params p;
  Layout L;
  if (logits_params(prm, &p) != FEF_OK || make_layout(&p, K, block, &L) != FEF_OK) return 0;
  drop_logits(&L);
  return L.total;
}

fef_status fef_verify_logits(const fef_params* prm, const float* logits, int64_t ld, int32_t K, int32_t block, uint64_t seed,
                             int32_t* out_tokens, int32_t* out_accept_len, uint8_t* out_remask) {
  fef_params p;
  fef_status s = logits_params(prm, &p);
  if (s != FEF_OK) return s;
  if (!logits || ((uintptr_t)logits & 15)) return fail(FEF_ERR_INVALID_ARG, "logits must not be NULL and be 16-byte aligned");
  if (ld < p.V || ld % 64 != 0 || ld > (1L << 40)) return fail(FEF_ERR_INVALID_ARG, "ld = %ld must be a multiple of 64 in [V, 2^40]", (long)ld);
  if (p.ev_head_begin || p.ev_head_end) return fail(FEF_ERR_INVALID_ARG, "no head kernel runs in this call: ev_head_begin and ev_head_end must be NULL");
  return run_step(&p, p.phase, 0, nullptr, nullptr, nullptr, K, block, seed, out_tokens, out_accept_len, out_remask, p.workspace,
                  p.workspace_bytes, logits, ld);
}

fef_status fef_mx4_logits(const fef_params* prm, const void* h, const uint8_t* codes, const uint8_t* scales, int32_t R,
                          float* out_logits, int64_t ld) {
  if (!prm) return fail(FEF_ERR_INVALID_ARG, "params is NULL");
  if (prm->struct_size != sizeof(fef_params))
    return fail(FEF_ERR_INVALID_ARG, "struct_size %u does not match this library's %zu", prm->struct_size, sizeof(fef_params));
  if (R < 1 || R > (1 << 24)) return fail(FEF_ERR_INVALID_ARG, "R = %d out of range [1, 2^24]", R);
  if (prm->V < 1 || prm->d < 1) return fail(FEF_ERR_INVALID_ARG, "V and d must be positive");
  if (prm->V > kMaxGivenV) return fail(FEF_ERR_INVALID_ARG, "V = %d exceeds 2^29", prm->V);
  if (prm->d % 32 != 0 || prm->d > (1 << 20))
    return fail(FEF_ERR_INVALID_ARG, "a 4-bit head needs d to be a multiple of 32, at most 2^20 (got %d)", prm->d);
  if (prm->dtype != FEF_BF16 && prm->dtype != FEF_F32) return fail(FEF_ERR_INVALID_ARG, "unknown dtype %d", prm->dtype);
  if (!scales_logits(prm->temperature)) return fail(FEF_ERR_INVALID_ARG, "temperature must be a positive finite number with a finite reciprocal");
  if (!h || !codes || !scales || !out_logits) return fail(FEF_ERR_INVALID_ARG, "h, codes, scales and out_logits must not be NULL");
  if (((uintptr_t)h | (uintptr_t)codes | (uintptr_t)scales) & 15)
    return fail(FEF_ERR_INVALID_ARG, "h, codes and scales must be 16-byte aligned");
  if ((uintptr_t)out_logits & 3) return fail(FEF_ERR_INVALID_ARG, "out_logits must be 4-byte aligned");
  if (ld < prm->V || ld > (1L << 40)) return fail(FEF_ERR_INVALID_ARG, "ld = %ld must lie in [V, 2^40]", (long)ld);
  if (!prm->ev_head_begin != !prm->ev_head_end)
    return fail(FEF_ERR_INVALID_ARG, "ev_head_begin and ev_head_end must be given together");
  fef::Mx4Args a{};
  a.h = h; a.codes = codes; a.scales = scales;
  a.R = R; a.d = prm->d; a.V = prm->V; a.f32 = prm->dtype == FEF_F32;
  a.inv_tau = 1.0f / prm->temperature;
  a.logits = out_logits; a.ld = ld;
  a.stream = (hipStream_t)prm->stream;
  a.ev_begin = (hipEvent_t)prm->ev_head_begin; a.ev_end = (hipEvent_t)prm->ev_head_end;
  const hipError_t e = fef::launch_mx4(a);
  if (e != hipSuccess) return fail(FEF_ERR_HIP, "4-bit head kernel launch: %s", hipGetErrorString(e));
  return FEF_OK;
}

namespace {

struct GradLayout {
  int rows, padded, nT, shares_h, blocks;
  long ldl;
  size_t off_z, off_partials, off_g, off_h, off_rest, off_part, off_acc, total;
};

fef_status grad_layout(const fef_params* p, int32_t R, GradLayout* L) {
  if (!p) return fail(FEF_ERR_INVALID_ARG, "params is NULL");
  if (p->struct_size != sizeof(fef_params))
    return fail(FEF_ERR_INVALID_ARG, "struct_size %u does not match this library's %zu", p->struct_size, sizeof(fef_params));
  if (R < 1 || R > (1 << 24)) return fail(FEF_ERR_INVALID_ARG, "R = %d out of range [1, 2^24]", R);
  if (p->V < 1 || p->d < 1) return fail(FEF_ERR_INVALID_ARG, "V and d must be positive");
  if (p->V > kMaxGivenV) return fail(FEF_ERR_INVALID_ARG, "V = %d exceeds 2^29", p->V);
  if (p->d > (1 << 20)) return fail(FEF_ERR_INVALID_ARG, "d = %d exceeds 2^20", p->d);
  if (p->dtype != FEF_BF16 && p->dtype != FEF_F32) return fail(FEF_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
  const bool bf16 = p->dtype == FEF_BF16;
  if (bf16 && p->d % 64 != 0) return fail(FEF_ERR_INVALID_ARG, "bf16 needs d to be a multiple of 64 (got %d)", p->d);
  if (!scales_logits(p->temperature)) return fail(FEF_ERR_INVALID_ARG, "temperature must be a positive finite number with a finite reciprocal");
  if (p->gemm_variant != FEF_GEMM_AUTO && p->gemm_variant != (bf16 ? FEF_GEMM_TILED256 : FEF_GEMM_F32))
    return fail(FEF_ERR_UNSUPPORTED, "gradients run through the TILED256 (bf16) or the F32 head kernel");
  if (p->ev_head_begin || p->ev_head_end) return fail(FEF_ERR_INVALID_ARG, "ev_head_begin and ev_head_end must be NULL in this call");
  L->rows = R < fef::kGradRows ? R : fef::kGradRows;
  L->blocks = (R + fef::kGradRows - 1) / fef::kGradRows;
  L->padded = (int)align_up((size_t)L->rows, 64);
  L->ldl = (long)align_up((size_t)p->V, 64);
  L->nT = bf16 ? (p->V + fef::kTiled256Tn - 1) / fef::kTiled256Tn : (p->V + fef::kTiledTn - 1) / fef::kTiledTn;
  const size_t e = bf16 ? 2 : 4, d = (size_t)p->d;
  L->shares_h = bf16 ? fef::grad_h_shares(L->rows, p->d, p->V) : fef::grad_f32_shares(L->rows, p->d, p->V);
  size_t o = 0;
  auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, 256); return at; };
  L->off_z = take((size_t)(bf16 ? L->rows : L->padded) * L->ldl * 4);
  L->off_partials = take((size_t)L->rows * L->nT * sizeof(float2));
  L->off_g = bf16 ? take((size_t)L->padded * L->ldl * 2) : L->off_z;
  L->off_h = take((size_t)L->padded * d * e);
  L->off_rest = take((size_t)L->rows * 4);
  // (a last block of fewer rows may take more shares of as many rows less)
  L->off_part = take(align_up((size_t)L->rows * d, 4) * 4 * (size_t)L->shares_h);
  L->off_acc = take(bf16 && L->blocks > 1 ? (size_t)p->V * d * 4 : 0);
  L->total = o;
  return FEF_OK;
}
}  // namespace

size_t fef_cross_entropy_grad_workspace_bytes(const fef_params* prm, int32_t R) {
  GradLayout L;
  return grad_layout(prm, R, &L) == FEF_OK ? L.total : 0;
}

fef_status fef_head_cross_entropy_grad(const fef_params* prm, const void* h, const void* W_vocab, const int32_t* labels,
                                       const float* weights, int32_t R, float* out_ce, float* out_loss, void* grad_h, void* grad_w) {
  GradLayout L;
  const fef_status s = grad_layout(prm, R, &L);
  if (s != FEF_OK) return s;
  if (!h || !W_vocab || !labels || !out_ce) return fail(FEF_ERR_INVALID_ARG, "h, W_vocab, labels and out_ce must not be NULL");
  if (!grad_h && !grad_w) return fail(FEF_ERR_INVALID_ARG, "grad_h and grad_w must not both be NULL");
  if (((uintptr_t)h | (uintptr_t)W_vocab | (uintptr_t)grad_h | (uintptr_t)grad_w) & 15)
    return fail(FEF_ERR_INVALID_ARG, "h, W_vocab, grad_h and grad_w must be 16-byte aligned");
  if (((uintptr_t)labels | (uintptr_t)weights | (uintptr_t)out_ce | (uintptr_t)out_loss) & 3)
    return fail(FEF_ERR_INVALID_ARG, "labels, weights, out_ce and out_loss must be 4-byte aligned");
  const bool bf16 = prm->dtype == FEF_BF16;
  const size_t e = bf16 ? 2 : 4, d = (size_t)prm->d, V = (size_t)prm->V;
  const struct { uintptr_t at; size_t bytes; } in[2] = {{(uintptr_t)h, R * d * e}, {(uintptr_t)W_vocab, V * d * e}},
                                                out[2] = {{(uintptr_t)grad_h, grad_h ? R * d * e : 0}, {(uintptr_t)grad_w, grad_w ? V * d * e : 0}};
  auto meet = [](auto& x, auto& y) { return x.bytes && y.bytes && x.at < y.at + y.bytes && y.at < x.at + x.bytes; };
  if (meet(out[0], in[0]) || meet(out[0], in[1]) || meet(out[1], in[0]) || meet(out[1], in[1]) || meet(out[0], out[1]))
    return fail(FEF_ERR_INVALID_ARG, "grad_h and grad_w must overlap neither each other nor h and W_vocab");
  if (!prm->workspace) return fail(FEF_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", L.total);
  if ((uintptr_t)prm->workspace & 255) return fail(FEF_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (prm->workspace_bytes < L.total) return fail(FEF_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", prm->workspace_bytes, L.total);

  char* ws = (char*)prm->workspace;
  hipStream_t stream = (hipStream_t)prm->stream;
  float* const part = (float*)(ws + L.off_part);
  float* const acc = (float*)(ws + L.off_acc);
  hipError_t err = hipSuccess;
  for (int b = 0; b < L.blocks; ++b) {
    const size_t r0 = (size_t)b * fef::kGradRows;
    const int rows = (int)std::min((size_t)fef::kGradRows, (size_t)R - r0);
    const char* hb = (const char*)h + r0 * d * e;
    fef::HeadArgs a{};
    a.h_draft = a.h_target = hb; a.W = W_vocab;
    a.BK = rows; a.d = prm->d; a.V = prm->V; a.row0 = 0; a.nrows = rows;
    a.inv_tau = 1.0f / prm->temperature;
    a.logits = (float*)(ws + L.off_z); a.ldl = L.ldl;
    a.partials = (float2*)(ws + L.off_partials); a.nT = L.nT;
    a.stream = stream;
    err = bf16 ? fef::launch_head_tiled256(a) : fef::launch_head_f32(a);
    if (err != hipSuccess) return fail(FEF_ERR_HIP, "head kernel launch: %s", hipGetErrorString(err));
    fef::GradArgs g{};
    g.rows = rows; g.padded = (int)align_up((size_t)rows, 64); g.V = prm->V; g.d = prm->d; g.nT = L.nT; g.ldl = L.ldl;
    g.z = a.logits; g.partials = a.partials; g.labels = labels + r0; g.weights = weights ? weights + r0 : nullptr; g.inv_tau = a.inv_tau;
    g.h = hb; g.H = grad_w ? ws + L.off_h : nullptr; g.G = ws + L.off_g; g.out_ce = out_ce + r0;
    g.rest = bf16 ? (float*)(ws + L.off_rest) : nullptr;
    err = fef::launch_grad_rows(g, bf16, stream);
    if (err != hipSuccess) return fail(FEF_ERR_HIP, "gradient kernel launch: %s", hipGetErrorString(err));
    const size_t n_h = (size_t)rows * d, stride_h = align_up(n_h, 4), n_w = V * d;
    char* const gh = (char*)grad_h + r0 * d * e;
    if (bf16) {
      if (grad_h) {
        fef::ProductArgs p{};
        p.rows = rows; p.labels = g.labels; p.rest = g.rest;
        p.A = (const __bf16*)g.G; p.lda = L.ldl; p.B = (const __bf16*)W_vocab; p.ldb = prm->d; p.b_rows = prm->V;
        p.M = rows; p.N = prm->d; p.K = (int)L.ldl; p.shares = std::min(fef::grad_h_shares(rows, prm->d, prm->V), L.shares_h); p.stride = stride_h;
        p.C = p.shares > 1 ? (void*)part : (void*)gh;
        err = fef::launch_grad_h(p, stream);
        if (err == hipSuccess && p.shares > 1) err = fef::launch_grad_sum(part, p.shares, stride_h, n_h, gh, true, g.labels, p.N, g.rest, p.B, stream);
      }
      if (err == hipSuccess && grad_w) {
        fef::ProductArgs p{};
        p.rows = rows; p.labels = g.labels; p.rest = g.rest;
        p.A = (const __bf16*)g.G; p.lda = L.ldl; p.B = (const __bf16*)g.H; p.ldb = prm->d; p.b_rows = g.padded;
        p.M = prm->V; p.N = prm->d; p.K = g.padded; p.shares = 1; p.n_first = 1;
        p.C = L.blocks > 1 ? (void*)acc : grad_w; p.add = b > 0;
        err = fef::launch_grad_w(p, L.blocks > 1, stream);
        if (err == hipSuccess && L.blocks > 1 && b + 1 == L.blocks) err = fef::launch_grad_sum(acc, 1, 0, n_w, grad_w, true, nullptr, 1, nullptr, nullptr, stream);
      }
    } else {
      if (grad_h) {
        fef::ProductF32Args p{};
        p.A = (const float*)g.G; p.lda = L.ldl; p.B = (const float*)W_vocab; p.b_rows = prm->V; p.M = rows; p.N = prm->d; p.K = (int)L.ldl;
        p.shares = std::min(fef::grad_f32_shares(rows, prm->d, prm->V), L.shares_h); p.stride = stride_h;
        p.C = p.shares > 1 ? part : (float*)gh; p.labels = p.shares > 1 ? nullptr : g.labels;
        err = fef::launch_grad_product_f32(p, false, stream);
        if (err == hipSuccess && p.shares > 1) err = fef::launch_grad_sum(part, p.shares, stride_h, n_h, gh, false, g.labels, p.N, nullptr, nullptr, stream);
      }
      if (err == hipSuccess && grad_w) {
        fef::ProductF32Args p{};
        p.A = (const float*)g.G; p.lda = L.ldl; p.B = (const float*)g.H; p.b_rows = g.padded; p.M = prm->V; p.N = prm->d; p.K = (int)align_up((size_t)rows, 32); p.shares = 1;
        p.C = (float*)grad_w; p.add = b > 0;
        err = fef::launch_grad_product_f32(p, true, stream);
      }
    }
    if (err != hipSuccess) return fail(FEF_ERR_HIP, "gradient product launch: %s", hipGetErrorString(err));
  }
  if (out_loss) {
    fef::CeArgs c{};
    c.R = R; c.out_ce = out_ce; c.out_loss = out_loss; c.stream = stream;
    err = fef::launch_ce_sum(c);
    if (err != hipSuccess) return fail(FEF_ERR_HIP, "cross-entropy kernel launch: %s", hipGetErrorString(err));
  }
  return FEF_OK;
}

namespace {
// Rows of an output one behind another, slots inside sequences or sequences inside slots.
bool rows_apart(int B, int K, int V, int64_t sq, int64_t sl) {
  return (K == 1 || sl >= V) && (B == 1 || sq >= V) && (K == 1 || B == 1 || sq >= sl * (K - 1) + V || sl >= sq * (B - 1) + V);
}

fef_status check_edit(const fef_edit_params* p, size_t* total) {
  if (!p) return fail(FEF_ERR_INVALID_ARG, "params is NULL");
  if (p->struct_size != sizeof(fef_edit_params))
    return fail(FEF_ERR_INVALID_ARG, "struct_size %u does not match this library's %zu", p->struct_size, sizeof(fef_edit_params));
  if (p->B < 1 || p->V < 1) return fail(FEF_ERR_INVALID_ARG, "B and V must be >= 1 (got %d, %d)", p->B, p->V);
  if (p->V > kMaxGivenV) return fail(FEF_ERR_INVALID_ARG, "V = %d exceeds 2^29", p->V);
  if (p->K < 1 || p->K > FEF_MAX_K) return fail(FEF_ERR_INVALID_ARG, "K = %d out of range [1, %d]", p->K, FEF_MAX_K);
  if ((long)p->B * p->K > (1L << 24)) return fail(FEF_ERR_INVALID_ARG, "B*K = %ld exceeds 2^24 rows per call", (long)p->B * p->K);
  if (p->dtype != FEF_BF16 && p->dtype != FEF_F32) return fail(FEF_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
  if (!scales_logits(p->temperature)) return fail(FEF_ERR_INVALID_ARG, "temperature must be a positive finite number with a finite reciprocal");
  if (p->history_max < 0 || p->n_bias < 0) return fail(FEF_ERR_INVALID_ARG, "history_max and n_bias must not be negative");
  if (p->history_max > kMaxList || p->n_bias > kMaxList)
    return fail(FEF_ERR_INVALID_ARG, "history_max = %d and n_bias = %d must not exceed 2^30", p->history_max, p->n_bias);
  if (p->masks != 0 && p->masks != 1 && p->masks != p->K)
    return fail(FEF_ERR_INVALID_ARG, "masks must be 0, 1 or K (got %d)", p->masks);
  for (const int64_t s : {p->seq_stride, p->slot_stride, p->out_seq_stride, p->out_slot_stride})
    if (s < 0 || s > (1L << 40)) return fail(FEF_ERR_INVALID_ARG, "strides must lie in [0, 2^40]");
  if (!rows_apart(p->B, p->K, p->V, p->out_seq_stride, p->out_slot_stride)) return fail(FEF_ERR_INVALID_ARG, "rows of the output overlap");
  *total = align_up((size_t)p->B * p->K * (size_t)fef::edit_partials(p->V) * sizeof(float2), 256);
  return FEF_OK;
}
}  // namespace

size_t fef_edit_workspace_bytes(const fef_edit_params* prm) {
  size_t total;
  return check_edit(prm, &total) == FEF_OK ? total : 0;
}

fef_status fef_edit_logits(const fef_edit_params* p, const void* logits, float* out, float* out_lse) {
  size_t total;
  const fef_status s = check_edit(p, &total);
  if (s != FEF_OK) return s;
  if (!logits || !out) return fail(FEF_ERR_INVALID_ARG, "logits and out must not be NULL");
  if ((uintptr_t)logits & (p->dtype == FEF_BF16 ? 1 : 3) || (uintptr_t)out & 3 || (uintptr_t)out_lse & 3)
    return fail(FEF_ERR_INVALID_ARG, "logits, out and out_lse must be aligned to their elements");
  if ((const void*)out == logits &&
      (p->dtype != FEF_F32 || (p->B > 1 && p->seq_stride != p->out_seq_stride) || (p->K > 1 && p->slot_stride != p->out_slot_stride)))
    return fail(FEF_ERR_INVALID_ARG, "editing in place needs float32 logits and the same strides");
  if (p->history_max > 0 && !p->history) return fail(FEF_ERR_INVALID_ARG, "history is NULL with history_max %d", p->history_max);
  if (p->n_bias > 0 && (!p->bias_ids || !p->bias_values)) return fail(FEF_ERR_INVALID_ARG, "bias_ids and bias_values must not be NULL with n_bias %d", p->n_bias);
  if (p->masks > 0 && !p->allowed) return fail(FEF_ERR_INVALID_ARG, "allowed is NULL with masks %d", p->masks);
  const uintptr_t lists = (uintptr_t)p->history | (uintptr_t)p->history_len | (uintptr_t)p->prompt_len | (uintptr_t)p->prefix |
                          (uintptr_t)p->repetition | (uintptr_t)p->presence | (uintptr_t)p->frequency | (uintptr_t)p->bias_ids |
                          (uintptr_t)p->bias_values | (uintptr_t)p->allowed;
  if (lists & 3) return fail(FEF_ERR_INVALID_ARG, "lists, penalties and masks must be 4-byte aligned");
  if (!p->workspace) return fail(FEF_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", total);
  if ((uintptr_t)p->workspace & 255) return fail(FEF_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (p->workspace_bytes < total) return fail(FEF_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", p->workspace_bytes, total);
  fef::EditArgs a{};
  a.B = p->B; a.K = p->K; a.V = p->V; a.bf16 = p->dtype == FEF_BF16;
  a.inv_tau = 1.0f / p->temperature;
  a.logits = logits; a.seq_stride = p->seq_stride; a.slot_stride = p->slot_stride;
  a.out = out; a.out_seq_stride = p->out_seq_stride; a.out_slot_stride = p->out_slot_stride;
  if (p->repetition || p->presence || p->frequency) {  // without penalties nothing depends on what occurred
    a.history_max = p->history_max; a.history = p->history; a.history_len = p->history_len; a.prompt_len = p->prompt_len;
    a.prefix = p->prefix;
    a.repetition = p->repetition; a.presence = p->presence; a.frequency = p->frequency;
  }
  a.n_bias = p->n_bias; a.bias_ids = p->bias_ids; a.bias_values = p->bias_values;
  a.masks = p->masks; a.allowed = p->allowed;
  a.partials = (float2*)p->workspace; a.out_lse = out_lse;
  a.stream = (hipStream_t)p->stream;
  const hipError_t e = fef::launch_edit(a);
  if (e != hipSuccess) return fail(FEF_ERR_HIP, "edit kernel launch: %s", hipGetErrorString(e));
  return FEF_OK;
}

namespace {
fef_status check_draw(const fef_draw_params* p, size_t* total) {
  if (!p) return fail(FEF_ERR_INVALID_ARG, "params is NULL");
  if (p->struct_size != sizeof(fef_draw_params))
    return fail(FEF_ERR_INVALID_ARG, "struct_size %u does not match this library's %zu", p->struct_size, sizeof(fef_draw_params));
  if (p->B < 1 || p->V < 1) return fail(FEF_ERR_INVALID_ARG, "B and V must be >= 1 (got %d, %d)", p->B, p->V);
  if (p->V > kMaxGivenV) return fail(FEF_ERR_INVALID_ARG, "V = %d exceeds 2^29", p->V);
  if (p->K < 1 || p->K > FEF_MAX_K) return fail(FEF_ERR_INVALID_ARG, "K = %d out of range [1, %d]", p->K, FEF_MAX_K);
  // (a workgroup of 512 threads per row: 2^30 threads)
  if ((long)p->B * p->K > (1L << 21)) return fail(FEF_ERR_INVALID_ARG, "B*K = %ld exceeds 2^21 rows per call", (long)p->B * p->K);
  if (p->dtype != FEF_BF16 && p->dtype != FEF_F32) return fail(FEF_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
  if (!scales_logits(p->temperature)) return fail(FEF_ERR_INVALID_ARG, "temperature must be a positive finite number with a finite reciprocal");
  for (const int64_t s : {p->seq_stride, p->slot_stride, p->out_seq_stride, p->out_slot_stride})
    if (s < 0 || s > (1L << 40)) return fail(FEF_ERR_INVALID_ARG, "strides must lie in [0, 2^40]");
  *total = align_up(fef::draw_workspace(p->B * p->K, p->V), 256);
  return FEF_OK;
}
}  // namespace

namespace {
// Whether a row of `out` meets one of the logits, each of which is read several times.  Row by row only where one lies within the other's reach.
fef_status check_draw_apart(const fef_draw_params* p, uintptr_t logits, uintptr_t out) {
  const size_t e = p->dtype == FEF_BF16 ? 2 : 4, V = (size_t)p->V, rows = (size_t)p->B * p->K;
  auto in = [&](size_t b, size_t m) { return logits + (b * p->seq_stride + m * p->slot_stride) * e; };
  auto to = [&](size_t b, size_t m) { return out + (b * p->out_seq_stride + m * p->out_slot_stride) * 4; };
  if (out >= in(p->B - 1, p->K - 1) + V * e || logits >= to(p->B - 1, p->K - 1) + V * 4) return FEF_OK;
  std::unique_ptr<uintptr_t[]> at(new (std::nothrow) uintptr_t[rows]);
  if (!at) return fail(FEF_ERR_UNSUPPORTED, "no host memory for the check of %zu rows", rows);
  for (size_t r = 0; r < rows; ++r) at[r] = in(r / p->K, r % p->K);
  std::sort(at.get(), at.get() + rows);  // all of one length: the last that begins in front of a row's end reaches furthest
  for (size_t r = 0; r < rows; ++r) {
    const uintptr_t begin = to(r / p->K, r % p->K), end = begin + V * 4;
    const uintptr_t* const next = std::lower_bound(at.get(), at.get() + rows, end);
    if (next != at.get() && next[-1] + V * e > begin) return fail(FEF_ERR_INVALID_ARG, "out must not overlap the logits: a row is read several times");
  }
  return FEF_OK;
}
}  // namespace

size_t fef_draw_workspace_bytes(const fef_draw_params* prm) {
  size_t total;
  return check_draw(prm, &total) == FEF_OK ? total : 0;
}

fef_status fef_draw_logits(const fef_draw_params* p, const void* logits, float* out) {
  size_t total;
  const fef_status s = check_draw(p, &total);
  if (s != FEF_OK) return s;
  if (!logits) return fail(FEF_ERR_INVALID_ARG, "logits must not be NULL");
  if ((uintptr_t)logits & (p->dtype == FEF_BF16 ? 1 : 3) || (uintptr_t)out & 3)
    return fail(FEF_ERR_INVALID_ARG, "logits and out must be aligned to their elements");
  if (out && !rows_apart(p->B, p->K, p->V, p->out_seq_stride, p->out_slot_stride)) return fail(FEF_ERR_INVALID_ARG, "rows of the output overlap");
  if (out) {
    const fef_status apart = check_draw_apart(p, (uintptr_t)logits, (uintptr_t)out);
    if (apart != FEF_OK) return apart;
  }
  const uintptr_t lists = (uintptr_t)p->temperatures | (uintptr_t)p->top_k | (uintptr_t)p->top_p | (uintptr_t)p->min_p | (uintptr_t)p->uniforms |
                          (uintptr_t)p->out_lse | (uintptr_t)p->out_kept | (uintptr_t)p->out_tokens | (uintptr_t)p->out_conf;
  if (lists & 3) return fail(FEF_ERR_INVALID_ARG, "limits, uniforms and outputs must be 4-byte aligned");
  if (!p->workspace) return fail(FEF_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", total);
  if ((uintptr_t)p->workspace & 255) return fail(FEF_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (p->workspace_bytes < total) return fail(FEF_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", p->workspace_bytes, total);
  fef::DrawArgs a{};
  a.B = p->B; a.K = p->K; a.V = p->V; a.bf16 = p->dtype == FEF_BF16;
  a.inv_tau = 1.0f / p->temperature;
  a.logits = logits; a.seq_stride = p->seq_stride; a.slot_stride = p->slot_stride;
  a.temperatures = p->temperatures; a.top_k = p->top_k; a.top_p = p->top_p; a.min_p = p->min_p; a.uniforms = p->uniforms;
  a.out = out; a.out_seq_stride = p->out_seq_stride; a.out_slot_stride = p->out_slot_stride;
  a.out_lse = p->out_lse; a.out_kept = p->out_kept; a.out_tokens = p->out_tokens; a.out_conf = p->out_conf;
  a.workspace = p->workspace;
  a.stream = (hipStream_t)p->stream;
  const hipError_t e = fef::launch_draw(a);
  if (e != hipSuccess) return fail(FEF_ERR_HIP, "draw kernel launch: %s", hipGetErrorString(e));
  return FEF_OK;
}

namespace {
// An address range of an AdamW step; ranges that are written may not meet any other.
struct Range {
  uintptr_t begin, end;
  bool written;
};

fef_status check_adamw(const fef_adamw_params* p, const fef_adamw_tensor* ts, int32_t count) {
  if (!p) return fail(FEF_ERR_INVALID_ARG, "params is NULL");
  if (p->struct_size != sizeof(fef_adamw_params))
    return fail(FEF_ERR_INVALID_ARG, "struct_size %u does not match this library's %zu", p->struct_size, sizeof(fef_adamw_params));
  if (count < 0 || count > 65536) return fail(FEF_ERR_INVALID_ARG, "count = %d out of range [0, 65536]", count);
  if (count > 0 && !ts) return fail(FEF_ERR_INVALID_ARG, "tensors is NULL with count %d", count);
  if (p->dtype != FEF_BF16 && p->dtype != FEF_F32) return fail(FEF_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
  if (p->grad_dtype != FEF_BF16 && p->grad_dtype != FEF_F32) return fail(FEF_ERR_INVALID_ARG, "unknown grad_dtype %d", p->grad_dtype);
  if (p->state_dtype != FEF_STATE_F32 && p->state_dtype != FEF_STATE_E4M3 && p->state_dtype != FEF_STATE_E4M3_RECIPROCAL)
    return fail(FEF_ERR_INVALID_ARG, "unknown state_dtype %d", p->state_dtype);
  if (!(std::fabs(p->lr) <= 1e30)) return fail(FEF_ERR_INVALID_ARG, "lr must be a finite number");
  if (!(p->beta1 >= 0 && (float)p->beta1 < 1.f) || !(p->beta2 >= 0 && (float)p->beta2 < 1.f))
    return fail(FEF_ERR_INVALID_ARG, "beta1 and beta2 must lie in [0, 1)");
  if (!(p->eps <= 1e30) || !((float)p->eps > 0.f)) return fail(FEF_ERR_INVALID_ARG, "eps must be a positive finite number");
  if (p->step < 1) return fail(FEF_ERR_INVALID_ARG, "step must be at least 1 (got %ld)", (long)p->step);
  if (((uintptr_t)p->schedule | (uintptr_t)p->grad_scale) & 3)
    return fail(FEF_ERR_INVALID_ARG, "schedule and grad_scale must be 4-byte aligned");
  if (count == 0) return FEF_OK;
  const bool eight = p->state_dtype != FEF_STATE_F32;
  const uintptr_t pa = p->dtype == FEF_BF16 ? 1 : 3, ga = p->grad_dtype == FEF_BF16 ? 1 : 3, sa = eight ? 0 : 3;
  std::unique_ptr<Range[]> ranges(new (std::nothrow) Range[(size_t)count * 7 + 2]);
  if (!ranges) return fail(FEF_ERR_UNSUPPORTED, "no host memory for the check of %d tensors", count);
  size_t used = 0;
  auto add = [&](const void* at, size_t bytes, bool written) {
    ranges[used++] = Range{(uintptr_t)at, (uintptr_t)at + bytes, written};
  };
  if (p->schedule) add(p->schedule, 12, false);
  if (p->grad_scale) add(p->grad_scale, 4, false);
  for (int i = 0; i < count; ++i) {
    const fef_adamw_tensor& t = ts[i];
    if (t.n < 0 || t.n > (1L << 36)) return fail(FEF_ERR_INVALID_ARG, "tensor %d: n = %ld out of range [0, 2^36]", i, (long)t.n);
    if (!(t.weight_decay >= 0 && t.weight_decay <= 1e30)) return fail(FEF_ERR_INVALID_ARG, "tensor %d: weight_decay must be finite and not negative", i);
    if (t.n == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v) return fail(FEF_ERR_INVALID_ARG, "tensor %d: param, grad, m and v must not be NULL", i);
    if (t.master && p->dtype != FEF_BF16) return fail(FEF_ERR_INVALID_ARG, "tensor %d: master is for bf16 parameters", i);
    if (eight ? !t.m_scale || !t.v_scale : t.m_scale || t.v_scale)
      return fail(FEF_ERR_INVALID_ARG, "tensor %d: m_scale and v_scale belong to states in 8 bits", i);
    if (((uintptr_t)t.param & pa) || ((uintptr_t)t.grad & ga) || (((uintptr_t)t.m | (uintptr_t)t.v) & sa) ||
        (((uintptr_t)t.master | (uintptr_t)t.m_scale | (uintptr_t)t.v_scale) & 3))
      return fail(FEF_ERR_INVALID_ARG, "tensor %d: addresses must be aligned to their elements", i);
    const size_t n = (size_t)t.n, s = eight ? 1 : 4, blocks = (n + fef::kAdamwBlock - 1) / fef::kAdamwBlock * 4;
    add(t.param, n * (pa + 1), true);
    add(t.grad, n * (ga + 1), false);
    if (t.master) add(t.master, n * 4, true);
    add(t.m, n * s, true);
    add(t.v, n * s, true);
    if (eight) {
      add(t.m_scale, blocks, true);
      add(t.v_scale, blocks, true);
    }
  }
  std::sort(ranges.get(), ranges.get() + used, [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t any = 0, written = 0;  // ends of the ranges so far
  for (size_t i = 0; i < used; ++i) {
    const Range& r = ranges[i];
    if (r.begin < (r.written ? any : written)) return fail(FEF_ERR_INVALID_ARG, "tensors of the step overlap");
    any = std::max(any, r.end);
    if (r.written) written = std::max(written, r.end);
  }
  return FEF_OK;
}
}  // namespace

fef_status fef_adamw_step(const fef_adamw_params* prm, const fef_adamw_tensor* tensors, int32_t count) {
  const fef_status s = check_adamw(prm, tensors, count);
  if (s != FEF_OK) return s;
  fef::AdamwConst c{};
  c.lr = (float)prm->lr;
  c.b1 = (float)prm->beta1; c.one_b1 = (float)(1.0 - prm->beta1);
  c.b2 = (float)prm->beta2; c.one_b2 = (float)(1.0 - prm->beta2);
  c.c1 = (float)(1.0 / (1.0 - std::pow(prm->beta1, (double)prm->step)));
  c.c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(prm->beta2, (double)prm->step)));
  c.eps = (float)prm->eps;
  c.schedule = prm->schedule; c.grad_scale = prm->grad_scale;
  const bool eight = prm->state_dtype != FEF_STATE_F32;
  c.reciprocal = prm->state_dtype == FEF_STATE_E4M3_RECIPROCAL;
  fef::AdamwTensor some[fef::kAdamwTensors];  // a launch's worth at a time
  for (int32_t i = 0; i < count;) {
    int k = 0;
    for (; i < count && k < fef::kAdamwTensors; ++i) {
      const fef_adamw_tensor& t = tensors[i];
      if (t.n == 0) continue;
      const uintptr_t all = (uintptr_t)t.param | (uintptr_t)t.grad | (uintptr_t)t.master | (eight ? 0 : (uintptr_t)t.m | (uintptr_t)t.v);
      const uintptr_t codes = eight ? (uintptr_t)t.m | (uintptr_t)t.v : 0;
      some[k++] = fef::AdamwTensor{t.param, t.grad, t.master, t.m, t.v, t.m_scale, t.v_scale, (long)t.n, (float)t.weight_decay,
                                   !(all & 15) && !(codes & 3)};
    }
    const hipError_t e = fef::launch_adamw(c, some, k, prm->dtype == FEF_BF16, prm->grad_dtype == FEF_BF16, eight, (hipStream_t)prm->stream);
    if (e != hipSuccess) return fail(FEF_ERR_HIP, "AdamW kernel launch: %s", hipGetErrorString(e));
  }
  return FEF_OK;
}

float fef_uniform(uint64_t seed, uint32_t position, uint32_t step, uint32_t sequence, uint32_t stream) {
  return fef::philox_uniform(seed, position, step, sequence, stream);
}

const char* fef_status_string(fef_status s) {
  switch (s) {
    case FEF_OK: return "ok";
    case FEF_ERR_INVALID_ARG: return "invalid argument";
    case FEF_ERR_UNSUPPORTED: return "unsupported configuration";
    case FEF_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
    case FEF_ERR_HIP: return "HIP runtime error";
  }
  return "unknown status";
}

const char* fef_last_error(void) { return g_err; }

int32_t fef_abi_version(void) { return FEF_ABI_VERSION; }

}  // extern "C"
