"""ctypes binding of libfef.so (see include/fef.h).  Argument marshalling only: every step of
the verify path runs in the library's HIP kernels.  PyTorch supplies device memory and the
current stream.  There is no fallback: if the library has not been built, loading raises.
"""
import ctypes
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("FEF_LIB") or os.path.join(_HERE, "libfef.so")  # FEF_LIB: another build of the same library

FEF_OK = 0
FEF_ERR_INVALID_ARG = -1
FEF_ERR_UNSUPPORTED = -2
FEF_ERR_WORKSPACE = -3
FEF_ERR_HIP = -4
FEF_BF16, FEF_F32 = 0, 1
FEF_GEMM_AUTO, FEF_GEMM_SKINNY, FEF_GEMM_TILED, FEF_GEMM_F32, FEF_GEMM_TILED256, FEF_GEMM_STREAM = 0, 1, 2, 3, 4, 5
FEF_GEMM_ROWSTREAM = 6
FEF_MAX_K, FEF_MAX_BLOCK = 64, 4096
FEF_PHASE_FUSED, FEF_PHASE_DRAFT, FEF_PHASE_TARGET = 0, 1, 2
FEF_STATE_F32, FEF_STATE_E4M3, FEF_STATE_E4M3_RECIPROCAL = 0, 1, 3

ABI_VERSION = 12   # FEF_ABI_VERSION of include/fef.h this binding's fef_params mirrors

EXPORTS = ["fef_workspace_bytes", "fef_verify_step", "fef_select_gemm", "fef_uniform",
           "fef_status_string", "fef_last_error", "fef_abi_version", "fef_copy_probe", "fef_read_probe",
           "fef_cross_entropy_workspace_bytes", "fef_head_cross_entropy", "fef_topn_step",
           "fef_verify_step_static", "fef_mx4_logits", "fef_edit_workspace_bytes", "fef_edit_logits",
           "fef_verify_logits_workspace_bytes", "fef_verify_logits", "fef_adamw_step",
           "fef_draw_workspace_bytes", "fef_draw_logits", "fef_cross_entropy_grad_workspace_bytes", "fef_head_cross_entropy_grad"]
FEF_STATIC_SCRATCH_BYTES = 32 << 20


class fef_params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("B", ctypes.c_int32), ("d", ctypes.c_int32), ("V", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("temperature", ctypes.c_float),
        ("step", ctypes.c_uint32), ("seq_base", ctypes.c_uint32), ("pos_base", ctypes.c_uint32),
        ("n_rm", ctypes.c_int32), ("final_pass", ctypes.c_int32),
        ("lowconf_scope", ctypes.c_int32), ("gemm_variant", ctypes.c_int32),
        ("mask_in", ctypes.c_void_p), ("pass_mask", ctypes.c_void_p), ("conf", ctypes.c_void_p),
        ("draft_tokens", ctypes.c_void_p),
        ("diag_draft_tokens", ctypes.c_void_p), ("diag_alpha", ctypes.c_void_p),
        ("diag_resid_mass", ctypes.c_void_p), ("diag_lse", ctypes.c_void_p),
        ("diag_logits", ctypes.c_void_p), ("diag_conf_tok", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("stream", ctypes.c_void_p),
        ("ev_head_begin", ctypes.c_void_p), ("ev_head_end", ctypes.c_void_p),
        ("n_pass", ctypes.c_int32), ("seq_pass", ctypes.c_void_p), ("seq_rounds", ctypes.c_void_p),
        ("tokens_state", ctypes.c_void_p), ("phase", ctypes.c_int32),
        ("recorrupt_prob", ctypes.c_float), ("greedy", ctypes.c_int32),
    ]


_PARAMS_SIZE = ctypes.sizeof(fef_params)
_DIAG = ("draft_tokens", "alpha", "resid_mass", "lse", "logits", "conf_tok")  # VerifyStep.diag in the order of the fields
_NO_DIAG = (None,) * len(_DIAG)


class fef_edit_params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("B", ctypes.c_int32), ("K", ctypes.c_int32), ("V", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("temperature", ctypes.c_float),
        ("seq_stride", ctypes.c_int64), ("slot_stride", ctypes.c_int64),
        ("out_seq_stride", ctypes.c_int64), ("out_slot_stride", ctypes.c_int64),
        ("history_max", ctypes.c_int32), ("history", ctypes.c_void_p),
        ("history_len", ctypes.c_void_p), ("prompt_len", ctypes.c_void_p), ("prefix", ctypes.c_void_p),
        ("repetition", ctypes.c_void_p), ("presence", ctypes.c_void_p), ("frequency", ctypes.c_void_p),
        ("n_bias", ctypes.c_int32), ("bias_ids", ctypes.c_void_p), ("bias_values", ctypes.c_void_p),
        ("masks", ctypes.c_int32), ("allowed", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("stream", ctypes.c_void_p),
    ]


_EDIT_PARAMS_SIZE = ctypes.sizeof(fef_edit_params)
_PACK_EDIT = struct.Struct("@I4if4qi7Pi2PiPPNP").pack_into  # fef_edit_params, field by field in native alignment


class fef_draw_params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("B", ctypes.c_int32), ("K", ctypes.c_int32), ("V", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("temperature", ctypes.c_float),
        ("seq_stride", ctypes.c_int64), ("slot_stride", ctypes.c_int64),
        ("out_seq_stride", ctypes.c_int64), ("out_slot_stride", ctypes.c_int64),
        ("temperatures", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p), ("min_p", ctypes.c_void_p),
        ("uniforms", ctypes.c_void_p),
        ("out_lse", ctypes.c_void_p), ("out_kept", ctypes.c_void_p), ("out_tokens", ctypes.c_void_p), ("out_conf", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("stream", ctypes.c_void_p),
    ]


_DRAW_PARAMS_SIZE = ctypes.sizeof(fef_draw_params)
_PACK_DRAW = struct.Struct("@I4if4q10PNP").pack_into  # fef_draw_params, field by field in native alignment


class fef_adamw_tensor(ctypes.Structure):
    _fields_ = [
        ("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("master", ctypes.c_void_p),
        ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
        ("n", ctypes.c_int64), ("weight_decay", ctypes.c_double),
    ]


class fef_adamw_params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("state_dtype", ctypes.c_int32),
        ("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
        ("step", ctypes.c_int64),
        ("schedule", ctypes.c_void_p), ("grad_scale", ctypes.c_void_p),
        ("stream", ctypes.c_void_p),
    ]


class FefError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"fef status {status}: {message}")
        self.status = status


_lib = None


def lib():
    """Load libfef.so once.  Raises if it has not been built (python -m paper_2605_14305_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2605_14305_amd.build`; "
                "there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        L.fef_workspace_bytes.restype = ctypes.c_size_t
        L.fef_workspace_bytes.argtypes = [ctypes.POINTER(fef_params), ctypes.c_int32, ctypes.c_int32]
        L.fef_verify_step.restype = ctypes.c_int
        L.fef_verify_step.argtypes = [ctypes.POINTER(fef_params), ctypes.c_void_p, ctypes.c_void_p,
                                      ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_uint64,
                                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.fef_verify_step_static.restype = ctypes.c_int
        L.fef_verify_step_static.argtypes = L.fef_verify_step.argtypes
        L.fef_select_gemm.restype = ctypes.c_int32
        L.fef_select_gemm.argtypes = [ctypes.POINTER(fef_params), ctypes.c_int32]
        L.fef_uniform.restype = ctypes.c_float
        L.fef_uniform.argtypes = [ctypes.c_uint64, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint32,
                                  ctypes.c_uint32]
        L.fef_status_string.restype = ctypes.c_char_p
        L.fef_status_string.argtypes = [ctypes.c_int]
        L.fef_last_error.restype = ctypes.c_char_p
        L.fef_last_error.argtypes = []
        L.fef_copy_probe.restype = ctypes.c_int
        L.fef_copy_probe.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.fef_read_probe.restype = ctypes.c_int
        L.fef_read_probe.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]
        L.fef_abi_version.restype = ctypes.c_int32
        L.fef_abi_version.argtypes = []
        L.fef_cross_entropy_workspace_bytes.restype = ctypes.c_size_t
        L.fef_cross_entropy_workspace_bytes.argtypes = [ctypes.POINTER(fef_params), ctypes.c_int32]
        L.fef_topn_step.restype = ctypes.c_int
        L.fef_topn_step.argtypes = [ctypes.POINTER(fef_params), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                    ctypes.c_int32, ctypes.c_uint64, ctypes.c_int32, ctypes.c_void_p,
                                    ctypes.c_void_p, ctypes.c_void_p]
        L.fef_head_cross_entropy.restype = ctypes.c_int
        L.fef_head_cross_entropy.argtypes = [ctypes.POINTER(fef_params), ctypes.c_void_p, ctypes.c_void_p,
                                             ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
        L.fef_mx4_logits.restype = ctypes.c_int
        L.fef_mx4_logits.argtypes = [ctypes.POINTER(fef_params), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                     ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64]
        L.fef_verify_logits_workspace_bytes.restype = ctypes.c_size_t
        L.fef_verify_logits_workspace_bytes.argtypes = [ctypes.POINTER(fef_params), ctypes.c_int32, ctypes.c_int32]
        L.fef_verify_logits.restype = ctypes.c_int
        L.fef_verify_logits.argtypes = [ctypes.POINTER(fef_params), ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                        ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.fef_edit_workspace_bytes.restype = ctypes.c_size_t
        L.fef_edit_workspace_bytes.argtypes = [ctypes.POINTER(fef_edit_params)]
        L.fef_edit_logits.restype = ctypes.c_int
        L.fef_edit_logits.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.fef_cross_entropy_grad_workspace_bytes.restype = ctypes.c_size_t
        L.fef_cross_entropy_grad_workspace_bytes.argtypes = [ctypes.POINTER(fef_params), ctypes.c_int32]
        L.fef_head_cross_entropy_grad.restype = ctypes.c_int
        L.fef_head_cross_entropy_grad.argtypes = [ctypes.POINTER(fef_params), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                                  ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.fef_draw_workspace_bytes.restype = ctypes.c_size_t
        L.fef_draw_workspace_bytes.argtypes = [ctypes.POINTER(fef_draw_params)]
        L.fef_draw_logits.restype = ctypes.c_int
        L.fef_draw_logits.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.fef_adamw_step.restype = ctypes.c_int
        L.fef_adamw_step.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32]
        if L.fef_abi_version() != ABI_VERSION:
            raise RuntimeError(f"{LIB_PATH} has ABI version {L.fef_abi_version()}, this binding needs {ABI_VERSION}: "
                               "rebuild it with `python -m paper_2605_14305_amd.build`")
        _lib = L
    return _lib


def _ptr(t):
    """Device address of a tensor for a c_void_p argument or field (None = NULL)."""
    return None if t is None else t.data_ptr()


def _stream(device):
    """Raw handle of torch's current stream on `device` (a device without an index: the current one), without
    building a Stream object around it: 2 us less per call."""
    index = device.index
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice() if index is None else index)


def make_params(B, d, V, dtype=FEF_BF16, temperature=1.0, step=0, seq_base=0, pos_base=0,
                n_rm=-1, final_pass=0, lowconf_scope=0, gemm_variant=FEF_GEMM_AUTO):
    p = fef_params()
    p.struct_size = ctypes.sizeof(fef_params)
    p.B, p.d, p.V, p.dtype = B, d, V, dtype
    p.temperature = temperature
    p.step, p.seq_base, p.pos_base = step, seq_base, pos_base
    p.n_rm, p.final_pass, p.lowconf_scope, p.gemm_variant = n_rm, int(final_pass), lowconf_scope, gemm_variant
    p.recorrupt_prob = 1.0
    return p


def fef_workspace_bytes(params, K, block):
    return lib().fef_workspace_bytes(ctypes.byref(params), K, block)


def fef_select_gemm(params, K):
    return lib().fef_select_gemm(ctypes.byref(params), K)


def fef_uniform(seed, position, step, sequence, stream):
    return lib().fef_uniform(seed, position, step, sequence, stream)


def fef_last_error():
    return lib().fef_last_error().decode()


def fef_verify_step(params, h_draft, h_target, W_vocab, K, block, seed, out_tokens, out_accept_len,
                    out_remask):
    """Raw call: tensors (or None) are passed as device pointers; raises FefError on failure."""
    s = (_lib or lib()).fef_verify_step(ctypes.byref(params), _ptr(h_draft), _ptr(h_target), _ptr(W_vocab), K,
                                        block, seed & 0xFFFFFFFFFFFFFFFF, _ptr(out_tokens),
                                        _ptr(out_accept_len), _ptr(out_remask))
    if s != FEF_OK:
        raise FefError(s, fef_last_error())
    return s


def fef_verify_step_static(params, h_draft, h_target, W_vocab, K, block, seed, out_tokens, out_accept_len,
                           out_remask):
    """fef_verify_step on the library's built-in scratch buffer: no workspace, no allocation."""
    s = lib().fef_verify_step_static(ctypes.byref(params), _ptr(h_draft), _ptr(h_target), _ptr(W_vocab), K,
                                     block, seed & 0xFFFFFFFFFFFFFFFF, _ptr(out_tokens),
                                     _ptr(out_accept_len), _ptr(out_remask))
    if s != FEF_OK:
        raise FefError(s, fef_last_error())
    return s


def fef_copy_probe(dst, src):
    """Plain device copy of known traffic (profiler counter calibration)."""
    assert dst.numel() * dst.element_size() == src.numel() * src.element_size()
    s = lib().fef_copy_probe(_ptr(dst), _ptr(src), src.numel() * src.element_size(),
                             torch.cuda.current_stream().cuda_stream)
    if s != FEF_OK:
        raise FefError(s, fef_last_error())


def fef_read_probe(src, sink):
    """Plain streaming read of `src` (the practical HBM read ceiling); `sink` is a 4-byte device tensor."""
    s = lib().fef_read_probe(_ptr(src), src.numel() * src.element_size(), _ptr(sink),
                             torch.cuda.current_stream().cuda_stream)
    if s != FEF_OK:
        raise FefError(s, fef_last_error())


class HeadCrossEntropy:
    """Token-level cross-entropy of R rows through the vocabulary head (fef_head_cross_entropy);
    holds workspace and outputs of one shape so that repeated calls do no allocation."""

    def __init__(self, R, d, V, dtype="bf16", device="cuda", gemm_variant=FEF_GEMM_AUTO):
        self.R, self.d, self.V, self.device = R, d, V, torch.device(device)
        self.dtype = FEF_BF16 if dtype == "bf16" else FEF_F32
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.gemm_variant = gemm_variant
        n = lib().fef_cross_entropy_workspace_bytes(ctypes.byref(self._params()), R)
        if n == 0:
            raise FefError(FEF_ERR_INVALID_ARG, fef_last_error())
        self.workspace = torch.empty(n, dtype=torch.uint8, device=self.device)
        self.out_ce = torch.empty(R, dtype=torch.float32, device=self.device)
        self.out_loss = torch.empty(1, dtype=torch.float32, device=self.device)

    def _params(self, temperature=1.0):
        return make_params(1, self.d, self.V, dtype=self.dtype, temperature=temperature,
                           gemm_variant=self.gemm_variant)

    def __call__(self, h, W_vocab, labels, temperature=1.0, head_events=None):
        assert h.shape == (self.R, self.d) and W_vocab.shape == (self.V, self.d)
        assert h.dtype == self.torch_dtype and W_vocab.dtype == self.torch_dtype
        assert labels.dtype == torch.int32 and labels.shape == (self.R,)
        for t in (h, W_vocab, labels):
            assert t.is_contiguous() and t.is_cuda
        p = self._params(temperature)
        p.workspace = self.workspace.data_ptr()
        p.workspace_bytes = self.workspace.numel()
        p.stream = _stream(self.device)
        if head_events is not None:
            p.ev_head_begin, p.ev_head_end = head_events
        s = lib().fef_head_cross_entropy(ctypes.byref(p), _ptr(h), _ptr(W_vocab), _ptr(labels), self.R,
                                         _ptr(self.out_ce), _ptr(self.out_loss))
        if s != FEF_OK:
            raise FefError(s, fef_last_error())
        return self.out_ce, self.out_loss


class HeadCrossEntropyGrad:
    """Cross-entropy of R rows through the vocabulary head with its gradients in h and W (fef_head_cross_entropy_grad); holds workspace and
    outputs of one shape.  A call returns out_ce [R], out_loss [1], grad_h [R, d] and grad_w [V, d] (None where the constructor was told
    so).  `weights` [R] (float32): the gradient of the program's loss in each row's cross-entropy, 1 if left out."""

    def __init__(self, R, d, V, dtype="bf16", device="cuda", grad_h=True, grad_w=True):
        self.R, self.d, self.V, self.device = R, d, V, torch.device(device)
        self.dtype = FEF_BF16 if dtype == "bf16" else FEF_F32
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self._params = make_params(1, d, V, dtype=self.dtype)
        n = lib().fef_cross_entropy_grad_workspace_bytes(ctypes.byref(self._params), R)
        if n == 0:
            raise FefError(FEF_ERR_INVALID_ARG, fef_last_error())
        self.workspace = torch.empty(n, dtype=torch.uint8, device=self.device)
        self.out_ce = torch.empty(R, dtype=torch.float32, device=self.device)
        self.out_loss = torch.empty(1, dtype=torch.float32, device=self.device)
        self.grad_h = torch.empty(R, d, dtype=self.torch_dtype, device=self.device) if grad_h else None
        self.grad_w = torch.empty(V, d, dtype=self.torch_dtype, device=self.device) if grad_w else None

    def __call__(self, h, W_vocab, labels, weights=None, temperature=1.0):
        for t, shape, dt in ((h, (self.R, self.d), self.torch_dtype), (W_vocab, (self.V, self.d), self.torch_dtype),
                             (labels, (self.R,), torch.int32), (weights, (self.R,), torch.float32)):
            assert t is None or (t.shape == shape and t.dtype == dt and t.is_contiguous() and t.is_cuda)
        p = self._params
        p.temperature = temperature
        p.workspace, p.workspace_bytes, p.stream = self.workspace.data_ptr(), self.workspace.numel(), _stream(self.device)
        s = (_lib or lib()).fef_head_cross_entropy_grad(ctypes.byref(p), h.data_ptr(), W_vocab.data_ptr(), labels.data_ptr(), _ptr(weights), self.R,
                                                        self.out_ce.data_ptr(), self.out_loss.data_ptr(), _ptr(self.grad_h), _ptr(self.grad_w))
        if s != FEF_OK:
            raise FefError(s, fef_last_error())
        return self.out_ce, self.out_loss, self.grad_h, self.grad_w


class VerifyStep:
    """Holds the output and workspace tensors of one problem shape so that repeated calls do no
    allocation.  `diag=True` also returns draft tokens, alpha, residual mass, lse, confidences
    (and logits with diag_logits=True)."""

    def __init__(self, B, K, block, d, V, dtype="bf16", device="cuda", diag=False, diag_logits=False,
                 gemm_variant=FEF_GEMM_AUTO):
        self.B, self.K, self.block, self.d, self.V = B, K, block, d, V
        self.dtype = FEF_BF16 if dtype == "bf16" else FEF_F32
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.device = torch.device(device)
        self.gemm_variant = gemm_variant
        dev = self.device
        self.out_tokens = torch.empty(B, K, dtype=torch.int32, device=dev)
        self.out_accept_len = torch.empty(B, dtype=torch.int32, device=dev)
        self.out_remask = torch.empty(B, block, dtype=torch.uint8, device=dev)
        self.diag = {}
        if diag:
            self.diag = {
                "draft_tokens": torch.empty(B, K, dtype=torch.int32, device=dev),
                "alpha": torch.empty(B, K, dtype=torch.float32, device=dev),
                "resid_mass": torch.empty(B, K, dtype=torch.float32, device=dev),
                "lse": torch.empty(2, B, K, dtype=torch.float32, device=dev),
                "conf_tok": torch.empty(B, K, dtype=torch.float32, device=dev),
            }
            if diag_logits:
                self.diag["logits"] = torch.empty(2, B, K, V, dtype=torch.float32, device=dev)
        p = self._params()
        nbytes = fef_workspace_bytes(p, K, block)
        if nbytes == 0:
            raise FefError(FEF_ERR_INVALID_ARG, fef_last_error())
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)

    def _params(self, **kw):
        p = make_params(self.B, self.d, self.V, dtype=self.dtype, gemm_variant=self.gemm_variant, **kw)
        g = self.diag
        if g:
            p.diag_draft_tokens = g["draft_tokens"].data_ptr()
            p.diag_alpha = g["alpha"].data_ptr()
            p.diag_resid_mass = g["resid_mass"].data_ptr()
            p.diag_lse = g["lse"].data_ptr()
            p.diag_conf_tok = g["conf_tok"].data_ptr()
            if "logits" in g:
                p.diag_logits = g["logits"].data_ptr()
        return p

    def __call__(self, h_draft, h_target, W_vocab, seed, *, temperature=1.0, step=0, seq_base=0,
                 pos_base=0, n_rm=-1, final_pass=False, lowconf_scope=0, mask_in=None, pass_mask=None,
                 conf=None, draft_tokens=None, head_events=None, n_pass=0, seq_pass=None, seq_rounds=None,
                 tokens_state=None, phase=FEF_PHASE_FUSED, recorrupt_prob=1.0, greedy=False):
        B, block, dt = self.B, self.block, self.torch_dtype
        rows = (B, self.K, self.d)
        for t, shape in ((h_draft, rows), (h_target, rows), (W_vocab, (self.V, self.d))):
            if t is not None:
                assert t.shape == shape and t.dtype == dt and t.is_contiguous() and t.is_cuda
        for t, dt, shape in ((mask_in, torch.uint8, (B, block)), (pass_mask, torch.uint8, (B, block)),
                             (conf, torch.float32, (B, block)), (draft_tokens, torch.int32, (B, self.K)),
                             (seq_pass, torch.int32, (B,)), (seq_rounds, torch.int32, (B,)),
                             (tokens_state, torch.int32, (B, block))):
            if t is not None:
                assert t.dtype == dt and t.shape == shape and t.is_contiguous() and t.is_cuda
        g = self.diag
        diag = [_ptr(g.get(k)) for k in _DIAG] if g else _NO_DIAG
        ev_begin, ev_end = head_events if head_events is not None else (None, None)  # raw hipEvent_t handles (ints)
        # one constructor call over all fields in their order: a third of the time of setting them one by one
        p = fef_params(_PARAMS_SIZE, B, self.d, self.V, self.dtype, temperature, step, seq_base, pos_base, n_rm,
                       int(final_pass), lowconf_scope, self.gemm_variant, _ptr(mask_in), _ptr(pass_mask), _ptr(conf),
                       _ptr(draft_tokens), *diag, self.workspace.data_ptr(), self.workspace.numel(), _stream(self.device),
                       ev_begin, ev_end, n_pass, _ptr(seq_pass), _ptr(seq_rounds), _ptr(tokens_state), phase, recorrupt_prob,
                       int(greedy))
        fef_verify_step(p, h_draft, h_target, W_vocab, self.K, self.block, seed, self.out_tokens,
                        self.out_accept_len, self.out_remask)
        return self.out_tokens, self.out_accept_len, self.out_remask


def topn_step(vs, h, W_vocab, seed, n_transfer, *, temperature=1.0, step=0, seq_base=0, pos_base=0,
              mask_in=None, conf=None, tokens_state=None, greedy=False):
    """Baseline step (fef_topn_step) on the buffers of a VerifyStep of the same shape.  Returns
    (tokens [B,K], committed [B], remask [B,block])."""
    assert h.shape == (vs.B, vs.K, vs.d) and h.dtype == vs.torch_dtype and h.is_contiguous()
    p = vs._params(temperature=temperature, step=step, seq_base=seq_base, pos_base=pos_base)
    p.mask_in = None if mask_in is None else mask_in.data_ptr()
    p.conf = None if conf is None else conf.data_ptr()
    p.tokens_state = None if tokens_state is None else tokens_state.data_ptr()
    p.greedy = int(greedy)
    p.workspace = vs.workspace.data_ptr()
    p.workspace_bytes = vs.workspace.numel()
    p.stream = _stream(vs.device)
    s = lib().fef_topn_step(ctypes.byref(p), _ptr(h), _ptr(W_vocab), vs.K, vs.block, ctypes.c_uint64(seed),
                            n_transfer, _ptr(vs.out_tokens), _ptr(vs.out_accept_len), _ptr(vs.out_remask))
    if s != FEF_OK:
        raise FefError(s, fef_last_error())
    return vs.out_tokens, vs.out_accept_len, vs.out_remask


class BlockDecoder:
    """Device-side state of Algorithm 2's outer loops for one block of B sequences: block mask,
    pass set, confidences, tokens, per-sequence pass and round counters.  `round()` enqueues one
    speculative round on top of that state and reads nothing back, so the rounds of a block can
    be queued back to back; a sequence that has finished its last pass is left untouched."""

    def __init__(self, step, n_pass, n_rm=-1, lowconf_scope=0, recorrupt_prob=1.0, greedy=False):
        self.vs, self.n_pass, self.n_rm, self.lowconf_scope = step, n_pass, n_rm, lowconf_scope
        self.recorrupt_prob, self.greedy = recorrupt_prob, greedy
        B, block, dev = step.B, step.block, step.device
        self.mask = torch.ones(B, block, dtype=torch.uint8, device=dev)
        self.pass_mask = torch.zeros(B, block, dtype=torch.uint8, device=dev)
        self.conf = torch.zeros(B, block, dtype=torch.float32, device=dev)
        self.tokens = torch.full((B, block), -1, dtype=torch.int32, device=dev)
        self.seq_pass = torch.zeros(B, dtype=torch.int32, device=dev)
        self.seq_rounds = torch.zeros(B, dtype=torch.int32, device=dev)

    def max_rounds(self):
        n_rm = self.vs.block // 2 if self.n_rm < 0 else min(self.n_rm, self.vs.block)
        return self.vs.block + (self.n_pass - 1) * max(n_rm, 1)

    def round(self, h_draft, h_target, W_vocab, seed, step, **kw):
        self.vs(h_draft, h_target, W_vocab, seed, step=step, n_rm=self.n_rm, lowconf_scope=self.lowconf_scope,
                recorrupt_prob=self.recorrupt_prob, greedy=self.greedy,
                mask_in=self.mask, pass_mask=self.pass_mask, conf=self.conf, n_pass=self.n_pass,
                seq_pass=self.seq_pass, seq_rounds=self.seq_rounds, tokens_state=self.tokens, **kw)
        # out_remask of this round is the mask of the next one (device-to-device, stream ordered)
        self.mask.copy_(self.vs.out_remask)


class Mx4Logits:
    """Logits of R rows through a vocabulary head held in 4 bits (fef_mx4_logits): codes [V, d / 2] and scales [V, d / 32], both
    uint8.  Holds the output of one shape; a call returns it (float32 [R, V]), or `out` if the caller gives one, whose rows may lie
    further apart."""

    def __init__(self, R, d, V, dtype="bf16", device="cuda"):
        self.R, self.d, self.V, self.device = R, d, V, torch.device(device)
        self.dtype = FEF_BF16 if dtype == "bf16" else FEF_F32
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.out = torch.empty(R, V, dtype=torch.float32, device=self.device)
        self._params = make_params(1, d, V, dtype=self.dtype)

    def __call__(self, h, codes, scales, temperature=1.0, out=None, head_events=None):
        R, d, V = self.R, self.d, self.V
        if out is None:
            out = self.out
        for t, shape, dt in ((h, (R, d), self.torch_dtype), (codes, (V, d // 2), torch.uint8), (scales, (V, d // 32), torch.uint8)):
            assert t.shape == shape and t.dtype == dt and t.is_contiguous() and t.is_cuda
        if out is not self.out:
            assert out.shape == (R, V) and out.dtype == torch.float32 and (V == 1 or out.stride(1) == 1) and out.is_cuda
        p = self._params
        p.temperature = temperature
        p.stream = _stream(self.device)
        p.ev_head_begin, p.ev_head_end = head_events if head_events is not None else (None, None)
        s = (_lib or lib()).fef_mx4_logits(p, h.data_ptr(), codes.data_ptr(), scales.data_ptr(), R, out.data_ptr(),
                                           out.stride(0) if R > 1 else V)
        if s != FEF_OK:
            raise FefError(s, fef_last_error())
        return out


class Edits:
    """What is done to the logits of B sequences (fef_edit_logits says what each means); everything is optional.
    history [B, H], history_len [B], prompt_len [B], prefix [B, K], bias_ids [B, n]: int32; repetition, presence, frequency [B],
    bias_values [B, n]: float32; allowed [B, 1 or K, ceil(V / 32)]: int32, bit v % 32 of word v / 32.  Holds the tensors, which it
    checks once; their contents may change between calls, the tensors themselves may not be exchanged."""

    _DTYPES = {"history": torch.int32, "history_len": torch.int32, "prompt_len": torch.int32, "prefix": torch.int32,
               "repetition": torch.float32, "presence": torch.float32, "frequency": torch.float32,
               "bias_ids": torch.int32, "bias_values": torch.float32, "allowed": torch.int32}
    __slots__ = (*_DTYPES, "sizes")

    def __init__(self, history=None, history_len=None, prompt_len=None, prefix=None, repetition=None, presence=None,
                 frequency=None, bias_ids=None, bias_values=None, allowed=None):
        given = (history, history_len, prompt_len, prefix, repetition, presence, frequency, bias_ids, bias_values, allowed)
        B = next((t.shape[0] for t in given if t is not None), None)
        for (name, dtype), t in zip(self._DTYPES.items(), given):
            if t is not None:
                assert t.dtype == dtype, f"{name} must be {dtype}"
                dims = 3 if name == "allowed" else 2 if name in ("history", "prefix", "bias_ids", "bias_values") else 1
                assert t.dim() == dims and t.shape[0] == B, f"{name} must have {dims} dimensions, the first of {B} sequences"
            object.__setattr__(self, name, t)
        assert (bias_ids is None) == (bias_values is None), "bias_ids and bias_values belong together"
        assert bias_ids is None or bias_ids.shape == bias_values.shape, "a value per id"
        assert history is not None or (history_len is None and prompt_len is None), "lengths of no history"
        for t in given:
            assert t is None or (t.is_contiguous() and t.is_cuda)
        # sequences, slots of prefix and masks, words of a mask (None: any), and the lists' lengths
        object.__setattr__(self, "sizes", (
            B, None if prefix is None else prefix.shape[1], None if allowed is None else allowed.shape[2],
            0 if history is None else history.shape[1], 0 if bias_ids is None else bias_ids.shape[1],
            0 if allowed is None else allowed.shape[1]))

    def __setattr__(self, name, value):
        raise AttributeError(f"the tensors of Edits are fixed: make another one to change {name}")


class EditLogits:
    """Edits of logits [B, K, V] of `dtype` ("f32" or "bf16", any strides whose last is 1).  Holds workspace, output (float32
    [B, K, V]) and log-sum-exps [B, K] of one shape; a call returns both outputs.  `out` may be given, and may be the logits."""

    def __init__(self, B, K, V, dtype="f32", device="cuda"):
        self.B, self.K, self.V, self.device = B, K, V, torch.device(device)
        self.dtype = FEF_BF16 if dtype == "bf16" else FEF_F32
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        p = fef_edit_params(struct_size=_EDIT_PARAMS_SIZE, B=B, K=K, V=V, dtype=self.dtype, temperature=1.0,
                            seq_stride=K * V, slot_stride=V, out_seq_stride=K * V, out_slot_stride=V)
        n = lib().fef_edit_workspace_bytes(ctypes.byref(p))
        if n == 0:
            raise FefError(FEF_ERR_INVALID_ARG, fef_last_error())
        self.workspace = torch.empty(n, dtype=torch.uint8, device=self.device)
        self.out = torch.empty(B, K, V, dtype=torch.float32, device=self.device)
        self.out_lse = torch.empty(B, K, dtype=torch.float32, device=self.device)
        self._words = (V + 31) // 32
        self._params = ctypes.create_string_buffer(_EDIT_PARAMS_SIZE)

    def __call__(self, logits, edits, temperature=1.0, out=None):
        B, K, V = shape = (self.B, self.K, self.V)
        if out is None:
            out = self.out
        assert logits.shape == shape and logits.dtype == self.torch_dtype and logits.is_cuda
        assert out.shape == shape and out.dtype == torch.float32 and out.is_cuda
        s, o = logits.stride(), out.stride()
        assert V == 1 or (s[2] == 1 and o[2] == 1)
        e = edits
        sequences, slots, words, H, n_bias, masks = e.sizes
        assert sequences in (None, B) and slots in (None, K) and words in (None, self._words) and masks in (0, 1, K)
        lists = [0 if t is None else t.data_ptr() for t in (
            e.history, e.history_len, e.prompt_len, e.prefix, e.repetition, e.presence, e.frequency, e.bias_ids, e.bias_values,
            e.allowed)]
        # one call over all fields in their order: a third of the time of a ctypes constructor
        _PACK_EDIT(self._params, 0, _EDIT_PARAMS_SIZE, B, K, V, self.dtype, temperature, s[0], s[1], o[0], o[1], H, *lists[:7],
                   n_bias, lists[7], lists[8], masks, lists[9], self.workspace.data_ptr(), self.workspace.numel(),
                   _stream(self.device))
        r = (_lib or lib()).fef_edit_logits(self._params, logits.data_ptr(), out.data_ptr(), self.out_lse.data_ptr())
        if r != FEF_OK:
            raise FefError(r, fef_last_error())
        return out, self.out_lse


class DrawLogits:
    """Truncation of the laws of logits [B, K, V] of `dtype` ("f32" or "bf16", any strides whose last is 1), and a token of each
    (fef_draw_logits).  Holds workspace and outputs of one shape; a call returns tokens [B, K] (int32), their probabilities, how many tokens
    are kept (int32), log-sum-exps, and the truncated logits (float32 [B, K, V], or None with write=False), or `out` if the caller gives
    one, which may not be the logits.  uniforms [B, K]: float32; without them a token is the smallest kept one.  Limits of each sequence,
    all optional: top_k [B] (int32), top_p, min_p [B] (float32); temperatures [B] (float32) stand in for `temperature`, 0 for the first
    token alone."""

    def __init__(self, B, K, V, dtype="f32", device="cuda", write=True):
        self.B, self.K, self.V, self.device = B, K, V, torch.device(device)
        self.dtype = FEF_BF16 if dtype == "bf16" else FEF_F32
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        p = fef_draw_params(struct_size=_DRAW_PARAMS_SIZE, B=B, K=K, V=V, dtype=self.dtype, temperature=1.0)
        n = lib().fef_draw_workspace_bytes(ctypes.byref(p))
        if n == 0:
            raise FefError(FEF_ERR_INVALID_ARG, fef_last_error())
        self.workspace = torch.empty(n, dtype=torch.uint8, device=self.device)
        self.out = torch.empty(B, K, V, dtype=torch.float32, device=self.device) if write else None
        self.out_lse, self.out_conf = (torch.empty(B, K, dtype=torch.float32, device=self.device) for _ in range(2))
        self.out_tokens, self.out_kept = (torch.empty(B, K, dtype=torch.int32, device=self.device) for _ in range(2))
        self._params = ctypes.create_string_buffer(_DRAW_PARAMS_SIZE)
        self._outputs = [t.data_ptr() for t in (self.out_lse, self.out_kept, self.out_tokens, self.out_conf, self.workspace)]

    def __call__(self, logits, uniforms=None, temperature=1.0, top_k=None, top_p=None, min_p=None, temperatures=None, out=None):
        B, K, V = shape = (self.B, self.K, self.V)
        if out is None:
            out = self.out
        assert logits.shape == shape and logits.dtype == self.torch_dtype and logits.is_cuda
        s = logits.stride()
        assert V == 1 or s[2] == 1
        o = (0, 0)
        if out is not None:
            assert out.shape == shape and out.dtype == torch.float32 and out.is_cuda and (V == 1 or out.stride(2) == 1)
            o = out.stride()
        lists = []
        for t, dtype, size in ((temperatures, torch.float32, (B,)), (top_k, torch.int32, (B,)), (top_p, torch.float32, (B,)),
                               (min_p, torch.float32, (B,)), (uniforms, torch.float32, (B, K))):
            assert t is None or (t.dtype == dtype and t.shape == size and t.is_contiguous() and t.is_cuda)
            lists.append(0 if t is None else t.data_ptr())
        _PACK_DRAW(self._params, 0, _DRAW_PARAMS_SIZE, B, K, V, self.dtype, temperature, s[0], s[1], o[0], o[1], *lists, *self._outputs,
                   self.workspace.numel(), _stream(self.device))
        r = (_lib or lib()).fef_draw_logits(self._params, logits.data_ptr(), _ptr(out))
        if r != FEF_OK:
            raise FefError(r, fef_last_error())
        return self.out_tokens, self.out_conf, self.out_kept, self.out_lse, out


class VerifyLogits:
    """The speculative round on logits that the program has (fef_verify_logits).  Holds the logits of one shape, [2, B, K, ld] with
    the draft rows first: `draft_logits` and `target_logits` are the two [B, K, V] views that Mx4Logits and EditLogits can write
    into.  `diag=True` also returns draft tokens, alpha, residual mass, lse and confidences."""

    def __init__(self, B, K, block, V, device="cuda", diag=False):
        self.B, self.K, self.block, self.V, self.device = B, K, block, V, torch.device(device)
        dev = self.device
        self.ld = (V + 63) // 64 * 64
        self.logits = torch.zeros(2, B, K, self.ld, dtype=torch.float32, device=dev)
        self.draft_logits, self.target_logits = self.logits[0, :, :, :V], self.logits[1, :, :, :V]
        self.out_tokens = torch.empty(B, K, dtype=torch.int32, device=dev)
        self.out_accept_len = torch.empty(B, dtype=torch.int32, device=dev)
        self.out_remask = torch.empty(B, block, dtype=torch.uint8, device=dev)
        self.diag = {}
        if diag:
            self.diag = {
                "draft_tokens": torch.empty(B, K, dtype=torch.int32, device=dev),
                "alpha": torch.empty(B, K, dtype=torch.float32, device=dev),
                "resid_mass": torch.empty(B, K, dtype=torch.float32, device=dev),
                "lse": torch.empty(2, B, K, dtype=torch.float32, device=dev),
                "conf_tok": torch.empty(B, K, dtype=torch.float32, device=dev),
            }
        p = self._params()
        n = lib().fef_verify_logits_workspace_bytes(ctypes.byref(p), K, block)
        if n == 0:
            raise FefError(FEF_ERR_INVALID_ARG, fef_last_error())
        self.workspace = torch.empty(n, dtype=torch.uint8, device=dev)

    def _params(self, **kw):
        p = make_params(self.B, 64, self.V, **kw)
        for name, t in self.diag.items():
            setattr(p, "diag_" + name, t.data_ptr())
        return p

    def __call__(self, seed, *, step=0, seq_base=0, pos_base=0, n_rm=-1, final_pass=False, lowconf_scope=0, mask_in=None,
                 pass_mask=None, conf=None, draft_tokens=None, n_pass=0, seq_pass=None, seq_rounds=None, tokens_state=None,
                 phase=FEF_PHASE_FUSED, recorrupt_prob=1.0, greedy=False):
        B, K, block = self.B, self.K, self.block
        p = self._params(step=step, seq_base=seq_base, pos_base=pos_base, n_rm=n_rm, final_pass=final_pass, lowconf_scope=lowconf_scope)
        for name, t, dt, shape in (("mask_in", mask_in, torch.uint8, (B, block)), ("pass_mask", pass_mask, torch.uint8, (B, block)),
                                   ("conf", conf, torch.float32, (B, block)), ("draft_tokens", draft_tokens, torch.int32, (B, K)),
                                   ("seq_pass", seq_pass, torch.int32, (B,)), ("seq_rounds", seq_rounds, torch.int32, (B,)),
                                   ("tokens_state", tokens_state, torch.int32, (B, block))):
            if t is not None:
                assert t.dtype == dt and t.shape == shape and t.is_contiguous() and t.is_cuda
                setattr(p, name, t.data_ptr())
        p.n_pass, p.phase, p.recorrupt_prob, p.greedy = n_pass, phase, recorrupt_prob, int(greedy)
        p.workspace, p.workspace_bytes, p.stream = self.workspace.data_ptr(), self.workspace.numel(), _stream(self.device)
        s = lib().fef_verify_logits(ctypes.byref(p), _ptr(self.logits), self.ld, K, block, seed & 0xFFFFFFFFFFFFFFFF,
                                    _ptr(self.out_tokens), _ptr(self.out_accept_len), _ptr(self.out_remask))
        if s != FEF_OK:
            raise FefError(s, fef_last_error())
        return self.out_tokens, self.out_accept_len, self.out_remask


class AdamW:
    """One AdamW step at a time over a list of parameters (fef_adamw_step), all bf16 or all float32, contiguous.  `grads`: their
    gradients, all of one of these types.  states "f32", "8bit" (e4m3 codes and a scale per 256 elements), or "8bit-reciprocal": the same in
    the bits of elementwise torch on the GPU, whose quotients of codes and scales are products with reciprocals.  `master`: True for
    float32 copies of bf16 parameters, made here, or a list of them.  `weight_decay`: one for all or one for each.  m, v (and m_scale,
    v_scale) go on from given states; left out, they start at zero.  `schedule` (device float32 [3]: lr, 1 / (1 - beta1^t),
    1 / sqrt(1 - beta2^t)) replaces lr and the step count, `grad_scale` (device float32 [1]) multiplies the gradients.
    Holds the tensors; their contents may change between steps (a backward pass writes the gradients), the tensors themselves may
    not be exchanged.  `lr` and `step_count` may be set between steps; a step adds one to `step_count` first."""

    def __init__(self, params, grads, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, states="f32", master=None, m=None, v=None,
                 m_scale=None, v_scale=None, step=0, schedule=None, grad_scale=None):
        self.params, self.grads, self.lr, self.step_count = list(params), list(grads), lr, step
        n = len(self.params)
        assert n and len(self.grads) == n, "a gradient per parameter"
        assert states in ("f32", "8bit", "8bit-reciprocal")
        self.device = self.params[0].device
        eight = states != "f32"

        def made(given, default):
            out = [default(p) for p in self.params] if given is None or given is True or len(given) == 0 else list(given)
            assert len(out) == n, "one for each parameter"
            return out

        def blocks(p):
            return (p.numel() + 255) // 256

        self.master = made(master, lambda p: p.float()) if master is True or master else None
        state = torch.float8_e4m3fn if eight else torch.float32
        self.m = made(m, lambda p: torch.zeros(p.numel(), dtype=torch.uint8 if eight else state, device=p.device).view(state))
        self.v = made(v, lambda p: torch.zeros(p.numel(), dtype=torch.uint8 if eight else state, device=p.device).view(state))
        if eight:
            self.m_scale = made(m_scale, lambda p: torch.zeros(blocks(p), device=p.device))
            self.v_scale = made(v_scale, lambda p: torch.zeros(blocks(p), device=p.device))
        else:
            assert not m_scale and not v_scale, "scales belong to states in 8 bits"
            self.m_scale = self.v_scale = None
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
        assert len(decay) == n, "one weight decay for each parameter"
        kinds = (torch.bfloat16, torch.float32)
        assert self.params[0].dtype in kinds and self.grads[0].dtype in kinds
        assert self.master is None or self.params[0].dtype == torch.bfloat16, "float32 copies are for bf16 parameters"
        self._tensors = (fef_adamw_tensor * n)()
        for i, p in enumerate(self.params):
            count = p.numel()
            for t, kind, size in ((p, self.params[0].dtype, count), (self.grads[i], self.grads[0].dtype, count),
                                  (self.master and self.master[i], torch.float32, count), (self.m[i], state, count), (self.v[i], state, count),
                                  (self.m_scale and self.m_scale[i], torch.float32, blocks(p)),
                                  (self.v_scale and self.v_scale[i], torch.float32, blocks(p))):
                assert t is None or (t.dtype == kind and t.numel() == size and t.is_contiguous() and t.device == self.device and t.is_cuda)
            e = self._tensors[i]
            e.param, e.grad, e.m, e.v = p.data_ptr(), self.grads[i].data_ptr(), self.m[i].data_ptr(), self.v[i].data_ptr()
            e.master = _ptr(self.master[i]) if self.master else None
            e.m_scale, e.v_scale = (self.m_scale[i].data_ptr(), self.v_scale[i].data_ptr()) if eight else (None, None)
            e.n, e.weight_decay = count, decay[i]
        for t, size in ((schedule, 3), (grad_scale, 1)):
            assert t is None or (t.dtype == torch.float32 and t.numel() == size and t.is_contiguous() and t.is_cuda)
        self.schedule, self.grad_scale = schedule, grad_scale
        self._params = fef_adamw_params(ctypes.sizeof(fef_adamw_params), FEF_BF16 if self.params[0].dtype == torch.bfloat16 else FEF_F32,
                                        FEF_BF16 if self.grads[0].dtype == torch.bfloat16 else FEF_F32,
                                        {"f32": FEF_STATE_F32, "8bit": FEF_STATE_E4M3}.get(states, FEF_STATE_E4M3_RECIPROCAL), lr, betas[0], betas[1], eps, max(step, 1), _ptr(schedule),
                                        _ptr(grad_scale), None)

    def step(self):
        p = self._params
        p.lr, p.step, p.stream = self.lr, self.step_count + 1, _stream(self.device)
        r = (_lib or lib()).fef_adamw_step(ctypes.byref(p), self._tensors, len(self.params))
        if r != FEF_OK:
            raise FefError(r, fef_last_error())
        self.step_count += 1
