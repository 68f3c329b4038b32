"""fef_head_cross_entropy_grad: what it refuses, on the host before any HIP call (the pointers are fake); sizes of its workspace."""
import ctypes
import os

import pytest

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.skipif(not os.path.exists(fb.LIB_PATH), reason="libfef.so not built")
H, W, L, WT, CE, LOSS, GH, GW = (0x10000000 * i for i in range(1, 9))


def _params(**kw):
    p = fb.make_params(1, 64, 100)
    p.workspace, p.workspace_bytes = 0x100, 1 << 50
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _call(p, R=10, h=H, w=W, labels=L, weights=WT, ce=CE, loss=LOSS, gh=GH, gw=GW):
    return fb.lib().fef_head_cross_entropy_grad(ctypes.byref(p), h, w, labels, weights, R, ce, loss, gh, gw)


@pytest.mark.parametrize("bad,word", [
    (dict(struct_size=4), "struct_size"), (dict(V=0), "positive"), (dict(d=0), "positive"), (dict(V=(1 << 29) + 1), "2^29"), (dict(d=96), "multiple of 64"),
    (dict(d=(1 << 20) + 64), "2^20"), (dict(dtype=5), "dtype"), (dict(temperature=0.0), "temperature"), (dict(temperature=1e-39), "temperature"),
    (dict(temperature=float("nan")), "temperature"), (dict(ev_head_begin=0x1000, ev_head_end=0x1000), "ev_head")])
def test_refusals(bad, word):
    assert _call(_params(**bad)) == fb.FEF_ERR_INVALID_ARG
    assert word in fb.fef_last_error()


def test_rows_and_variants():
    for R in (0, -1, (1 << 24) + 1):
        assert _call(_params(), R=R) == fb.FEF_ERR_INVALID_ARG
    for bad in (dict(gemm_variant=fb.FEF_GEMM_STREAM), dict(gemm_variant=fb.FEF_GEMM_F32), dict(dtype=fb.FEF_F32, gemm_variant=fb.FEF_GEMM_TILED256)):
        assert _call(_params(**bad)) == fb.FEF_ERR_UNSUPPORTED


@pytest.mark.parametrize("bad,word", [
    (dict(h=None), "NULL"), (dict(w=None), "NULL"), (dict(labels=None), "NULL"), (dict(ce=None), "NULL"), (dict(gh=None, gw=None), "both"),
    (dict(h=H + 8), "16-byte"), (dict(w=W + 2), "16-byte"), (dict(gh=GH + 8), "16-byte"), (dict(gw=GW + 4), "16-byte"), (dict(labels=L + 2), "4-byte"),
    (dict(weights=WT + 1), "4-byte"), (dict(loss=LOSS + 2), "4-byte"), (dict(gh=H), "overlap"), (dict(gw=W), "overlap"),
    (dict(gw=W + 100 * 64 * 2 - 16), "overlap"), (dict(gh=GW + 16), "overlap"), (dict(gw=H + 16), "overlap"), (dict(gh=W + 16), "overlap")])
def test_refused_pointers(bad, word):
    assert _call(_params(), **bad) == fb.FEF_ERR_INVALID_ARG
    assert word in fb.fef_last_error()


def test_workspace():
    need = fb.lib().fef_cross_entropy_grad_workspace_bytes(ctypes.byref(_params()), 10)
    assert need > 0 and need % 256 == 0
    for bad in (dict(workspace=None), dict(workspace=0x110), dict(workspace_bytes=need - 1)):
        assert _call(_params(**bad)) == fb.FEF_ERR_WORKSPACE
    assert fb.lib().fef_cross_entropy_grad_workspace_bytes(ctypes.byref(_params(V=0)), 10) == 0
    big = _params(d=4096, V=126464)
    one, many = (fb.lib().fef_cross_entropy_grad_workspace_bytes(ctypes.byref(big), R) for R in (8192, 1 << 20))
    assert one < 13 << 30 and many - one < 3 << 30  # a block of rows at a time, and float32 sums of grad_w
