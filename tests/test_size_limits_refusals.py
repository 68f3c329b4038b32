"""Sizes at which the 32-bit indices of the kernels behind fef_mx4_logits, fef_edit_logits and fef_verify_logits would wrap (a walk over a
list that starts again below zero, a tile past the last one) are refused on the host, before any HIP call (the pointers are fake)."""
import ctypes
import os

import pytest

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.skipif(not os.path.exists(fb.LIB_PATH), reason="libfef.so not built")
LAST = 2 ** 31 - 1


def _edit(**kw):
    V = kw.get("V", 100)
    p = fb.fef_edit_params(struct_size=ctypes.sizeof(fb.fef_edit_params), B=1, K=1, V=V, dtype=fb.FEF_F32, temperature=1.0, seq_stride=V,
                           slot_stride=V, out_seq_stride=V, out_slot_stride=V, workspace=0x10000, workspace_bytes=16)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("bad,word", [
    (dict(V=2 ** 29 + 1), "2^29"), (dict(V=LAST), "2^29"), (dict(history_max=LAST, history=0x1000, repetition=0x1000), "2^30"),
    (dict(n_bias=LAST, bias_ids=0x1000, bias_values=0x1000), "2^30"), (dict(history_max=2 ** 30 + 1, history=0x1000), "2^30")])
def test_edits(bad, word):
    p = _edit(**bad)
    assert fb.lib().fef_edit_logits(ctypes.byref(p), 0x1000, 0x2000, 0x3000) == fb.FEF_ERR_INVALID_ARG
    assert word in fb.fef_last_error()
    assert fb.lib().fef_edit_workspace_bytes(ctypes.byref(p)) == 0


@pytest.mark.parametrize("good", [dict(V=2 ** 29), dict(history_max=2 ** 30, history=0x1000), dict(n_bias=2 ** 30, bias_ids=0x1000, bias_values=0x1000)])
def test_edits_up_to_the_limit(good):
    """Nothing but the 16 bytes of workspace is refused."""
    assert fb.lib().fef_edit_logits(ctypes.byref(_edit(**good)), 0x1000, 0x2000, 0x3000) == fb.FEF_ERR_WORKSPACE


@pytest.mark.parametrize("V", [2 ** 29 + 1, LAST])
def test_head_and_round(V):
    p = fb.make_params(1, 32, V)
    assert fb.lib().fef_mx4_logits(p, 0x1000, 0x1000, 0x1000, 1, 0x1000, V) == fb.FEF_ERR_INVALID_ARG
    assert "2^29" in fb.fef_last_error()
    p.workspace, p.workspace_bytes = 0x10000, 16
    assert fb.lib().fef_verify_logits_workspace_bytes(ctypes.byref(p), 1, 1) == 0
    assert fb.lib().fef_verify_logits(ctypes.byref(p), 0x1000, 2 ** 32, 1, 1, 0, 0x1000, 0x1000, 0x1000) == fb.FEF_ERR_INVALID_ARG
    assert "2^29" in fb.fef_last_error()


def test_round_up_to_the_limit():
    p = fb.make_params(1, 64, 2 ** 29)
    p.workspace, p.workspace_bytes = 0x10000, 16
    assert fb.lib().fef_verify_logits(ctypes.byref(p), 0x1000, 2 ** 29, 1, 1, 0, 0x1000, 0x1000, 0x1000) == fb.FEF_ERR_WORKSPACE


@pytest.mark.parametrize("tau", [1e-45, 1e-40, 2.9e-39])
def test_a_temperature_without_a_reciprocal(tau):
    """1 / tau would be infinite, and a logit of 0 NaN."""
    assert fb.lib().fef_edit_logits(ctypes.byref(_edit(temperature=tau)), 0x1000, 0x2000, 0x3000) == fb.FEF_ERR_INVALID_ARG
    assert "reciprocal" in fb.fef_last_error()
    p = fb.make_params(1, 32, 100, temperature=tau)
    assert fb.lib().fef_mx4_logits(p, 0x1000, 0x1000, 0x1000, 1, 0x1000, 100) == fb.FEF_ERR_INVALID_ARG
    assert "reciprocal" in fb.fef_last_error()
