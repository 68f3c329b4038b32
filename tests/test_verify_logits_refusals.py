"""fef_verify_logits: what it refuses, on the host before any HIP call (the pointers are fake); its workspace."""
import ctypes
import os

import pytest

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.skipif(not os.path.exists(fb.LIB_PATH), reason="libfef.so not built")


def _call(logits=0x1000, ld=1024, K=4, block=8, out=0x1000, **params):
    p = fb.make_params(2, 1, 1000, dtype=77, temperature=-1.0, gemm_variant=99)   # fields that the call does not read
    p.workspace, p.workspace_bytes = 0x10000, 1 << 30
    for k, v in params.items():
        setattr(p, k, v)
    return fb.lib().fef_verify_logits(ctypes.byref(p), logits, ld, K, block, 0, out, out, out)


@pytest.mark.parametrize("bad,word", [
    (dict(struct_size=4), "struct_size"), (dict(B=0), "B, d, V"), (dict(V=0), "B, d, V"), (dict(K=0), "K="), (dict(K=9), "K="),
    (dict(logits=None), "logits"), (dict(logits=0x1008), "16-byte"), (dict(ld=1000), "ld"), (dict(ld=960), "ld"), (dict(ld=-64), "ld"),
    (dict(out=None), "out_tokens"), (dict(recorrupt_prob=0.0), "recorrupt"), (dict(greedy=2), "greedy"), (dict(phase=3), "phase"),
    (dict(ev_head_begin=8, ev_head_end=8), "ev_head"), (dict(lowconf_scope=1), "conf")])
def test_refusals(bad, word):
    assert _call(**bad) == fb.FEF_ERR_INVALID_ARG
    assert word in fb.fef_last_error()


@pytest.mark.parametrize("bad", [dict(workspace=None), dict(workspace=0x10010), dict(workspace_bytes=100)])
def test_workspace_is_checked(bad):
    assert _call(**bad) == fb.FEF_ERR_WORKSPACE


def test_workspace_holds_no_logits():
    small, head = fb.make_params(4, 64, 100000), fb.make_params(4, 64, 100000, gemm_variant=fb.FEF_GEMM_TILED256)
    n = fb.lib().fef_verify_logits_workspace_bytes(ctypes.byref(small), 8, 32)
    assert 0 < n < 1 << 20 and n % 256 == 0
    assert n + 64 * 100032 * 4 <= fb.fef_workspace_bytes(head, 8, 32)
    assert fb.lib().fef_verify_logits_workspace_bytes(ctypes.byref(small), 0, 32) == 0
