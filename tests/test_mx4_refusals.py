"""fef_mx4_logits: what it refuses, on the host before any HIP call (the pointers are fake)."""
import ctypes
import os

import pytest

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.skipif(not os.path.exists(fb.LIB_PATH), reason="libfef.so not built")


def _call(h=0x1000, codes=0x1000, scales=0x1000, out=0x1000, R=4, ld=1000, **params):
    p = fb.make_params(1, 128, 1000)
    for k, v in params.items():
        setattr(p, k, v)
    return fb.lib().fef_mx4_logits(p, h, codes, scales, R, out, ld)


@pytest.mark.parametrize("bad,word", [
    (dict(struct_size=8), "struct_size"), (dict(R=0), "R ="), (dict(R=(1 << 24) + 1), "R ="), (dict(V=0, ld=1), "positive"),
    (dict(d=0), "positive"), (dict(d=48), "32"), (dict(d=(1 << 20) + 32), "32"), (dict(d=-32), "positive"), (dict(dtype=2), "dtype"), (dict(temperature=0.0), "temperature"),
    (dict(temperature=float("nan")), "temperature"), (dict(temperature=float("inf")), "temperature"), (dict(h=None), "NULL"),
    (dict(codes=None), "NULL"), (dict(scales=None), "NULL"), (dict(out=None), "NULL"), (dict(h=0x1008), "16-byte"),
    (dict(codes=0x1001), "16-byte"), (dict(scales=0x1004), "16-byte"), (dict(out=0x1002), "4-byte"), (dict(ld=999), "ld"),
    (dict(ld=-1), "ld"), (dict(ld=(1 << 40) + 1), "ld"), (dict(ev_head_begin=16), "together")])
def test_refusals(bad, word):
    assert _call(**bad) == fb.FEF_ERR_INVALID_ARG
    assert word in fb.fef_last_error()


def test_null_params():
    assert fb.lib().fef_mx4_logits(ctypes.POINTER(fb.fef_params)(), 0x1000, 0x1000, 0x1000, 1, 0x1000, 1) == fb.FEF_ERR_INVALID_ARG
