"""fef_draw_logits: what it refuses, on the host before any HIP call (the pointers are fake); sizes of its workspace."""
import ctypes
import os

import pytest

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.skipif(not os.path.exists(fb.LIB_PATH), reason="libfef.so not built")


def _params(**kw):
    p = fb.fef_draw_params(struct_size=ctypes.sizeof(fb.fef_draw_params), B=2, K=3, V=100, dtype=fb.FEF_F32, temperature=1.0, seq_stride=300,
                           slot_stride=100, out_seq_stride=300, out_slot_stride=100, workspace=0x10000, workspace_bytes=1 << 40)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("bad,word", [
    (dict(struct_size=4), "struct_size"), (dict(B=0), "B and V"), (dict(V=0), "B and V"), (dict(V=(1 << 29) + 1), "2^29"), (dict(K=0), "K ="),
    (dict(K=65), "K ="), (dict(B=1 << 20), "2^21"), (dict(dtype=7), "dtype"), (dict(temperature=0.0), "temperature"),
    (dict(temperature=float("nan")), "temperature"), (dict(temperature=1e-39), "temperature"), (dict(seq_stride=-1), "strides"),
    (dict(slot_stride=(1 << 40) + 1), "strides"), (dict(out_slot_stride=99), "overlap"), (dict(out_seq_stride=299), "overlap"),
    (dict(top_k=0x1002), "4-byte"), (dict(uniforms=0x1001), "4-byte"), (dict(out_conf=0x1002), "4-byte"), (dict(temperatures=0x1002), "4-byte")])
def test_refusals(bad, word):
    assert fb.lib().fef_draw_logits(ctypes.byref(_params(**bad)), 0x1000, 0x2000) == fb.FEF_ERR_INVALID_ARG
    assert word in fb.fef_last_error()


@pytest.mark.parametrize("logits,out,kw", [(None, 0x2000, {}), (0x1002, 0x2000, {}), (0x1001, 0x2000, dict(dtype=fb.FEF_BF16)), (0x1000, 0x2002, {}),
                                           (0x1000, 0x1000, {})])
def test_refused_pointers(logits, out, kw):
    assert fb.lib().fef_draw_logits(ctypes.byref(_params(**kw)), logits, out) == fb.FEF_ERR_INVALID_ARG


@pytest.mark.parametrize("logits,out,kw", [(0x1000, 0x1000 + 4 * 599, {}), (0x1000 + 4 * 599, 0x1000, {}), (0x1000, 0x1000 + 4 * 299, dict(dtype=fb.FEF_BF16)),
                                           (0x1000, 0x1000 + 4 * 100, dict(seq_stride=600, slot_stride=200, out_seq_stride=600, out_slot_stride=199)),
                                           (0x1000, 0x1000 + 4 * 100, dict(seq_stride=0, slot_stride=0, out_seq_stride=0, out_slot_stride=0, B=1, K=1, V=101))])
def test_an_output_that_meets_the_logits(logits, out, kw):
    assert fb.lib().fef_draw_logits(ctypes.byref(_params(**kw)), logits, out) == fb.FEF_ERR_INVALID_ARG
    assert "overlap" in fb.fef_last_error()


@pytest.mark.parametrize("logits,out,kw", [(0x1000, 0x1000 + 4 * 600, {}), (0x1000 + 4 * 600, 0x1000, {}),
                                           (0x1000, 0x1000 + 4 * 100, dict(seq_stride=600, slot_stride=200, out_seq_stride=600, out_slot_stride=200))])
def test_an_output_beside_the_logits_gets_past_this_check(logits, out, kw):
    """What is refused is the workspace, which is looked at later."""
    assert fb.lib().fef_draw_logits(ctypes.byref(_params(workspace=None, **kw)), logits, out) == fb.FEF_ERR_WORKSPACE


def test_workspace():
    need = fb.lib().fef_draw_workspace_bytes(ctypes.byref(_params()))
    assert need > 0 and need % 256 == 0
    for bad in (dict(workspace=None), dict(workspace=0x10010), dict(workspace_bytes=need - 1)):
        assert fb.lib().fef_draw_logits(ctypes.byref(_params(**bad)), 0x1000, 0x2000) == fb.FEF_ERR_WORKSPACE
    assert fb.lib().fef_draw_workspace_bytes(ctypes.byref(_params(K=0))) == 0


def test_the_packed_parameters_are_the_struct():
    names = [f[0] for f in fb.fef_draw_params._fields_]
    values = [ctypes.sizeof(fb.fef_draw_params), *range(2, 6), 0.5, *range(11, 11 + len(names) - 6)]
    buffer = ctypes.create_string_buffer(ctypes.sizeof(fb.fef_draw_params))
    fb._PACK_DRAW(buffer, 0, *values)
    p = fb.fef_draw_params.from_buffer(buffer)
    assert [getattr(p, n) for n in names] == values
