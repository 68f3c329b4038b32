"""fef_edit_logits: what it refuses, on the host before any HIP call (the pointers are fake); sizes of its workspace."""
import ctypes
import os

import pytest

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.skipif(not os.path.exists(fb.LIB_PATH), reason="libfef.so not built")


def _params(**kw):
    p = fb.fef_edit_params(struct_size=ctypes.sizeof(fb.fef_edit_params), B=2, K=3, V=100, dtype=fb.FEF_F32, temperature=1.0, seq_stride=300,
                           slot_stride=100, out_seq_stride=300, out_slot_stride=100, workspace=0x10000, workspace_bytes=1 << 30)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("bad,word", [
    (dict(struct_size=4), "struct_size"), (dict(B=0), "B and V"), (dict(V=0), "B and V"), (dict(K=0), "K ="), (dict(K=65), "K ="),
    (dict(B=1 << 23), "2^24"), (dict(dtype=7), "dtype"), (dict(temperature=-1.0), "temperature"), (dict(temperature=float("nan")), "temperature"),
    (dict(history_max=-1), "negative"), (dict(n_bias=-1), "negative"), (dict(masks=2), "masks"), (dict(masks=-1), "masks"),
    (dict(seq_stride=-1), "strides"), (dict(slot_stride=(1 << 40) + 1), "strides"), (dict(out_slot_stride=99), "overlap"),
    (dict(out_seq_stride=299), "overlap"), (dict(out_seq_stride=0), "overlap"), (dict(history_max=5), "history"), (dict(n_bias=1), "bias"),
    (dict(n_bias=1, bias_ids=0x1000), "bias"), (dict(masks=1), "allowed"), (dict(prefix=0x1002), "4-byte"), (dict(masks=3, allowed=0x1001), "4-byte")])
def test_refusals(bad, word):
    assert fb.lib().fef_edit_logits(ctypes.byref(_params(**bad)), 0x1000, 0x2000, 0x3000) == fb.FEF_ERR_INVALID_ARG
    assert word in fb.fef_last_error()


@pytest.mark.parametrize("logits,out,lse,kw", [
    (None, 0x2000, 0x3000, {}), (0x1000, None, 0x3000, {}), (0x1002, 0x2000, 0x3000, {}), (0x1001, 0x2000, 0x3000, dict(dtype=fb.FEF_BF16)),
    (0x1000, 0x2001, 0x3000, {}), (0x1000, 0x2000, 0x3002, {}), (0x1000, 0x1000, 0x3000, dict(dtype=fb.FEF_BF16)),
    (0x1000, 0x1000, 0x3000, dict(seq_stride=400)), (0x1000, 0x1000, 0x3000, dict(slot_stride=0))])
def test_refused_pointers(logits, out, lse, kw):
    assert fb.lib().fef_edit_logits(ctypes.byref(_params(**kw)), logits, out, lse) == fb.FEF_ERR_INVALID_ARG


def test_workspace():
    p = _params()
    need = fb.lib().fef_edit_workspace_bytes(p)
    assert need > 0 and need % 256 == 0
    for bad in (dict(workspace=None), dict(workspace=0x10010), dict(workspace_bytes=need - 1)):
        assert fb.lib().fef_edit_logits(ctypes.byref(_params(**bad)), 0x1000, 0x2000, 0x3000) == fb.FEF_ERR_WORKSPACE
    assert fb.lib().fef_edit_workspace_bytes(_params(K=0)) == 0
    assert fb.lib().fef_edit_workspace_bytes(_params(B=1 << 20, out_seq_stride=300)) >= 1 << 20
    # slots outside, sequences inside is a layout too
    assert fb.lib().fef_edit_workspace_bytes(_params(out_seq_stride=100, out_slot_stride=200)) == need


def test_edits_checks_types():
    import torch
    with pytest.raises(AssertionError):
        fb.Edits(history=torch.zeros(1, 4))
    with pytest.raises(AssertionError):
        fb.Edits(bias_ids=torch.zeros(1, 4, dtype=torch.int32))
    with pytest.raises(AssertionError):
        fb.Edits(prompt_len=torch.zeros(1, dtype=torch.int32))


def test_the_packed_parameters_are_the_struct():
    """EditLogits writes the fields in one go, in the order and alignment of fef_edit_params."""
    names = [f[0] for f in fb.fef_edit_params._fields_]
    values = [ctypes.sizeof(fb.fef_edit_params), *range(2, 6), 0.5, *range(11, 11 + len(names) - 6)]
    buffer = ctypes.create_string_buffer(ctypes.sizeof(fb.fef_edit_params))
    fb._PACK_EDIT(buffer, 0, *values)
    p = fb.fef_edit_params.from_buffer(buffer)
    assert [getattr(p, n) for n in names] == values


def test_the_tensors_of_edits_are_fixed():
    e = fb.Edits()
    with pytest.raises(AttributeError):
        e.history = None
