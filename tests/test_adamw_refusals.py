"""fef_adamw_step: what it refuses, on the host before any HIP call (the pointers are fake)."""
import ctypes
import os

import pytest

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.skipif(not os.path.exists(fb.LIB_PATH), reason="libfef.so not built")


def _params(**kw):
    p = fb.fef_adamw_params(struct_size=ctypes.sizeof(fb.fef_adamw_params), dtype=fb.FEF_BF16, grad_dtype=fb.FEF_BF16, state_dtype=fb.FEF_STATE_F32,
                            lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _tensors(*changes):
    """Tensors of 100 elements, 0x10000 bytes apart."""
    ts = (fb.fef_adamw_tensor * len(changes))()
    for i, change in enumerate(changes):
        base = 0x100000 * (i + 1)
        fields = dict(param=base, grad=base + 0x10000, m=base + 0x20000, v=base + 0x30000, n=100, weight_decay=0.1)
        fields.update(change)
        for k, v in fields.items():
            setattr(ts[i], k, v)
    return ts


def _refused(p, ts, word, count=None):
    count = len(ts) if count is None else count
    assert fb.lib().fef_adamw_step(ctypes.byref(p), ts, count) == fb.FEF_ERR_INVALID_ARG
    assert word in fb.fef_last_error()


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("bad,word", [
    (dict(struct_size=4), "struct_size"), (dict(dtype=2), "dtype"), (dict(grad_dtype=-1), "grad_dtype"), (dict(state_dtype=2), "state_dtype"),
    (dict(lr=NAN), "lr"), (dict(lr=INF), "lr"), (dict(beta1=1.0), "beta1"), (dict(beta1=-0.1), "beta1"), (dict(beta2=NAN), "beta1"),
    (dict(beta2=1.0 - 1e-12), "beta1"), (dict(eps=0.0), "eps"), (dict(eps=1e-60), "eps"), (dict(eps=NAN), "eps"), (dict(step=0), "step"),
    (dict(schedule=0x1002), "4-byte"), (dict(grad_scale=0x1001), "4-byte")])
def test_refused_parameters(bad, word):
    _refused(_params(**bad), _tensors({}), word)


@pytest.mark.parametrize("bad,word", [
    (dict(n=-1), "n ="), (dict(n=(1 << 36) + 1), "n ="), (dict(weight_decay=-0.1), "weight_decay"), (dict(weight_decay=NAN), "weight_decay"),
    (dict(param=None), "NULL"), (dict(grad=None), "NULL"), (dict(m=None), "NULL"), (dict(v=None), "NULL"), (dict(m_scale=0x5000), "8 bits"),
    (dict(param=0x1001), "aligned"), (dict(grad=0x1001), "aligned"), (dict(m=0x1002), "aligned"), (dict(master=0x1002), "aligned")])
def test_refused_tensors(bad, word):
    _refused(_params(), _tensors({}, bad), word)


def test_states_in_8_bits_need_scales():
    p = _params(state_dtype=fb.FEF_STATE_E4M3)
    _refused(p, _tensors({}), "8 bits")
    _refused(p, _tensors(dict(m_scale=0x5000)), "8 bits")
    _refused(p, _tensors(dict(m_scale=0x5002, v_scale=0x6000)), "aligned")


def test_copies_are_for_bf16():
    _refused(_params(dtype=fb.FEF_F32), _tensors(dict(master=0x5000)), "master")


def test_counts():
    _refused(_params(), _tensors({}), "count", -1)
    _refused(_params(), None, "NULL", 1)
    _refused(_params(), _tensors({}), "count", 65537)
    assert fb.lib().fef_adamw_step(ctypes.byref(_params()), None, 0) == fb.FEF_OK
    empty = _tensors(dict(n=0, param=None, grad=None, m=None, v=None))
    assert fb.lib().fef_adamw_step(ctypes.byref(_params()), empty, 1) == fb.FEF_OK


BASE = 0x100000


@pytest.mark.parametrize("changes", [
    [{}, dict(param=BASE)],                       # the same tensor twice
    [dict(m=BASE + 196)],                         # a state begins in the parameter's last elements
    [{}, dict(master=BASE + 0x30000 + 396)],      # ... in another tensor's state
    [dict(grad=BASE)],                            # the gradient is the parameter
    [{}, dict(grad=BASE + 0x20000)],              # ... another tensor's state
    [dict(n=0x20000)]])                           # the parameter reaches into the gradient
def test_overlaps(changes):
    _refused(_params(), _tensors(*changes), "overlap")


def test_gradient_scale_in_a_parameter():
    _refused(_params(grad_scale=BASE + 4), _tensors({}), "overlap")
    _refused(_params(schedule=BASE + 196), _tensors({}), "overlap")
