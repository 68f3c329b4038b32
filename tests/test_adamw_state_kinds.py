"""fef_adamw_step: which kinds of states there are, on the host before any HIP call (the pointers are fake)."""
import ctypes

import pytest

from paper_2605_14305_amd import binding as fb
from test_adamw_refusals import _params, _refused, _tensors, pytestmark  # noqa: F401


def test_reciprocals_are_states_in_8_bits():
    p = _params(state_dtype=fb.FEF_STATE_E4M3_RECIPROCAL)
    _refused(p, _tensors({}), "8 bits")
    _refused(p, _tensors(dict(m_scale=0x5002, v_scale=0x6000)), "aligned")
    _refused(p, _tensors(dict(m_scale=0x5000, v_scale=0x100000)), "overlap")
    assert fb.lib().fef_adamw_step(ctypes.byref(p), None, 0) == fb.FEF_OK


@pytest.mark.parametrize("kind", [-1, 2, 4, 5, 17])
def test_no_other_kinds(kind):
    _refused(_params(state_dtype=kind), _tensors({}), "state_dtype")
