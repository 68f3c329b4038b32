"""fef_head_cross_entropy_grad: a row whose label is negative has a CE and a row of grad_h of 0, whatever W holds."""
import pytest
import torch

from paper_2605_14305_amd import binding as fb
from test_gpu_grad import _case

pytestmark = pytest.mark.gpu


# one share of the tokens and several, every height of the products' tiles, rows that are whole pieces of 16 bytes and others
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("R,d,V,dtype", [(5, 64, 60, "bf16"), (40, 128, 64, "bf16"), (100, 64, 50, "bf16"), (300, 320, 60, "bf16"), (5, 64, 3000, "bf16"),
                                         (40, 320, 1000, "bf16"), (100, 64, 999, "bf16"), (300, 64, 4100, "bf16"), (5, 64, 30, "f32"), (40, 36, 31, "f32"),
                                         (100, 64, 30, "f32"), (5, 64, 3000, "f32"), (40, 36, 1000, "f32"), (100, 20, 3000, "f32"), (5, 33, 30, "f32"),
                                         (100, 31, 2000, "f32"), (9, 1, 70, "f32")])
def test_rows_that_do_not_count_have_gradients_of_0(R, d, V, dtype, bad):
    h, W, labels, w = _case(R, d, V, dtype)
    op = fb.HeadCrossEntropyGrad(R, d, V, dtype=dtype)
    W[V // 2, d // 2] = bad
    W[V - 1, 0] = bad
    ce, loss, gh, gw = op(h, W, labels, w)
    out = labels < 0
    assert bool(out.any()) and bool((ce[out] == 0).all()) and bool((gh[out] == 0).all())
    assert bool(gh[~out].isnan().any(dim=1).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_row_counts(dtype):
    h, W, labels, w = _case(70, 64, 300, dtype)
    labels.fill_(-1)
    W.fill_(float("nan"))
    ce, loss, gh, gw = fb.HeadCrossEntropyGrad(70, 64, 300, dtype=dtype)(h, W, labels, w)
    assert float(loss) == 0 and not bool(ce.any()) and bool((gh == 0).all()) and bool((gw == 0).all())
