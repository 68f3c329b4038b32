"""Rows masked with the lowest finite number in place of -inf, in a round on given logits: numbers below -2e38 count as -inf, so a row of nothing
else is no law."""
import numpy as np
import pytest
import torch

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.gpu
LOW = float(np.finfo(np.float32).min)


def _lowest(rows, first, V):
    rows.fill_(-float("inf"))
    rows[..., first:V] = LOW


@pytest.mark.parametrize("V,first", [(200, 7), (600, 256), (5000, 4097), (300000, 262401)])
@pytest.mark.parametrize("which", ["draft", "target", "both"])
def test_a_row_of_lowest_numbers_is_no_law(V, first, which):
    """Its slot is rejected; over such a draft row the token is one of the two that the target has, over such a target row its arg max."""
    B = 64
    vl = fb.VerifyLogits(B, 1, 1, V)
    vl.logits.fill_(LOW)                              # two equal tokens among masked ones
    vl.logits[..., 3] = vl.logits[..., V - 1] = 2.0
    if which != "target":
        _lowest(vl.logits[0], first, V)
    if which != "draft":
        _lowest(vl.logits[1], first, V)
    conf = torch.full((B, 1), -1.0, device="cuda")
    tok, acc, _ = (t.cpu().numpy() for t in vl(3, final_pass=True, conf=conf))
    assert (acc == 0).all()
    if which == "draft":
        assert 10 < (tok == 3).sum() < 54 and ((tok == 3) | (tok == V - 1)).all()   # of 64 even draws: exceeded with 1e-8
        assert bool(((conf - 0.5).abs() < 2.0 ** -20).all())
    else:
        assert (tok == first).all() and bool((conf == 0).all())


@pytest.mark.parametrize("V", [200, 5000])
def test_masked_with_lowest_numbers_is_masked(V):
    """The same bits as with -inf."""
    rng = np.random.default_rng(V)
    B, K = 16, 4
    one, two = fb.VerifyLogits(B, K, K, V, diag=True), fb.VerifyLogits(B, K, K, V, diag=True)
    x = torch.from_numpy(rng.standard_normal((2, B, K, V)).astype(np.float32) * 3).cuda()
    hide = torch.from_numpy(rng.random((2, B, K, V)) < 0.9).cuda()
    hide[..., 5] = False
    one.logits[..., :V] = torch.where(hide, -float("inf"), x)
    two.logits[..., :V] = torch.where(hide, LOW, x)
    for a, b in zip(one(9), two(9)):
        assert torch.equal(a, b)
    for k in one.diag:
        assert torch.equal(one.diag[k], two.diag[k])


@pytest.mark.parametrize("V,first", [(600, 256), (5000, 4097)])
def test_greedy_takes_such_rows_for_token_0(V, first):
    vl = fb.VerifyLogits(4, 1, 1, V)
    _lowest(vl.logits, first, V)
    tok, acc, _ = vl(3, final_pass=True, greedy=True)
    assert bool((tok == 0).all()) and bool((acc == 1).all())
