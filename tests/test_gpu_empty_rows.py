"""Rows that are no law in a round on given logits (nothing but -inf, or a +inf or NaN somewhere): over such a draft row the committed token
follows the target law itself; over such a target row it is the row's arg max with a confidence of 0; neither has mass in the diagnostics."""
import numpy as np
import pytest
import torch

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.gpu


def _spoil(rows, how):
    if how == "empty":
        rows.fill_(-float("inf"))
    else:
        rows[..., 3] = float("inf" if how == "inf" else "nan")


@pytest.mark.parametrize("how", ["empty", "inf", "nan"])
@pytest.mark.parametrize("V,B,diag", [(12, 40000, False), (12, 40000, True), (5000, 20000, False), (5000, 4000, True), (262500, 3000, False)])
def test_over_an_empty_draft_row_the_token_follows_the_target_law(V, B, diag, how):
    """Chi-square against a target law of 12 tokens somewhere in the vocabulary, 11 degrees of freedom; 40 is exceeded with probability
    4e-5."""
    rng = np.random.default_rng(V + B)
    at = np.sort(rng.choice(V, 12, replace=False))
    p = rng.standard_normal(12) * 0.7
    row = np.full(V, -np.inf, dtype=np.float32)
    row[at] = p
    vl = fb.VerifyLogits(B, 1, 1, V, diag=diag)
    vl.draft_logits.copy_(torch.from_numpy(rng.standard_normal(V).astype(np.float32)).cuda().expand(B, 1, V))
    _spoil(vl.draft_logits, how)
    vl.target_logits.copy_(torch.from_numpy(row).cuda().expand(B, 1, V))
    tok, acc, _ = (t.cpu().numpy() for t in vl(77, final_pass=True))
    assert not acc.any()
    law = np.exp(p - p.max())
    law /= law.sum()
    n = np.array([(tok == v).sum() for v in at])
    assert n.sum() == B
    assert (((n - B * law) ** 2) / (B * law)).sum() < 40
    if diag:                                          # twelve masses rounded a few times each: 2^-20 is a dozen and more half steps
        d = {k: t.cpu().numpy() for k, t in vl.diag.items()}
        assert (d["alpha"] == 0).all() and (np.abs(d["resid_mass"] - 1) < 2.0 ** -20).all()
        conf = law[np.searchsorted(at, tok[:, 0])]
        assert (np.abs(d["conf_tok"][:, 0] - conf) < 2.0 ** -20).all()


@pytest.mark.parametrize("how", ["empty", "inf", "nan"])
@pytest.mark.parametrize("greedy", [False, True])
@pytest.mark.parametrize("V,diag", [(12, True), (5000, True), (5000, False), (262500, False)])
def test_a_target_row_without_a_law(V, diag, greedy, how):
    rng = np.random.default_rng(V)
    B = 8
    vl = fb.VerifyLogits(B, 2, 2, V, diag=diag)
    vl.draft_logits.copy_(torch.from_numpy(rng.standard_normal((B, 2, V)).astype(np.float32)))
    vl.target_logits.copy_(vl.draft_logits)
    _spoil(vl.target_logits[:, 1], how)
    best = {"empty": 0, "inf": 3}.get(how)
    if greedy and best is not None:
        vl.draft_logits[:, 1, 5] = 50.0               # the draft's arg max is another
    conf = torch.full((B, 2), -1.0, device="cuda")
    tok, acc, _ = (t.cpu().numpy() for t in vl(5, final_pass=True, greedy=greedy, conf=conf))
    assert ((tok >= 0) & (tok < V)).all()
    if best is not None:
        assert (acc == 1).all() and (tok[:, 1] == best).all()
    assert bool((conf[:, 0] > 0).all()) and bool((conf[:, 1] == 0).all())
    if diag:
        d = {k: t.cpu().numpy() for k, t in vl.diag.items()}
        assert (d["alpha"][:, 1] == 0).all() and (d["resid_mass"][:, 1] == 0).all() and (d["conf_tok"][:, 1] == 0).all()
        assert (np.abs(d["alpha"][:, 0] - 1) < 2.0 ** -16).all()  # V masses of one law summed in a tree, each off by its own half step
