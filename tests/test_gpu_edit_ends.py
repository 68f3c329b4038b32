"""fef_edit_logits at the ends of what its arguments may be: ids just past the vocabulary, repetition penalties at the ends of the numbers."""
import numpy as np
import pytest
import torch

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.gpu


def _run(logits, **x):
    B, K, V = logits.shape
    call = fb.EditLogits(B, K, V)
    out, lse = call(logits, fb.Edits(**{k: torch.from_numpy(v).cuda() for k, v in x.items()}))
    return out.clone(), lse.clone()


@pytest.mark.parametrize("rep,freq", [(0.0, 0.1), (-1.0, 0.1), (1.2, -float("inf"))])
@pytest.mark.parametrize("V,H", [(700, 40), (2100, 40), (700, 17000), (5000, 17000)])
def test_ids_just_past_the_vocabulary_stand_for_no_token(V, H, rep, freq):
    """Between the last token and the end of a workgroup's chunk, with penalties that make something of -inf."""
    rng = np.random.default_rng(V + H)
    B, K = 2, 3
    logits = torch.from_numpy(rng.standard_normal((B, K, V)).astype(np.float32)).cuda()
    none, past = np.full((B, H), -1, np.int32), (V + rng.integers(0, 60, (B, H))).astype(np.int32)
    kw = dict(repetition=np.full(B, rep, np.float32), frequency=np.full(B, freq, np.float32), presence=np.full(B, 0.5, np.float32))
    want = _run(logits, history=none, prefix=none[:, :K].copy(), **kw)
    assert torch.equal(want[0], logits) and bool(torch.isfinite(want[1]).all())
    for history, prefix in ((past, none), (none, past), (past, past)):
        got = _run(logits, history=history, prefix=prefix[:, :K].copy(), **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


REPS = [0.0, 1e-45, 1e-40, 1.1754944e-38, 3e-38, 1e-30, 0.3, 1.0, 1.7, 1e20, 2.0 ** 101, 2.0 ** 126, 1.5 * 2.0 ** 126, 2.0 ** 127, 3.4028235e38, float("inf"),
        -2.0, -1e-40, -3e38, float("nan")]


def test_repetition_penalties_at_the_ends_of_the_numbers():
    """x / rep for positive and x * rep for other logits, to a step of the result (a division by way of the reciprocal may miss the nearest
    number by one): 2^-23 of it, or 2^-149 among subnormal ones."""
    x = np.array([1e-45, 3e-39, 1.2e-38, 1e-30, 0.1, 1.0, 3.0, 100.0, 7e19, 3.4028235e38, np.inf, 0.0, -0.0, -1e-45, -1e-30, -1.0, -5.5, -3e38, -np.inf],
                 dtype=np.float32)
    V, B = len(x), len(REPS)
    logits = torch.from_numpy(np.broadcast_to(x, (B, 1, V)).copy()).cuda()
    rep = np.array(REPS, dtype=np.float32)
    out, _ = _run(logits, history=np.broadcast_to(np.arange(V, dtype=np.int32), (B, V)).copy(), repetition=rep)
    with np.errstate(all="ignore"):
        x64, r64 = x.astype(np.float64)[None], rep.astype(np.float64)[:, None]
        want = np.where(x64 > 0, x64 / r64, x64 * r64)
        rounded = want.astype(np.float32)
    got = out[:, 0].cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(rounded))
    assert np.array_equal(got[np.isinf(rounded)], rounded[np.isinf(rounded)])
    live = np.isfinite(rounded)
    off = np.abs(got.astype(np.float64) - want)
    assert np.all(off[live] <= 2.0 ** -23 * np.abs(want[live]) + 2.0 ** -149)
