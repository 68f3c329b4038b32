"""fef_edit_logits at the ends of what its arguments may be: ids just past the vocabulary."""
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
