"""Draws never end at a token without mass.

A draw is the first index whose prefix sum reaches a target; each lane sums its own stretch in order, from a start that a tree over the
lanes gives, and the two round differently.  A target between the end of one lane and the start of the next meets the next lane's first
element.  The laws here are made so that this happens as often as it can: all but a lane's first element is positive, but so light that
the sum in order, which stands above 1/2, does not move (less than half of its step of 2^-24), while the tree sees the lane's total; the
first element has no mass at all.  With `gap` steps between end and start of each lane, a draw lands in one of them with a probability of
gap x lanes x 2^-24; the numbers of draws are chosen so that a search which takes such an element shows it many times.  Past the last
element of a law the same holds: V = 250 ends at the end of a lane, and the next lane's first element would be token 250."""
import math

import numpy as np
import pytest
import torch

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.gpu

LIGHT = 0.45 * 2.0 ** -24


def _masses(n, per):
    """Masses of n elements in lanes of `per`: without mass at the start of each lane, heavy in the first and the last lane."""
    m = np.full(n, LIGHT)
    m[::per] = 0
    m[1], m[n - 1] = 0, 0
    left = 1 - m.sum()
    m[1], m[n - 1] = 0.55 * left, 0.45 * left
    return m


def _logits(m):
    with np.errstate(divide="ignore"):
        return np.log(m)


def _spread(m, V, unit):
    """Masses of tiles or chunks of `unit` tokens as a law over V tokens: one token of each holds it all, the first one never."""
    out = np.zeros(V)
    at = np.minimum(np.arange(len(m)) * unit + 1 + np.arange(len(m)) % 7, V - 1)
    out[at] = m
    return out


def _draw(kind, row, B, launches, V):
    """Tokens without mass among B x launches draws from the law of `row`, and how often each half of the law was drawn."""
    vl = fb.VerifyLogits(B, 1, 1, V)
    law = torch.from_numpy(row.astype(np.float32)).cuda()
    allowed = torch.isfinite(law)
    if kind == "draft":
        vl.draft_logits.copy_(law.expand(B, 1, V))
    else:                                             # the draft is always token 0, which the target does not have
        assert not bool(allowed[0])
        vl.draft_logits.fill_(-float("inf"))
        vl.draft_logits[:, :, 0] = 0
        vl.target_logits.copy_(law.expand(B, 1, V))
    phase = fb.FEF_PHASE_DRAFT if kind == "draft" else fb.FEF_PHASE_FUSED
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    late = torch.zeros((), dtype=torch.int64, device="cuda")
    for seed in range(launches):
        tok, acc, _ = vl(seed, final_pass=True, phase=phase)
        if kind != "draft":
            assert seed or not bool(acc.any())
        at = tok[:, 0].long()
        inside = (at >= 0) & (at < V)
        bad += (~(inside & allowed[at.clamp(0, V - 1)])).sum()
        late += (at > V // 2).sum()
    return int(bad), int(late) / (B * launches)


CASES = [("residual", "token", 256, 4, 1 << 18, 60),        # four tokens per lane, one workgroup alone
         ("residual", "chunk", 65536, 16, 4096, 600),       # 16 chunks per lane
         ("residual", "chunk", 262400, 5, 512, 900),        # five chunks per thread of a workgroup
         ("draft", "token", 250, 10, 1 << 18, 60),          # ten tokens per lane
         ("draft", "chunk", 65536, 4, 4096, 600),           # four, ten and (from memory) 41 tiles per lane
         ("draft", "chunk", 151936, 10, 1024, 600),
         ("draft", "chunk", 660000, 41, 256, 600)]


@pytest.mark.parametrize("kind,level,V,per,B,launches", CASES)
def test_no_draw_of_a_token_without_mass(kind, level, V, per, B, launches):
    if level == "token":
        m = _masses(V, per)
    else:
        n = (V + 255) // 256
        m = _spread(_masses(n - 1 if V % 256 else n, per), V, 256)
    bad, late = _draw(kind, _logits(m), B, launches, V)
    assert abs(late - 0.45) < 0.01                    # the draws are there
    assert bad == 0


def test_no_draw_of_a_token_without_mass_in_a_chunk_of_a_workgroup():
    """One token per thread: pairs of light tokens, then one without mass, all in one chunk of a vocabulary of more than 1024 chunks."""
    V = 262400
    m = np.zeros(V)
    m[1024:1280] = _masses(256, 3)
    bad, late = _draw("residual", _logits(np.roll(m, 1)), 512, 900, V)
    assert bad == 0 and late == 0


@pytest.mark.parametrize("V,per,B", [(65536, 4, 4096), (151936, 10, 1024)])
def test_a_tile_whose_tokens_are_lighter_than_a_number(V, per, B):
    """The first tile of each lane has a mass that is a (subnormal) number, its tokens' masses are none, and its first token is masked."""
    n = V // 256
    m = _masses(n, per)
    row = _logits(_spread(m, V, 256))
    top = math.log(0.55)
    for t in range(per, n, per):
        row[t * 256 + 1:(t + 1) * 256] = top - 103.5  # exp(-103.5) is 2^-149 rounded, times 0.55 it is none
    bad, late = _draw("draft", row, B, 600, V)
    assert abs(late - 0.45) < 0.01
    assert bad == 0
