"""fef_verify_logits against the CPU oracle, whose head is the identity where the logits are given, and the example that joins it with
the 4-bit head and the edits.  Tolerances: tests/parity.py, whose margins are those of float32 log-sum-exps and prefix sums over
logits that both sides hold alike."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import fef_oracle as O
from paper_2605_14305_amd import binding as fb
from paper_2605_14305_amd import synth
import parity

pytestmark = pytest.mark.gpu


def _np(t):
    return t.detach().cpu().numpy()


def _logits(rng, B, K, V, spread=3.0, rho=0.9):
    q = rng.standard_normal((B, K, V)) * spread
    p = rho * q + np.sqrt(1 - rho * rho) * spread * rng.standard_normal((B, K, V))
    return q.astype(np.float32), p.astype(np.float32)


def _given(vl, q, p):
    vl.logits.fill_(float("nan"))                  # what lies past V is not used
    vl.draft_logits.copy_(torch.from_numpy(q))
    vl.target_logits.copy_(torch.from_numpy(p))


@pytest.mark.parametrize("B,K,block,V,diag", [(1, 1, 1, 1, True), (1, 4, 8, 7, False), (3, 5, 16, 255, True), (2, 8, 32, 256, False), (4, 8, 32, 257, True),
                                              (2, 16, 64, 1000, False), (5, 3, 9, 4097, False), (2, 8, 32, 4500, True)])
def test_against_the_oracle(B, K, block, V, diag):
    rng = np.random.default_rng(V)
    vl = fb.VerifyLogits(B, K, block, V, diag=diag)
    eye = np.eye(V)
    for step in range(3):
        q, p = _logits(rng, B, K, V)
        _given(vl, q, p)
        mask = (rng.random((B, block)) < 0.7).astype(np.uint8)
        tok, acc, rem = (_np(t) for t in vl(11, step=step, seq_base=5, pos_base=100, mask_in=torch.from_numpy(mask).cuda()))
        ref = O.verify_step(q.astype(np.float64), p.astype(np.float64), eye, K, block, 11, step=step, seq_base=5, pos_base=100, mask_in=mask)
        parity.compare(ref, tok, acc, rem, {k: _np(v) for k, v in vl.diag.items()} or None)


@pytest.mark.parametrize("V,d", [(50257, 128), (126464, 64)])
def test_the_logits_of_a_head(V, d):
    """The same round through the head's own call and through its logits."""
    B, K, block = 2, 8, 32
    W = synth.make_head(V, d, 3)
    hd, ht = synth.make_hidden(B, K, d, 3, 0.9, 3.0 / (0.02 * np.sqrt(d)))
    vs = fb.VerifyStep(B, K, block, d, V, diag=True, diag_logits=True, gemm_variant=fb.FEF_GEMM_TILED256)
    vs(hd.cuda(), ht.cuda(), W.cuda(), 21)
    vl = fb.VerifyLogits(B, K, block, V, diag=True)
    vl.logits[..., :V].copy_(vs.diag["logits"])
    tok, acc, rem = (_np(t) for t in vl(21))
    ref = O.verify_step(synth.to_f64(hd), synth.to_f64(ht), synth.to_f64(W), K, block, 21)
    parity.compare(ref, tok, acc, rem, {k: _np(v) for k, v in vl.diag.items()})
    assert torch.allclose(vl.diag["lse"], vs.diag["lse"], rtol=0, atol=1e-5)


@pytest.mark.parametrize("V", [900, 5000])
def test_draft_then_target_is_the_fused_round(V):
    rng = np.random.default_rng(V)
    B, K, block = 3, 8, 16
    q, p = _logits(rng, B, K, V)
    one, two = fb.VerifyLogits(B, K, block, V), fb.VerifyLogits(B, K, block, V)
    _given(one, q, p)
    fused = [t.clone() for t in one(7)]
    two.draft_logits.copy_(torch.from_numpy(q))
    two.target_logits.fill_(float("nan"))
    drafts = two(7, phase=fb.FEF_PHASE_DRAFT)[0].clone()
    assert bool(((drafts >= 0) & (drafts < V)).all())
    two.target_logits.copy_(torch.from_numpy(p))
    for a, b in zip(fused, two(7, phase=fb.FEF_PHASE_TARGET)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("V", [300, 5000])
@pytest.mark.parametrize("kind", ["sampled", "greedy", "given"])
def test_masked_tokens_are_no_tokens(V, kind):
    """-inf on the device where the oracle has a logit of -1e30."""
    rng = np.random.default_rng(V + len(kind))
    B, K, block = 4, 6, 12
    q, p = _logits(rng, B, K, V)
    q[rng.random((B, K, V)) < 0.8] = -np.inf
    gone = rng.random((B, K, V)) < 0.8
    p[gone] = -np.inf
    q[:, :, 1] = p[:, :, 2] = 0.5                    # no row is empty
    gone[:, :, 2] = False
    vl = fb.VerifyLogits(B, K, block, V)
    _given(vl, q, p)
    drafts = np.ascontiguousarray(q.argmax(2).astype(np.int32)) if kind == "given" else None
    kw = dict(greedy=kind == "greedy")
    tok, acc, rem = (_np(t) for t in vl(3, draft_tokens=None if drafts is None else torch.from_numpy(drafts).cuda(), **kw))
    far = [np.where(np.isinf(x), -1e30, x).astype(np.float64) for x in (q, p)]
    ref = O.verify_step(*far, np.eye(V), K, block, 3, draft_tokens=drafts, **kw)
    parity.compare(ref, tok, acc, rem, drafts_given=drafts is not None)
    for b in range(B):
        for m in range(min(int(acc[b]) + 1, K)):
            assert not gone[b, m, tok[b, m]]


@pytest.mark.parametrize("V", [200, 5000])
@pytest.mark.parametrize("greedy", [False, True])
def test_a_row_that_leaves_nothing(V, greedy):
    """Its slot is rejected with some token of the vocabulary; the sequences beside it do not notice."""
    rng = np.random.default_rng(V)
    B, K, block = 3, 4, 8
    q, p = _logits(rng, B, K, V, rho=1.0)           # equal laws: every draft is accepted
    vl = fb.VerifyLogits(B, K, block, V)
    _given(vl, q, p)
    want = [t.clone() for t in vl(9, greedy=greedy)]
    assert want[1].tolist() == [K] * B
    for which in ("draft", "target", "both"):
        _given(vl, q, p)
        if which != "target":
            vl.draft_logits[1, 2] = -float("inf")
        if which != "draft":
            vl.target_logits[1, 2] = -float("inf")
        tok, acc, rem = vl(9, greedy=greedy)
        if not (greedy and which == "both"):        # (two point masses at token 0 agree)
            assert int(acc[1]) == 2 or (greedy and which != "both" and int(acc[1]) >= 2)
        assert bool(((tok >= -1) & (tok < V)).all())
        for got, ref in zip((tok, acc, rem), want):
            assert torch.equal(got[[0, 2]], ref[[0, 2]])


def test_committed_tokens_follow_the_target_law_whatever_drafts_them():
    """First committed token of 40000 sequences with the same two rows: chi-square against the target law, 11 degrees of freedom; 40 is
    exceeded with probability 4e-5."""
    rng = np.random.default_rng(0)
    B, V = 40000, 12
    q, p = rng.standard_normal(V) * 1.5, rng.standard_normal(V) * 1.5
    q[3] = -np.inf                                  # a draft law that lacks what the target has, and the other way round
    p[5] = -np.inf
    vl = fb.VerifyLogits(B, 1, 1, V)
    _given(vl, np.broadcast_to(q.astype(np.float32), (B, 1, V)).copy(), np.broadcast_to(p.astype(np.float32), (B, 1, V)).copy())
    tok = _np(vl(1234, final_pass=True)[0])[:, 0]
    law = np.exp(p - p.max())
    law /= law.sum()
    n = np.bincount(tok, minlength=V)
    assert n[5] == 0
    live = law > 0
    assert (((n - B * law) ** 2)[live] / (B * law[live])).sum() < 40


def test_in_a_graph_and_on_another_stream():
    rng = np.random.default_rng(2)
    B, K, block, V = 2, 4, 8, 6000
    vl, eager = fb.VerifyLogits(B, K, block, V), fb.VerifyLogits(B, K, block, V)
    _given(vl, *_logits(rng, B, K, V))
    vl(5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vl(5)
    for i in range(4):
        q, p = _logits(rng, B, K, V)
        _given(vl, q, p)
        _given(eager, q, p)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = eager(5)
        torch.cuda.current_stream().wait_stream(side)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((vl.out_tokens, vl.out_accept_len, vl.out_remask), want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("args", [["--batch", "3", "--vocab", "1003", "--hidden", "256", "--window", "4", "--block", "10"],
                                  ["--batch", "2", "--vocab", "20011", "--hidden", "512", "--window", "8", "--block", "16"]])
def test_the_example(args):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import constrained_decode
    tokens, rounds, accepted, allowed = constrained_decode.main(args)
    assert bool((tokens >= 0).all()) and allowed
    block = int(args[-1])
    assert rounds < block and accepted > 0           # drafts from the 4-bit head pay
    again = constrained_decode.main(args)
    assert torch.equal(tokens, again[0]) and again[1:3] == (rounds, accepted)
