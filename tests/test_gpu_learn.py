"""Draws, gradients and steps together, as a program learns from its own draws: logits of the head, tokens of their truncated laws, the
gradient of the weighted log-probabilities of these tokens, a step of the head and of the rows; again with the new head."""
import numpy as np
import pytest
import torch

import draw_oracle
from paper_2605_14305_amd import binding as fb
from test_gpu_adamw import Oracle, _same
from test_gpu_grad import KIND, _definition, _tolerances

pytestmark = pytest.mark.gpu
LR, BETAS, EPS, DECAY = 2e-2, (0.9, 0.95), 1e-8, 0.1


class Program:
    """B sequences of K rows of a table h [R, d], and a head W [V, d]."""

    def __init__(self, B, K, d, V, dtype, states, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        R = B * K
        self.h = (torch.randn(R, d, generator=g, device="cuda") * 3).to(KIND[dtype])
        self.W = (torch.randn(V, d, generator=g, device="cuda") * 0.1).to(KIND[dtype])
        self.u, self.reward = torch.zeros(B, K, device="cuda"), torch.zeros(R, device="cuda")
        self.top_k = torch.tensor([(0, 40, 7)[b % 3] for b in range(B)], dtype=torch.int32, device="cuda")
        self.top_p = torch.tensor([(0.9, 0.95, 1.0)[b % 3] for b in range(B)], device="cuda")
        self.schedule = torch.ones(3, device="cuda")
        self.logits = torch.zeros(B, K, V, device="cuda")
        self.draw = fb.DrawLogits(B, K, V)
        self.grad = fb.HeadCrossEntropyGrad(R, d, V, dtype=dtype)
        self.adamw = fb.AdamW([self.W, self.h], [self.grad.grad_w, self.grad.grad_h], betas=BETAS, eps=EPS, weight_decay=[DECAY, 0.0],
                              states=states, master=dtype == "bf16", schedule=self.schedule)
        self.B, self.K, self.d, self.V, self.t = B, K, d, V, 0

    def inputs(self, seed):
        g = torch.Generator(device="cuda").manual_seed(1000 + seed)
        self.u.copy_(torch.rand(self.u.shape, generator=g, device="cuda"))
        self.reward.copy_(torch.randn(self.reward.shape, generator=g, device="cuda"))
        self.t += 1
        self.schedule.copy_(torch.tensor([LR, 1 / (1 - BETAS[0] ** self.t), 1 / np.sqrt(1 - BETAS[1] ** self.t)], dtype=torch.float64).float())

    def turn(self):
        torch.mm(self.h.float(), self.W.float().t(), out=self.logits.view(-1, self.V))
        tokens = self.draw(self.logits, self.u, top_k=self.top_k, top_p=self.top_p)[0]
        self.grad(self.h, self.W, tokens.view(-1), self.reward)
        self.adamw.step()


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("B,K,d,V,dtype", [(3, 5, 64, 1000, "bf16"), (4, 8, 128, 17000, "bf16"), (3, 7, 36, 2001, "f32")])
def test_turns(B, K, d, V, dtype, states):
    """Every stage against its definition, from what the stage before it left."""
    p = Program(B, K, d, V, dtype, states)
    oracles = [Oracle(t.float().cpu().numpy().ravel(), dtype == "bf16", dtype == "bf16", states == "8bit") for t in (p.W, p.h)]
    for turn in range(3):
        p.inputs(turn)
        h, W = p.h.clone(), p.W.clone()
        p.turn()
        tokens, rows, u = p.draw.out_tokens.cpu().numpy(), p.logits.cpu().numpy(), p.u.cpu().numpy()
        for b in range(B):
            for m in range(K):
                want = draw_oracle.truncate(rows[b, m], u[b, m], k=(0, 40, 7)[b % 3], p=float(np.float32((0.9, 0.95, 1.0)[b % 3])))
                assert tokens[b, m] == want[3]
        labels = p.draw.out_tokens.view(-1)
        ce, lse, G, want_h, want_w, mag_h, mag_w, z = _definition(h, W, labels, p.reward)
        of_z, of_p, tol_h, tol_w = _tolerances(h, W, 1.0, z, mag_h, mag_w, want_h, want_w, dtype)
        assert bool(((p.grad.out_ce.double() - ce).abs() <= of_p + 2.0 ** -23 * lse.abs()).all())
        assert bool(((p.grad.grad_h.double() - want_h).abs() <= tol_h).all()) and bool(((p.grad.grad_w.double() - want_w).abs() <= tol_w).all())
        for o, g, decay in zip(oracles, (p.grad.grad_w, p.grad.grad_h), (DECAY, 0.0)):
            o.step(g.float().cpu().numpy().ravel(), turn + 1, LR, *BETAS, EPS, decay)
        _same(p.adamw, oracles, states == "8bit")


@pytest.mark.parametrize("B,K,d,V,dtype", [(3, 5, 64, 1000, "bf16"), (4, 8, 128, 17000, "bf16"), (3, 7, 36, 2001, "f32")])
def test_captured_turns(B, K, d, V, dtype):
    """A turn as a graph, replayed on its own results, beside an eager program of the same start."""
    captured, eager = (Program(B, K, d, V, dtype, "8bit") for _ in range(2))
    for p in (captured, eager):
        p.inputs(0)
        p.turn()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.turn()
    for turn in range(1, 5):
        for p in (captured, eager):
            p.inputs(turn)
        graph.replay()
        eager.turn()
        torch.cuda.synchronize()
        for a, b in ((captured.draw.out_tokens, eager.draw.out_tokens), (captured.draw.out, eager.draw.out), (captured.grad.out_loss, eager.grad.out_loss),
                     (captured.W, eager.W), (captured.h, eager.h)):
            assert torch.equal(a, b)
        for a, b in zip(captured.adamw.m + captured.adamw.v, eager.adamw.m + eager.adamw.v):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_a_clipped_step():
    """Rows that do not count keep their place, and a scale on the device clips the step: both without a host in between."""
    R, d, V = 12, 64, 300
    p = Program(3, 4, d, V, "bf16", "f32")
    scale = torch.ones(1, device="cuda")
    step = fb.AdamW([p.W, p.h], [p.grad.grad_w, p.grad.grad_h], lr=LR, betas=BETAS, eps=EPS, weight_decay=0.0, master=True, grad_scale=scale)
    labels = torch.arange(R, dtype=torch.int32, device="cuda")
    labels[::4] = -1
    before = p.h.clone()
    p.grad(p.h, p.W, labels)
    norm = torch.sqrt(p.grad.grad_w.float().square().sum() + p.grad.grad_h.float().square().sum())
    scale.copy_((0.5 / norm).clamp(max=1.0).view(1))
    oracles = [Oracle(t.float().cpu().numpy().ravel(), True, True, False) for t in (p.W, p.h)]
    step.step()
    for o, g in zip(oracles, (p.grad.grad_w, p.grad.grad_h)):
        o.step(g.float().cpu().numpy().ravel(), 1, LR, *BETAS, EPS, 0.0, float(scale))
    _same(step, oracles, False)
    assert torch.equal(p.h[::4], before[::4]) and not torch.equal(p.h[1::4], before[1::4])
