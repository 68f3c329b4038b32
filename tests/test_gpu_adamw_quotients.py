"""States in 8 bits in both arithmetics of their quotients (FEF_STATE_E4M3, FEF_STATE_E4M3_RECIPROCAL), at the numbers that tell them apart: every
bit against numpy's float32, and against the same formulas in elementwise torch."""
import math

import numpy as np
import pytest
import torch

import test_gpu_adamw as one
from paper_2605_14305_amd import binding as fb

F = np.float32
BETAS, EPS = (0.9, 0.95), 1e-8


def _quotients(top, reciprocal):
    """fl(448 / top) and fl(top / 448), or by reciprocals."""
    if reciprocal:
        return (F(1) / top) * F(448), top * (F(1) / F(448))
    return F(448) / top, top / F(448)


def _held(reciprocal):
    def held(x, root):
        code, scale = np.zeros(x.size, np.uint8), np.zeros((x.size + 255) // 256, F)
        for b in range(scale.size):
            part = x[256 * b:256 * b + 256]
            top = np.abs(part).max()
            if top < F(2.0 ** -100):
                continue
            inv, scale[b] = _quotients(top, reciprocal)
            c = one._encode(np.abs(part) * inv)
            if root:
                c[(part > 0) & (c == 0)] = 1
            code[256 * b:256 * b + 256] = c | (128 * np.signbit(part)).astype(np.uint8)
        return code, scale
    return held


def _between_codes(blocks):
    """Blocks of 256 numbers: a largest one, and others that the two arithmetics code differently."""
    rng = np.random.default_rng(0)
    middles = ((one.VALUES[1:] + one.VALUES[:-1]) / 2).astype(F)[8:-1]
    out = np.zeros((blocks, 256), F)
    b = 0
    while b < blocks:
        top = F(1 + rng.random())
        x = middles / (F(448) / top)
        x = (x.view(np.int32)[:, None] + np.arange(-3, 4, dtype=np.int32)).astype(np.int32).ravel().view(F)
        codes = [one._encode(x * _quotients(top, r)[0]) for r in (False, True)]
        apart = x[codes[0] != codes[1]]
        if apart.size:
            out[b, 0], out[b, 1:1 + min(apart.size, 255)] = top, apart[:255] * rng.choice([-1, 1], min(apart.size, 255))
            b += 1
    return out.ravel()


def test_the_arithmetics_differ_there():
    x = _between_codes(20)
    (a, s), (b, t) = _held(False)(x, False), _held(True)(x, False)
    assert (a != b).sum() >= 20 and (s != t).any() and np.abs(s / t - 1).max() <= 2.0 ** -22


@pytest.mark.gpu
@pytest.mark.parametrize("states", ["8bit", "8bit-reciprocal"])
def test_every_bit_between_two_codes(states, monkeypatch):
    """beta1 = 0: the first state is the gradient, and a second step reads what the first one has left."""
    monkeypatch.setattr(one, "_held", _held(states == "8bit-reciprocal"))
    g = _between_codes(60)
    p = np.zeros(g.size, F)
    op = fb.AdamW([torch.from_numpy(p).cuda()], [torch.from_numpy(g).cuda()], lr=1e-3, betas=(0.0, 0.95), eps=EPS, weight_decay=0.0, states=states)
    o = one.Oracle(p, False, False, True)
    for t in (1, 2):
        op.step()
        o.step(g, t, 1e-3, 0.0, 0.95, EPS, 0.0)
        one._same(op, [o], True)


@pytest.mark.gpu
@pytest.mark.parametrize("bf16,master", [(True, True), (True, False), (False, False)])
@pytest.mark.parametrize("sizes", [[1], [255, 256, 257], [20000, 3]])
def test_every_bit_by_reciprocals(sizes, bf16, master, monkeypatch):
    monkeypatch.setattr(one, "_held", _held(True))
    ps, gs = one._tensors(sizes, bf16, bf16, 31 + len(sizes))
    kind = torch.bfloat16 if bf16 else torch.float32
    grads = [torch.zeros(n, dtype=kind, device="cuda") for n in sizes]
    op = fb.AdamW([torch.from_numpy(p).cuda().to(kind) for p in ps], grads, lr=3e-3, betas=BETAS, eps=EPS, weight_decay=0.1, states="8bit-reciprocal",
                  master=master)
    oracles = [one.Oracle(p, bf16, master, True) for p in ps]
    for t in range(1, 4):
        for g, new in zip(grads, gs[t - 1]):
            g.copy_(torch.from_numpy(new))
        op.step()
        for o, g in zip(oracles, gs[t - 1]):
            o.step(g, t, 3e-3, *BETAS, EPS, 0.1)
        one._same(op, oracles, True)


def _coded(x, root):
    """Codes and scales by elementwise torch; x in whole blocks."""
    rows = x.view(-1, 256)
    top = rows.abs().amax(1)
    y = rows * (448.0 / top)[:, None]
    if root:
        y = torch.where((rows > 0) & (y < 2.0 ** -9), torch.full((), 2.0 ** -9, device=x.device), y)
    return y.to(torch.float8_e4m3fn).view(-1), top / 448.0


@pytest.mark.gpu
def test_ten_steps_of_elementwise_torch():
    """The states of ten steps in every bit, each side going on from its own."""
    n = 1 << 20
    g = torch.Generator(device="cuda").manual_seed(5)
    grad = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    op = fb.AdamW([torch.zeros(n, dtype=torch.bfloat16, device="cuda")], [grad], lr=1e-4, betas=BETAS, eps=EPS, weight_decay=0.1, states="8bit-reciprocal",
                  master=True)
    m, v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    ms, vs = (torch.zeros(n // 256, device="cuda") for _ in range(2))

    def value(code, scale):
        return (code.float().view(-1, 256) * scale[:, None]).view(-1)

    spread = torch.exp(torch.randn(n, generator=g, device="cuda")) * 1e-3
    for t in range(1, 11):
        grad.copy_(torch.randn(n, generator=g, device="cuda") * spread)
        op.step()
        x = grad.float()
        first = value(m, ms) * BETAS[0] + x * (1.0 - BETAS[0])
        second = value(v, vs)
        second = second * second * BETAS[1] + x * x * (1.0 - BETAS[1])
        (m, ms), (v, vs) = _coded(first, False), _coded(torch.sqrt(second), True)
        for a, b in ((op.m[0].float(), m.float()), (op.v[0].float(), v.float()), (op.m_scale[0], ms), (op.v_scale[0], vs)):
            assert torch.equal(a, b), t
    assert math.isfinite(float(op.master[0].abs().max()))
