"""fef_adamw_step against the same formulas in numpy's float32, whose operations are correctly rounded like the kernel's: every bit of
parameters, copies, states, codes and scales has to be equal, so no tolerance is used there.  Against the formulas in 64 bits the error of
one step is bounded by counting roundings."""
import numpy as np
import pytest
import torch

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.gpu
F = np.float32


def _e4m3_values():
    """Magnitudes of the 127 finite codes: 3 mantissa bits, exponent bias 7, subnormals at 2^-9."""
    return np.array([(m / 8 * 2.0 ** -6) if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


VALUES = _e4m3_values()


def _encode(y):
    """Codes of float32 magnitudes up to 448 (and a rounding), to nearest, ties to the even code."""
    y = y.astype(np.float64)
    hi = np.clip(np.searchsorted(VALUES, y), 1, 126)
    low, high = VALUES[hi - 1], VALUES[hi]
    up = (y - low > high - y) | ((y - low == high - y) & (hi % 2 == 0))
    return np.where(y >= VALUES[126], 126, np.where(up, hi, hi - 1)).astype(np.uint8)


def _held(x, root):
    """Codes and scales of float32 x, 256 at a time."""
    code, scale = np.zeros(x.size, np.uint8), np.zeros((x.size + 255) // 256, F)
    for b in range(scale.size):
        part = x[256 * b:256 * b + 256]
        top = np.abs(part).max()
        if top < F(2.0 ** -100):
            continue
        y = np.abs(part) * (F(448) / top)
        c = _encode(y)
        if root:
            c[(part > 0) & (c == 0)] = 1
        code[256 * b:256 * b + 256] = c | (128 * np.signbit(part)).astype(np.uint8)
        scale[b] = top / F(448)
    return code, scale


def _value(code, scale):
    x = VALUES[code & 127].astype(F) * np.repeat(scale, 256)[:code.size]
    return np.where(code & 128, -x, x).astype(F)


def _bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).float().numpy()


class Oracle:
    """One tensor, numpy float32."""

    def __init__(self, p, bf16, master, eight):
        self.bf16, self.has_copy, self.eight = bf16, master, eight
        self.p, self.copy = p.copy(), p.copy()
        self.m, self.v = np.zeros(p.size, F), np.zeros(p.size, F)
        if eight:
            self.m, self.v = np.zeros(p.size, np.uint8), np.zeros(p.size, np.uint8)
            self.ms, self.vs = np.zeros((p.size + 255) // 256, F), np.zeros((p.size + 255) // 256, F)

    def step(self, g, t, lr, b1, b2, eps, wd, gs=1.0):
        c1, c2 = F(1.0 / (1.0 - b1 ** t)), F(1.0 / np.sqrt(1.0 - b2 ** t))
        lr = F(lr)
        keep, rate = F(1) - lr * F(wd), lr * c1
        g = g * F(gs)
        m, v = (_value(self.m, self.ms), _value(self.v, self.vs)) if self.eight else (self.m, self.v)
        if self.eight:
            v = v * v
        m = m * F(b1) + g * F(1.0 - b1)
        v = v * F(b2) + g * g * F(1.0 - b2)
        r = np.sqrt(v)
        x = self.copy if self.has_copy else self.p
        x = x * keep - m / (r * c2 + F(eps)) * rate
        assert x.dtype == m.dtype == v.dtype == F
        self.copy = x
        self.p = _bf16(x) if self.bf16 else x
        if self.eight:
            self.m, self.ms = _held(m, False)
            self.v, self.vs = _held(r, True)
        else:
            self.m, self.v = m, v


def _tensors(sizes, bf16, grad_bf16, seed):
    rng = np.random.default_rng(seed)
    ps = [(rng.standard_normal(n) * 0.02).astype(F) for n in sizes]
    if bf16:
        ps = [_bf16(p) for p in ps]
    gs = [[(rng.standard_normal(n) * np.exp(rng.standard_normal(n)) * 1e-3).astype(F) for n in sizes] for _ in range(3)]
    if grad_bf16:
        gs = [[_bf16(g) for g in step] for step in gs]
    return ps, gs


def _same(op, oracles, eight):
    for i, o in enumerate(oracles):
        assert np.array_equal(op.params[i].float().cpu().numpy().ravel(), o.p), i
        if op.master:
            assert np.array_equal(op.master[i].cpu().numpy().ravel(), o.copy), i
        for t, want in ((op.m[i], o.m), (op.v[i], o.v)):
            got = t.view(torch.uint8).cpu().numpy() if eight else t.cpu().numpy()
            assert np.array_equal(got, want), i
        if eight:
            assert np.array_equal(op.m_scale[i].cpu().numpy(), o.ms) and np.array_equal(op.v_scale[i].cpu().numpy(), o.vs), i


HYPER = dict(lr=3e-3, betas=(0.9, 0.95), eps=1e-8)


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("bf16,grad_bf16,master", [(True, True, True), (True, True, False), (True, False, True), (False, False, False), (False, True, False)])
@pytest.mark.parametrize("sizes", [[1], [3, 255, 256, 257], [4095, 4096, 4097, 1, 20000], [513] * 100])
def test_every_bit_over_three_steps(sizes, bf16, grad_bf16, master, states):
    ps, gs = _tensors(sizes, bf16, grad_bf16, 7 + len(sizes))
    kind, gkind = torch.bfloat16 if bf16 else torch.float32, torch.bfloat16 if grad_bf16 else torch.float32
    decay = [0.1 if i % 2 == 0 else 0.0 for i in range(len(sizes))]
    params, grads = [torch.from_numpy(p).cuda().to(kind) for p in ps], [torch.zeros(n, dtype=gkind, device="cuda") for n in sizes]
    op = fb.AdamW(params, grads, weight_decay=decay, states=states, master=master, **HYPER)
    oracles = [Oracle(p, bf16, master, states == "8bit") for p in ps]
    for t in range(1, 4):
        for g, new in zip(grads, gs[t - 1]):
            g.copy_(torch.from_numpy(new))
        op.step()
        for o, g, wd in zip(oracles, gs[t - 1], decay):
            o.step(g, t, HYPER["lr"], *HYPER["betas"], HYPER["eps"], wd)
        _same(op, oracles, states == "8bit")


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_addresses_that_suit_no_vector_load(states):
    """Every tensor one element behind an aligned address, with guards around all of them."""
    n = 5000
    ps, gs = _tensors([n], True, True, 3)
    def shifted(x, kind):
        whole = torch.full((n + 9,), 7.0, device="cuda").to(kind)
        whole[1:n + 1] = torch.from_numpy(x).cuda().to(kind)
        return whole
    p, g, copy = shifted(ps[0], torch.bfloat16), shifted(gs[0][0], torch.bfloat16), shifted(ps[0], torch.float32)
    state = torch.float8_e4m3fn if states == "8bit" else torch.float32
    m, v = (torch.full(((n + 9) * (1 if states == "8bit" else 4),), 0, dtype=torch.uint8, device="cuda").view(state) for _ in range(2))
    for t in (m, v):
        t.view(torch.uint8)[-8 * t.element_size():] = 77
    op = fb.AdamW([p[1:n + 1]], [g[1:n + 1]], states=states, master=[copy[1:n + 1]], m=[m[1:n + 1]], v=[v[1:n + 1]], weight_decay=0.1, **HYPER)
    op.step()
    o = Oracle(ps[0], True, True, states == "8bit")
    o.step(gs[0][0], 1, HYPER["lr"], *HYPER["betas"], HYPER["eps"], 0.1)
    _same(op, [o], states == "8bit")
    for t in (p, copy):
        assert float(t[0]) == 7.0 and bool((t[n + 1:].float() == 7.0).all())
    for t in (m, v):
        assert bool((t.view(torch.uint8)[-8 * t.element_size():] == 77).all())


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_blocks_of_zeros_and_of_tiny_numbers(states):
    """Gradients that are 0 for a whole block, for some elements, and far below the smallest reciprocal."""
    n = 1024
    ps, gs = _tensors([n], False, False, 5)
    for step in gs:
        step[0][:256] = 0
        step[0][256:512:2] = 0
        step[0][512:768] *= F(1e-35)
        step[0][768:1024] *= F(1e-28)
        step[0][768] = F(1e-2)           # one large element: the others' roots take the smallest code
    params, grads = [torch.from_numpy(ps[0]).cuda()], [torch.zeros(n, device="cuda")]
    op = fb.AdamW(params, grads, states=states, weight_decay=0.0, **HYPER)
    o = Oracle(ps[0], False, False, states == "8bit")
    for t in range(1, 4):
        grads[0].copy_(torch.from_numpy(gs[t - 1][0]))
        op.step()
        o.step(gs[t - 1][0], t, HYPER["lr"], *HYPER["betas"], HYPER["eps"], 0.0)
        _same(op, [o], states == "8bit")
    assert bool(torch.isfinite(op.params[0]).all()) and torch.equal(op.params[0][:256].cpu(), torch.from_numpy(ps[0][:256]))


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_gradient_that_is_no_number_stays_where_it_is(bad, states):
    ps, gs = _tensors([600], True, True, 9)
    gs[0][0][300] = bad
    op = fb.AdamW([torch.from_numpy(ps[0]).cuda().bfloat16()], [torch.from_numpy(gs[0][0]).cuda().bfloat16()], states=states, master=True,
                  weight_decay=0.1, **HYPER)
    op.step()
    o = Oracle(ps[0], True, True, False)
    with np.errstate(all="ignore"):
        o.step(gs[0][0], 1, HYPER["lr"], *HYPER["betas"], HYPER["eps"], 0.1)
    got = op.master[0].cpu().numpy()
    assert np.array_equal(got, o.copy, equal_nan=True) and not np.isfinite(got[300]) and np.isfinite(np.delete(got, 300)).all()
    if states == "8bit":
        assert not np.isfinite(op.m_scale[0].cpu().numpy()[1]) and np.isfinite(op.m_scale[0].cpu().numpy()[[0, 2]]).all()


def test_scales_of_the_gradient_and_the_schedule_on_the_device():
    ps, gs = _tensors([700], False, False, 11)
    b1, b2 = HYPER["betas"]
    def schedule(t, lr):
        return torch.tensor([lr, 1.0 / (1.0 - b1 ** t), 1.0 / np.sqrt(1.0 - b2 ** t)], dtype=torch.float32)
    on_device, scale = torch.zeros(3, device="cuda"), torch.zeros(1, device="cuda")
    params, grads = [torch.from_numpy(ps[0]).cuda()], [torch.zeros(700, device="cuda")]
    op = fb.AdamW(params, grads, weight_decay=0.1, schedule=on_device, grad_scale=scale, **HYPER)
    o = Oracle(ps[0], False, False, False)
    for t in range(1, 4):
        grads[0].copy_(torch.from_numpy(gs[t - 1][0]))
        on_device.copy_(schedule(t, 1e-2 / t))
        scale.fill_(0.5 + t)
        op.step()
        o.step(gs[t - 1][0], t, 1e-2 / t, b1, b2, HYPER["eps"], 0.1, gs=0.5 + t)
        _same(op, [o], False)


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_captured_steps_go_on(states):
    """A captured step replayed with new gradients and a new schedule between replays, against eager steps."""
    sizes = [5000, 33]
    ps, gs = _tensors(sizes, True, True, 13)
    b1, b2 = HYPER["betas"]
    sides = []
    for _ in range(2):
        grads = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in sizes]
        schedule = torch.zeros(3, device="cuda")
        op = fb.AdamW([torch.from_numpy(p).cuda().bfloat16() for p in ps], grads, states=states, master=True, schedule=schedule, **HYPER)
        sides.append((op, grads, schedule))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sides[0][0].step()
    for t in range(1, 4):
        for op, grads, schedule in sides:
            for g, new in zip(grads, gs[t - 1]):
                g.copy_(torch.from_numpy(new))
            schedule.copy_(torch.tensor([1e-3, 1.0 / (1.0 - b1 ** t), 1.0 / np.sqrt(1.0 - b2 ** t)], dtype=torch.float32))
        graph.replay()
        sides[1][0].step()
        torch.cuda.synchronize()
        for a, b in zip(sides[0][0].params + sides[0][0].master, sides[1][0].params + sides[1][0].master):
            assert torch.equal(a, b)
        for a, b in zip(sides[0][0].m + sides[0][0].v, sides[1][0].m + sides[1][0].v):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_another_stream():
    ps, gs = _tensors([100000], True, True, 17)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        op = fb.AdamW([torch.from_numpy(ps[0]).cuda().bfloat16()], [torch.from_numpy(gs[0][0]).cuda().bfloat16()], master=True, weight_decay=0.1, **HYPER)
        op.step()
    stream.synchronize()
    o = Oracle(ps[0], True, True, False)
    o.step(gs[0][0], 1, HYPER["lr"], *HYPER["betas"], HYPER["eps"], 0.1)
    _same(op, [o], False)


def test_one_step_in_64_bits():
    """x = p keep - m / (r c2 + eps) rate.  keep and the product with it: 3 roundings of at most 2^-24 |p| (1.1 for what keep leaves).  The
    update u: the rounded constants b1, 1 - b1, c1, c2, lr, rate, b2, 1 - b2, eps and the operations on the way (m 3, v 4, root 1, 2 for
    the denominator, quotient and product 2) are at most 24 relative roundings of 2^-24 of terms without cancellation, of which those in
    v count half; m starts from zero here and does not cancel.  The final difference adds 2^-24 (|p| + |u|)."""
    n = 20000
    ps, gs = _tensors([n], False, False, 19)
    op = fb.AdamW([torch.from_numpy(ps[0]).cuda()], [torch.from_numpy(gs[0][0]).cuda()], weight_decay=0.1, **HYPER)
    op.step()
    p, g = ps[0].astype(np.float64), gs[0][0].astype(np.float64)
    (b1, b2), lr = HYPER["betas"], HYPER["lr"]
    m, v = (1 - b1) * g, (1 - b2) * g * g
    u = lr * (m / (1 - b1)) / (np.sqrt(v / (1 - b2)) + HYPER["eps"])
    want = p * (1 - lr * 0.1) - u
    assert np.all(np.abs(op.params[0].cpu().numpy() - want) <= 2.0 ** -24 * (4.4 * np.abs(p) + 25 * np.abs(u)))
