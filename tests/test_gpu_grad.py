"""fef_head_cross_entropy_grad against its definition in 64 bits, against differences of the loss, and, where every term is a whole number
of the same small fraction, to the last bit."""
import numpy as np
import pytest
import torch

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.gpu
KIND = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(R, d, V, dtype, seed=0, tau=1.0, weights=True, skip=True, std=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed + R + d + V)
    W = (torch.randn(V, d, generator=g, device="cuda") * 0.02).to(KIND[dtype])
    h = (torch.randn(R, d, generator=g, device="cuda") * (std * tau / (0.02 * d ** 0.5))).to(KIND[dtype])
    labels = torch.randint(0, V, (R,), generator=g, device="cuda")
    labels[0], labels[-1] = V - 1, 0
    if skip and R > 2:
        labels[1::3] = -1
        labels[R // 2] = -7
    w = (0.25 + torch.rand(R, generator=g, device="cuda")) * torch.where(torch.rand(R, generator=g, device="cuda") < 0.5, -1.0, 1.0) if weights else None
    return h, W, labels.to(torch.int32), w


def _definition(h, W, labels, w, tau=1.0):
    """ce, G, grad_h, grad_w and the sums of magnitudes behind the last two, in 64 bits."""
    h, W, labels = h.double(), W.double(), labels.long()
    z = (h @ W.t().contiguous()) / tau
    lse = torch.logsumexp(z, 1)
    on = labels >= 0
    rows = torch.nonzero(on)[:, 0]
    ce = torch.zeros_like(lse)
    ce[rows] = lse[rows] - z[rows, labels[rows]]
    p = torch.exp(z - lse[:, None])
    G = p.clone()
    G[rows, labels[rows]] -= 1
    scale = (on.double() * (1.0 if w is None else w.double()) / tau)[:, None]
    G, p = G * scale, (p + torch.nn.functional.one_hot(labels.clamp(min=0), z.shape[1]) * on[:, None]) * scale.abs()
    return ce, lse, G, G @ W, G.t().contiguous() @ h, p @ W.abs(), p.t().contiguous() @ h.abs(), z


def _tolerances(h, W, tau, z, mag_h, mag_w, want_h, want_w, dtype):
    """A logit is a sum of d products, in float32 a relative error of at most (d + 2) 2^-24 of the sum of their magnitudes M; p is off by the
    errors of two logits and of exp, log and the sum over V (V + 8 roundings at the most, none of them larger than the value).  G is rounded once
    (bf16: 2^-8), its products are summed in float32 (one rounding each of at most 2^-24 of the sum of magnitudes), and the result is
    rounded once."""
    R, d = h.shape
    V = W.shape[0]
    M = float((h.double().abs() @ W.double().abs().t().contiguous()).amax()) / tau
    of_z = (d + 2) * 2.0 ** -24 * M
    of_p = 2 * of_z + (V + 12 + float(z.abs().amax())) * 2.0 ** -24
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tol_h = (of_p + half + (V + 300) * 2.0 ** -24) * mag_h + half * want_h.abs()
    tol_w = (of_p + half + (R + 8) * 2.0 ** -24) * mag_w + half * want_w.abs()
    return of_z, of_p, tol_h + 1e-37, tol_w + 1e-37


def _check(R, d, V, dtype, tau=1.0, weights=True, skip=True, seed=0):
    h, W, labels, w = _case(R, d, V, dtype, seed, tau, weights, skip)
    op = fb.HeadCrossEntropyGrad(R, d, V, dtype=dtype)
    for t in (op.out_ce, op.grad_h, op.grad_w):
        t.fill_(float("nan"))
    op.workspace.fill_(255)
    ce, loss, gh, gw = op(h, W, labels, w, temperature=tau)
    want_ce, lse, G, want_h, want_w, mag_h, mag_w, z = _definition(h, W, labels, w, tau)
    of_z, of_p, tol_h, tol_w = _tolerances(h, W, tau, z, mag_h, mag_w, want_h, want_w, dtype)
    assert bool(((ce.double() - want_ce).abs() <= of_p + 2.0 ** -23 * lse.abs()).all())
    assert abs(float(loss) - float(ce.double().sum())) <= R * 2.0 ** -24 * float(ce.double().abs().sum()) + 1e-30
    assert bool((ce[labels < 0] == 0).all()) and bool((gh[labels < 0] == 0).all())
    assert bool(((gh.double() - want_h).abs() <= tol_h).all()), float(((gh.double() - want_h).abs() / tol_h).max())
    assert bool(((gw.double() - want_w).abs() <= tol_w).all()), float(((gw.double() - want_w).abs() / tol_w).max())
    # and as a whole: independent roundings, so far below the sum of the worst ones
    near = 4e-3 if dtype == "bf16" else 2e-5
    assert float((gh.double() - want_h).norm()) <= near * float(want_h.norm()) + 1e-30
    assert float((gw.double() - want_w).norm()) <= near * float(want_w.norm()) + 1e-30


@pytest.mark.parametrize("R,d,V", [(1, 64, 1), (1, 64, 2), (2, 64, 63), (3, 128, 65), (31, 192, 1000), (33, 64, 257), (64, 320, 511), (65, 256, 2050),
                                   (128, 512, 999), (129, 64, 3001), (255, 448, 777), (256, 256, 256), (257, 128, 5000), (300, 1024, 4100), (513, 576, 1300)])
def test_bf16(R, d, V):
    _check(R, d, V, "bf16", tau=0.8)


@pytest.mark.parametrize("R,d,V", [(1, 1, 1), (1, 3, 5), (2, 64, 63), (17, 33, 100), (61, 64, 1000), (64, 100, 64), (65, 129, 515), (200, 31, 3000), (130, 257, 260)])
def test_f32(R, d, V):
    _check(R, d, V, "f32", tau=1.25)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_weights_and_with_all_rows(dtype):
    _check(40, 128, 900, dtype, weights=False, skip=False)


def test_a_long_vocabulary():
    _check(48, 512, 126464, "bf16")


def test_more_rows_than_a_block():
    """8192 rows at a time: 8300 are two blocks, the second one short; grad_w is summed over both in float32."""
    _check(8300, 64, 300, "bf16")
    _check(8300, 20, 70, "f32")


# ---- to the last bit -----------------------------------------------------------------------------
# With h = 0 (or W = 0) every p is 1 / V; with V a power of two G is w / V, or w (1 / V - 1), whose rounding to bf16 is made good, and whole numbers up to 4 in
# W (or h) make every product and every sum a whole number of w / V (or of the label's element) that float32 holds.
def _rounded(x):
    return x.to(torch.bfloat16).double()


def _uniform(R, V, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    labels = torch.randint(0, V, (R,), generator=g, device="cuda").to(torch.int32)
    labels[torch.rand(R, generator=g, device="cuda") < 0.2] = -1
    w = 2.0 ** torch.randint(-2, 3, (R,), generator=g, device="cuda").float()
    on = labels >= 0
    G = _rounded((w / V)[:, None].expand(R, V).clone())
    rows = torch.nonzero(on)[:, 0]
    G[rows, labels[rows].long()] = (w.double() * (1.0 / V - 1.0))[rows]
    return labels, w, G * on[:, None]


@pytest.mark.parametrize("V", [256, 1024, 16384])
@pytest.mark.parametrize("R,d", [(1, 64), (20, 128), (32, 256), (33, 320), (64, 512), (100, 64), (128, 1024), (129, 192), (256, 256), (300, 704), (700, 4096)])
def test_grad_h_to_the_last_bit(R, d, V):
    labels, w, G = _uniform(R, V, R + d)
    W = torch.randint(-4, 5, (V, d), generator=torch.Generator(device="cuda").manual_seed(d), device="cuda").to(torch.bfloat16)
    op = fb.HeadCrossEntropyGrad(R, d, V, grad_w=False)
    ce, loss, gh, gw = op(torch.zeros(R, d, dtype=torch.bfloat16, device="cuda"), W, labels, w)
    assert gw is None and torch.equal(gh, (G @ W.double()).float().to(torch.bfloat16))


@pytest.mark.parametrize("V", [256, 1024, 16384])
@pytest.mark.parametrize("R,d", [(1, 64), (20, 128), (64, 256), (65, 320), (127, 512), (128, 64), (300, 704), (1000, 4096), (2100, 192), (9000, 64)])
def test_grad_w_to_the_last_bit(R, d, V):
    labels, w, G = _uniform(R, V, R + d + 1)
    h = torch.randint(-4, 5, (R, d), generator=torch.Generator(device="cuda").manual_seed(d), device="cuda").to(torch.bfloat16)
    op = fb.HeadCrossEntropyGrad(R, d, V, grad_h=False)
    ce, loss, gh, gw = op(h, torch.zeros(V, d, dtype=torch.bfloat16, device="cuda"), labels, w)
    assert gh is None and torch.equal(gw, (G.t().contiguous() @ h.double()).float().to(torch.bfloat16))


# ---- differences ---------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_against_differences(dtype):
    """(L(x + e u) - L(x - e u)) / 2 e of the weighted loss in 64 bits along random directions.  The difference is off by e^2 / 6 times a third
    derivative, of at most 2 Z^3 per unit of weight for directions that change a logit by at most Z: below 1e-7 of the sum of weights here."""
    R, d, V = 24, 64, 130
    h, W, labels, w = _case(R, d, V, dtype)
    op = fb.HeadCrossEntropyGrad(R, d, V, dtype=dtype)
    _, _, gh, gw = (t.double() for t in op(h, W, labels, w))

    def loss(h, W):
        z = h @ W.t().contiguous()
        on = labels >= 0
        ce = torch.logsumexp(z, 1) - z.gather(1, labels.long().clamp(min=0)[:, None])[:, 0]
        return float((ce * w.double() * on).sum())

    g = torch.Generator(device="cuda").manual_seed(3)
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
    for x, grad, at in ((h, gh, 0), (W, gw, 1)):
        for _ in range(4):
            u = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64) * float(x.double().std())
            e = 1e-4
            args = [h.double(), W.double()]
            up, down = list(args), list(args)
            up[at], down[at] = args[at] + e * u, args[at] - e * u
            slope = (loss(*up) - loss(*down)) / (2 * e)
            Z = float((u @ W.double().t().contiguous() if at == 0 else h.double() @ u.t().contiguous()).abs().max())
            # six standard deviations of independent roundings of the elements of grad
            tol = e * e / 3 * Z ** 3 * float(w.abs().sum()) + 6 * 3 * half * float((grad * u).norm())
            assert abs(float((grad * u).sum()) - slope) <= tol


# ---- what may go wrong -----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_do_not_count_may_hold_anything(dtype):
    R, d, V = 70, 64, 300
    h, W, labels, w = _case(R, d, V, dtype)
    op = fb.HeadCrossEntropyGrad(R, d, V, dtype=dtype)
    want = [t.clone() for t in op(h, W, labels, w)]
    h[labels < 0] = float("nan")
    h[1, :5] = float("inf")
    w[labels < 0] = float("nan")
    for a, b in zip(want, op(h, W, labels, w)):
        assert torch.equal(a, b)


def test_no_row_counts():
    h, W, labels, w = _case(5, 64, 100, "bf16")
    labels.fill_(-1)
    ce, loss, gh, gw = fb.HeadCrossEntropyGrad(5, 64, 100)(h, W, labels, w)
    assert float(loss) == 0 and not bool(ce.any()) and not bool(gh.any()) and not bool(gw.any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_label_behind_the_vocabulary(dtype):
    h, W, labels, w = _case(70, 64, 300, dtype)
    op = fb.HeadCrossEntropyGrad(70, 64, 300, dtype=dtype)
    want = [t.clone() for t in op(h, W, labels, w)]
    labels[9] = 300
    ce, loss, gh, gw = op(h, W, labels, w)
    others = [i for i in range(70) if i != 9]
    assert bool(ce[9].isnan()) and bool(gh[9].isnan().all()) and bool(gw.isnan().all()) and bool(loss.isnan().all())
    assert torch.equal(ce[others], want[0][others]) and torch.equal(gh[others], want[2][others])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_confident_rows_and_large_logits(dtype):
    """Rows whose label has all the mass, and rows whose label has none: gradients of 0 and of the whole difference of two rows of W."""
    d, V = 64, 200
    W = torch.zeros(V, d, device="cuda")
    W[torch.arange(V), torch.arange(V) % d] = torch.where(torch.arange(V, device="cuda") < d, 8.0, 1.0)
    h = torch.zeros(2, d, device="cuda")
    h[:, 3] = 64.0  # logits 512 (token 3), 64 (tokens 67, 131, 195), 0
    op = fb.HeadCrossEntropyGrad(2, d, V, dtype=dtype)
    ce, loss, gh, gw = op(h.to(KIND[dtype]), W.to(KIND[dtype]), torch.tensor([3, 5], dtype=torch.int32, device="cuda"))
    assert ce.tolist() == [0.0, 512.0] and not bool(gh[0].any())
    assert torch.equal(gh[1].float(), W[3] - W[5])
    want = torch.zeros(V, d, device="cuda")
    want[3], want[5] = h[1], -h[1]
    assert torch.equal(gw.float(), want)


def test_the_same_loss_as_the_forward_call():
    R, d, V = 300, 256, 5000
    h, W, labels, w = _case(R, d, V, "bf16")
    a, b = fb.HeadCrossEntropy(R, d, V), fb.HeadCrossEntropyGrad(R, d, V)
    ce = a(h, W, labels)[0].clone()
    assert torch.allclose(ce, b(h, W, labels)[0], rtol=0, atol=1e-4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_same_bits_again_in_a_graph_and_on_another_stream(dtype):
    R, d, V = 150, 128, 3000
    op = fb.HeadCrossEntropyGrad(R, d, V, dtype=dtype)
    h, W, labels, w = _case(R, d, V, dtype)
    op(h, W, labels, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op(h, W, labels, w)
    other = fb.HeadCrossEntropyGrad(R, d, V, dtype=dtype)
    for turn in range(3):
        new = _case(R, d, V, dtype, seed=turn + 1)
        for a, b in zip((h, W, labels, w), new):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (op.out_ce, op.out_loss, op.grad_h, op.grad_w)]
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            want = other(h, W, labels, w)
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_calls_at_once():
    R, d, V = 200, 256, 4000
    ops = [fb.HeadCrossEntropyGrad(R, d, V) for _ in range(2)]
    cases = [_case(R, d, V, "bf16", seed=i) for i in range(2)]
    want = [[t.clone() for t in op(*c)] for op, c in zip(ops, cases)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for op, c, s in zip(ops, cases, streams):
            with torch.cuda.stream(s):
                op(*c)
    torch.cuda.synchronize()
    for op, ts in zip(ops, want):
        assert all(torch.equal(a, b) for a, b in zip((op.out_ce, op.out_loss, op.grad_h, op.grad_w), ts))


def test_nothing_is_written_behind_the_gradients():
    R, d, V = 33, 64, 130
    h, W, labels, w = _case(R, d, V, "bf16")
    op = fb.HeadCrossEntropyGrad(R, d, V)
    guard_h, guard_w = (torch.full((n + 4, d), 9.0, dtype=torch.bfloat16, device="cuda") for n in (R, V))
    op.grad_h, op.grad_w = guard_h[2:R + 2], guard_w[2:V + 2]
    op(h, W, labels, w)
    for g, n in ((guard_h, R), (guard_w, V)):
        assert bool((g[:2] == 9).all()) and bool((g[n + 2:] == 9).all())
