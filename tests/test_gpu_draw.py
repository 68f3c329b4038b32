"""fef_draw_logits against its definition in 64 bits (draw_oracle.py).  What is kept, the truncated logits and the tokens have to be equal:
the masses behind these decisions are exact to 2^-44, and the inputs are generic, so that a border is nearer than that once in 10^8
rows (the oracle refuses such a row).  lse is a float32 rounding of a number that 64 bits hold: half a step.  conf: half a step, and a weight
in units of 2^-s, s = 61 - bits of V >= 32, of which half a unit is lost."""
import numpy as np
import pytest
import torch

import draw_oracle as O
from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.gpu
INF = float("inf")


def _run(x, u=None, write=True, tau=1.0, **limits):
    """x [B, K, V] float32 or bf16 on the host; limits as lists of B."""
    B, K, V = x.shape
    op = fb.DrawLogits(B, K, V, dtype="bf16" if x.dtype == torch.bfloat16 else "f32", write=write)
    for t in (op.out_lse, op.out_conf):
        t.fill_(7.0)
    kinds = dict(top_k=torch.int32, top_p=torch.float32, min_p=torch.float32, temperatures=torch.float32)
    dev = {k: torch.tensor(v, dtype=kinds[k], device="cuda") for k, v in limits.items() if v is not None}
    got = op(x.cuda(), None if u is None else u.cuda(), temperature=tau, **dev)
    torch.cuda.synchronize()
    return [None if t is None else t.cpu().numpy() for t in got]


def _check(x, u, tau=1.0, temperatures=None, top_k=None, top_p=None, min_p=None):
    tokens, conf, kept, lse, out = _run(x, u, tau=tau, temperatures=temperatures, top_k=top_k, top_p=top_p, min_p=min_p)
    B, K, V = x.shape
    rows = x.float().numpy()
    for b in range(B):
        f = lambda v, none: none if v is None else float(np.float32(v[b]))  # noqa: E731
        t = tau if temperatures is None else f(temperatures, None)
        greedy = t == 0
        for m in range(K):
            k, p, mp = 0 if top_k is None else max(0, top_k[b]), f(top_p, 1.0), f(min_p, 0.0)
            want = O.truncate(rows[b, m], u[b, m], t, k, p, mp, greedy)
            where = (b, m, V, k, p, mp)
            assert kept[b, m] == want[2], (where, kept[b, m], want[2])
            assert np.array_equal(out[b, m], want[0]), where
            assert tokens[b, m] == want[3], where
            if want[2]:
                assert abs(lse[b, m] - want[1]) <= 2.0 ** -24 * abs(want[1]) * 1.01 + 1e-12, where
                assert abs(conf[b, m] - want[4]) <= 2.0 ** -24 * want[4] * 1.01 + 2.0 ** -31, where
            else:
                assert lse[b, m] == -INF and conf[b, m] == 0.0


def _u(B, K, seed):
    return torch.from_numpy(((np.random.default_rng(seed).integers(0, 1 << 23, (B, K)) + 0.5) * 2.0 ** -23).astype(np.float32))


def _x(B, K, V, seed, spread=3.0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(B, K, V, generator=g) * spread * (0.3 + torch.rand(B, K, 1, generator=g))).to(dtype)


LIMITS = [dict(), dict(top_k=5), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=40, top_p=0.83), dict(top_p=0.97, min_p=0.01),
          dict(top_k=1), dict(top_k=300, top_p=0.999, min_p=0.002), dict(top_p=0.31, top_k=100000)]


def _limits(which, B):
    """Each sequence its own: the limit, a neighbour, none."""
    made = {}
    for name, v in which.items():
        none = {"top_k": 0, "top_p": 1.0, "min_p": 0.0}[name]
        other = {"top_k": v + 3, "top_p": v * 0.97, "min_p": v * 1.3}[name]
        made[name] = [(v, other, none)[b % 3] for b in range(B)]
    return made


@pytest.mark.parametrize("V", [1, 2, 3, 7, 64, 255, 1001, 4096, 4097, 20000])
@pytest.mark.parametrize("which", range(len(LIMITS)))
def test_limits_and_sizes(V, which):
    x = _x(3, 2, V, 100 * which + V)
    _check(x, _u(3, 2, V), tau=0.8, **_limits(LIMITS[which], 3))


@pytest.mark.parametrize("V,dtype", [(126464, torch.float32), (151936, torch.bfloat16), (100003, torch.bfloat16), (50257, torch.float32)])
@pytest.mark.parametrize("which", [1, 2, 4, 7])
def test_long_vocabularies(V, dtype, which):
    x = _x(3, 2, V, which, dtype=dtype)
    _check(x, _u(3, 2, which), **_limits(LIMITS[which], 3))


def test_a_vocabulary_of_millions():
    V = (1 << 22) + 5
    _check(_x(2, 1, V, 5), _u(2, 1, 5), top_k=[0, 50000], top_p=[0.9, 0.95])


@pytest.mark.parametrize("V", [5, 3000, 60000])
@pytest.mark.parametrize("values", [1, 2, 9])
@pytest.mark.parametrize("which", [1, 2, 4, 5])
def test_equal_logits(V, values, which):
    """Few different values: ties go to the lower id, lists of equal logits are longer than what is sorted."""
    g = torch.Generator().manual_seed(V + values)
    x = torch.randint(0, values, (3, 2, V), generator=g).float() * 0.5
    limits = dict(LIMITS[which])
    if "top_p" in limits:
        limits["top_p"] = 0.617
    _check(x, _u(3, 2, V), **_limits(limits, 3))


@pytest.mark.parametrize("p,n", [(0.5, 1000), (0.25, 4096), (0.5, 8000), (0.75, 40000)])
def test_a_mass_that_meets_top_p_exactly(p, n):
    x = torch.zeros(1, 1, n)
    tokens, conf, kept, lse, out = _run(x, torch.tensor([[0.999]]), top_p=[p])
    assert kept[0, 0] == p * n and np.isfinite(out[0, 0, :int(p * n)]).all() and tokens[0, 0] == int(np.ceil(np.float32(0.999).astype(float) * p * n)) - 1


@pytest.mark.parametrize("offset,spread", [(500.0, 3.0), (-500.0, 3.0), (0.0, 60.0), (0.0, 1e4), (1e6, 100.0), (61.0, 1.0), (63.0, 1.0), (-40.0, 2.0),
                                           (0.0, 1e-4), (0.0, 1e36), (0.0, 1e-40)])
@pytest.mark.parametrize("which", [1, 2, 3, 4])
def test_magnitudes(offset, spread, which):
    x = _x(3, 2, 5000, 7) * spread + offset
    _check(x, _u(3, 2, 7), **_limits(LIMITS[which], 3))


@pytest.mark.parametrize("which", range(len(LIMITS)))
def test_masks(which):
    """-inf, the lowest finite number, -1e4 and numbers around the line in masked places; all but one; slots that leave nothing."""
    V = 3001
    x = _x(3, 8, V, 11)
    g = torch.Generator().manual_seed(11)
    for m, v in enumerate((-INF, torch.finfo(torch.float32).min, -1e4, -2.1e38, -1.9e38)):
        x[:, m] = torch.where(torch.rand(3, V, generator=g) < 0.8, torch.full((), v), x[:, m])
    x[:, 5] = -INF
    x[:, 5, 1234] = 0.5
    x[:, 6] = -INF
    x[:, 7] = torch.finfo(torch.float32).min
    _check(x, _u(3, 8, 11), **_limits(LIMITS[which], 3))


@pytest.mark.parametrize("bad", [float("nan"), INF])
def test_slots_without_a_law(bad):
    x = _x(2, 3, 777, 13)
    x[0, 1, 700] = bad
    x[1, 2, 0] = bad
    _check(x, _u(2, 3, 13), top_k=[9, 0], top_p=[1.0, 0.9])
    y = _x(1, 1, 777, 13) * 1e38  # a temperature that makes some infinite
    _check(y, _u(1, 1, 13), tau=0.1, top_k=[9])


def test_temperatures_of_each_sequence():
    x = _x(7, 2, 2000, 17)
    t = [1.0, 0.0, 0.3, 2.5, -1.0, float("nan"), 1e-39]
    tokens, conf, kept, lse, out = _run(x, _u(7, 2, 17), temperatures=t, top_p=[0.9] * 7)
    assert (tokens[4:6] == -1).all() and (kept[4:6] == 0).all() and (lse[4:6] == -INF).all() and np.isneginf(out[4:6]).all()
    assert (kept[[1, 6]] == 1).all() and (conf[[1, 6]] == 1.0).all()
    assert np.array_equal(tokens[[1, 6]], x[[1, 6]].argmax(2).numpy())
    good = [0, 1, 2, 3]
    _check(x[good], _u(7, 2, 17)[good], temperatures=[t[i] for i in good], top_p=[0.9] * 4)


@pytest.mark.parametrize("name,value,kept", [("top_p", 0.0, 1), ("top_p", -1.0, 1), ("top_p", 1e-30, 1), ("top_p", 2.0, 500), ("top_p", float("nan"), 500),
                                             ("min_p", 1.5, 1), ("min_p", -1.0, 500), ("min_p", float("nan"), 500), ("min_p", 1.0, 2),
                                             ("top_k", -5, 500), ("top_k", 500, 500), ("top_k", 499, 499), ("top_k", 2 ** 31 - 1, 500)])
def test_ends_of_the_limits(name, value, kept):
    x = _x(1, 1, 500, 19)
    x[0, 0, 77] = x[0, 0, 400] = 20.0
    got = _run(x, _u(1, 1, 19), **{name: [value]})
    assert got[2][0, 0] == kept
    assert np.isfinite(got[4]).sum() == kept and np.isfinite(got[4][0, 0, 77])


@pytest.mark.parametrize("u,token", [(0.0, 3), (1.0, 90), (-1.0, 3), (2.0, 90), (float("nan"), 3), (1e-30, 3), (1 - 2.0 ** -24, 90)])
def test_ends_of_the_uniforms(u, token):
    x = torch.full((1, 1, 100), -INF)
    x[0, 0, [3, 50, 90]] = torch.tensor([0.0, 1.0, 0.5])
    x[0, 0, 95] = x[0, 0, 1] = -100.0  # kept without a limit, and never drawn
    tokens, conf, kept, lse, out = _run(x, torch.tensor([[u]]))
    assert tokens[0, 0] == token and kept[0, 0] == 5


def test_without_uniforms_and_without_logits():
    x = _x(2, 2, 999, 23)
    tokens, conf, kept, lse, out = _run(x, None, write=False, top_k=[4, 4])
    assert out is None
    for b in range(2):
        for m in range(2):
            want = O.truncate(x[b, m].numpy(), 0.0, k=4)
            assert (tokens[b, m], kept[b, m]) == (want[3], 4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", range(5))
def test_rows_at_any_address(dtype, shift):
    """Rows inside a larger tensor, slots outside sequences, outputs at other addresses, and nothing written around them."""
    B, K, V = 2, 3, 1003
    whole = _x(K, B, V + 9, 29, dtype=dtype).cuda()
    x = whole.permute(1, 0, 2)[:, :, shift:shift + V]
    guard = torch.full((B, K, V + 11), 5.0, device="cuda")
    out = guard[:, :, (2 * shift) % 5:][:, :, :V]
    op = fb.DrawLogits(B, K, V, dtype="bf16" if dtype == torch.bfloat16 else "f32", write=False)
    u = _u(B, K, 29)
    tokens, conf, kept, lse, got = op(x, u.cuda(), top_p=torch.tensor([0.9, 0.6], device="cuda"), out=out)
    for b in range(B):
        for m in range(K):
            want = O.truncate(x[b, m].float().cpu().numpy(), float(u[b, m]), p=float(np.float32([0.9, 0.6][b])))
            assert np.array_equal(out[b, m].cpu().numpy(), want[0]) and int(tokens[b, m]) == want[3]
    out.fill_(5.0)
    assert bool((guard == 5.0).all())


def test_the_same_bits_again_and_in_a_graph():
    x, u = _x(4, 3, 30000, 31).cuda(), _u(4, 3, 31).cuda()
    x[1] = 0.25  # a list longer than what is sorted
    op = fb.DrawLogits(4, 3, 30000)
    limits = dict(top_k=torch.tensor([50, 7000, 0, 20], dtype=torch.int32, device="cuda"), top_p=torch.full((4,), 0.9, device="cuda"))
    want = [t.clone() for t in op(x, u, **limits)]
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(want, op(x, u, **limits)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op(x, u, **limits)
    for turn in range(3):
        x.copy_(_x(4, 3, 30000, 40 + turn))
        x[1] = 0.25
        for t in (op.out, op.out_tokens, op.out_conf, op.out_lse, op.out_kept):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (op.out_tokens, op.out_conf, op.out_kept, op.out_lse, op.out)]
        assert all(torch.equal(a, b) for a, b in zip(got, op(x, u, **limits)))


def test_a_round_draws_from_truncated_laws():
    """Truncated logits as both halves of a round: every token committed is one that was kept, and the greedy variant agrees."""
    B, K, block, V = 3, 8, 16, 2000
    x = _x(2 * B, K, V, 37).cuda()
    vl, op = fb.VerifyLogits(B, K, block, V, diag=True), fb.DrawLogits(B, K, V, write=False)
    limits = dict(top_k=torch.full((B,), 30, dtype=torch.int32, device="cuda"), top_p=torch.full((B,), 0.9, device="cuda"))
    op(x[:B], out=vl.draft_logits, **limits)
    lse_q = op.out_lse.clone()
    op(x[B:], out=vl.target_logits, **limits)
    lse_p = op.out_lse.clone()
    tokens, accepted, _ = vl(5)
    assert torch.allclose(vl.diag["lse"], torch.stack((lse_q, lse_p)), rtol=0, atol=1e-5)
    kept = torch.isfinite(vl.target_logits)
    drafted = torch.isfinite(vl.draft_logits)
    assert bool(torch.gather(drafted, 2, vl.diag["draft_tokens"].long()[..., None]).all())
    for b in range(B):
        for m in range(min(int(accepted[b]) + 1, K)):
            assert bool(kept[b, m, int(tokens[b, m])])


def test_frequencies_follow_the_law():
    """2^16 uniforms, evenly spaced: each token is drawn as often as its probability says, to within one draw."""
    V, n = 50, 1 << 16
    x = _x(1, 1, V, 41).expand(n // 64, 64, V)
    u = ((torch.arange(n, dtype=torch.float64) + 0.5) / n).float().view(n // 64, 64)
    op = fb.DrawLogits(n // 64, 64, V, write=False)
    tokens, conf, *_ = op(x.contiguous().cuda(), u.cuda(), top_p=torch.full((n // 64,), 0.9, device="cuda"))
    law = np.exp(O.truncate(x[0, 0].numpy(), 0.5, p=float(np.float32(0.9)))[0].astype(np.float64))
    law /= law.sum()
    assert np.abs(np.bincount(tokens.cpu().numpy().ravel(), minlength=V) - n * law).max() <= 1.0 + 1e-6 * n
