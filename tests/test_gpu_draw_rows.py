"""fef_draw_logits over many long rows (a workgroup each, which skips groups of tokens that nothing is kept of) and over slices of rows,
against its definition in 64 bits.  What is equal and what is rounded: test_gpu_draw.py."""
import numpy as np
import pytest
import torch

from paper_2605_14305_amd import binding as fb
from test_gpu_draw import INF, LIMITS, _check, _limits, _u, _x

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,K,V,dtype", [(16, 8, 16384, torch.float32), (130, 1, 20001, torch.bfloat16), (9, 15, 33333, torch.float32)])
@pytest.mark.parametrize("which", [0, 1, 2, 4, 5, 7, 8])
def test_many_rows(B, K, V, dtype, which):
    x = _x(B, K, V, 3 * which + V, dtype=dtype)
    _check(x, _u(B, K, which), tau=0.7, **_limits(LIMITS[which], B))


@pytest.mark.parametrize("V", [700, 9000, 30000])
def test_top_p_after_top_k(V):
    """Around the largest top-k whose list alone decides top-p; where fewer tokens exist than it asks for; with min-p."""
    ks = [2, 3, 64, 255, 511, 512, 513, 700, 1500]
    x = _x(len(ks), 2, V, V)
    x[:, 1, 400:] = -INF
    _check(x, _u(len(ks), 2, V), top_k=ks, top_p=[(0.9, 0.5, 0.999)[b % 3] for b in range(len(ks))], min_p=[(0.0, 1e-4)[b % 2] for b in range(len(ks))])


def test_many_rows_longer_than_the_groups():
    """2816 groups of 64 tokens: what lies behind token 180224 is read again whatever it holds."""
    B, V = 128, 200003
    x = _x(B, 1, V, 3)
    x[::2, :, 190000:190040] += 9.0  # what is kept lies there
    _check(x, _u(B, 1, 3), top_k=[(50, 0, 2000)[b % 3] for b in range(B)], top_p=[(0.9, 0.7, 1.0, 0.95)[b % 4] for b in range(B)])


def _hard(B, V, seed):
    """Rows that end elsewhere than most do, one kind after the other."""
    g = torch.Generator().manual_seed(seed)
    x = _x(B, 1, V, seed)
    for b in range(B):
        row, kind = x[b, 0], b % 10
        if kind == 0:
            row.fill_(0.25)                                                # all equal
        elif kind == 1:
            row.copy_(torch.randint(0, 3, (V,), generator=g).float() * 0.5)  # three values
        elif kind == 2:
            row[V // 2 + 77] = 300.0                                       # a maximum far above any sample of the row
        elif kind == 3:
            row.mul_(30.0)                                                 # top-k ends far below the maximum
        elif kind == 4:
            row[torch.rand(V, generator=g) < 0.999] = -INF                 # few tokens
        elif kind == 5:
            row.fill_(-INF)                                                # none
        elif kind == 6:
            row[V - 1] = float("nan")
        elif kind == 7:
            row[: V - 3] = torch.finfo(torch.float32).min                  # three tokens at the end
        elif kind == 8:
            row.mul_(1e-4)
        else:
            row.copy_(torch.log_softmax(row, 0))                           # log-probabilities
    return x


@pytest.mark.parametrize("V", [20000, 16384, 50001])
@pytest.mark.parametrize("B", [40, 130])
@pytest.mark.parametrize("which", [0, 1, 2, 4, 7])
def test_rows_that_end_elsewhere(B, V, which):
    limits = dict(LIMITS[which])
    if "top_p" in limits:
        limits["top_p"] = 0.617  # no sum of equal weights
    kinds = _limits(limits, 3 * B)  # each kind of row with each limit
    _check(_hard(B, V, B + V), _u(B, 1, V), **{n: [v[b // 10 % 3] for b in range(B)] for n, v in kinds.items()})


@pytest.mark.parametrize("B", [3, 140])
def test_other_streams_at_once(B):
    """Two calls in flight, each with its own workspace, give what they give alone."""
    V = 30000
    ops = [fb.DrawLogits(B, 1, V) for _ in range(2)]
    xs = [_hard(B, V, 50 + i).cuda() for i in range(2)]
    u = _u(B, 1, 5).cuda()
    limits = dict(top_k=torch.full((B,), 60, dtype=torch.int32, device="cuda"), top_p=torch.full((B,), 0.617, device="cuda"))
    outputs = lambda op: (op.out_tokens, op.out_conf, op.out_kept, op.out_lse, op.out)  # noqa: E731
    want = [[t.clone() for t in op(x, u, **limits)] for op, x in zip(ops, xs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ops]
    for _ in range(3):
        for op, x, s in zip(ops, xs, streams):
            with torch.cuda.stream(s):
                op(x, u, **limits)
    torch.cuda.synchronize()
    for op, ts in zip(ops, want):
        assert all(torch.equal(a, b) for a, b in zip(outputs(op), ts))


@pytest.mark.parametrize("B", [6, 129])
def test_replays_follow_their_inputs(B):
    """Logits, limits and uniforms change between replays; a row that was left by one replay is an ordinary one in the next."""
    V = 17000
    x, u = _hard(B, V, 60).cuda(), _u(B, 1, 60).cuda()
    k, p = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.ones(B, device="cuda")
    op, other = fb.DrawLogits(B, 1, V), fb.DrawLogits(B, 1, V)
    op(x, u, top_k=k, top_p=p)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op(x, u, top_k=k, top_p=p)
    for turn in range(3):
        x.copy_(_hard(B, V, 61 + turn).roll(turn, 0))
        u.copy_(_u(B, 1, 61 + turn))
        k.copy_(torch.randint(0, 90, (B,)))
        p.copy_(0.3 + torch.rand(B))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((op.out_tokens, op.out_conf, op.out_kept, op.out_lse, op.out), other(x, u, top_k=k, top_p=p)):
            assert torch.equal(a, b)
    assert np.isfinite(op.out_lse.cpu().numpy()).any()
