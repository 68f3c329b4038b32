"""The gradient's products to the last bit, in both types: every row's law is one token (its logit is 1344 above the others), so that G is
+-w at two tokens and 0 elsewhere, and whole numbers make every product and every sum exact.

The bf16 head takes its exponentials in base 2 with the maximum's product rounded: 2^(x log2e - fl(m log2e)) for the maximum itself is off
by |m| 2^-24, as is the rounding of the log-sum-exp to float32, so p of the one token is 1 - e, e <= 2^-23 |m| < 2^-12 here.  p rounds to
1 in bf16 (half a step is 2^-9); where the label is the token, G is -e w in place of 0.  Only these rows' terms have a tolerance (and
what they are added to that of a rounding)."""
import pytest
import torch

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.gpu
KIND = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rows(R, d, V, dtype, seed):
    """h: 64 in one of the first columns, whole numbers in the last ones, where W is the same for every token and moves no law."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    laws = max(1, min(d // 2, V))
    whole = lambda low, high, *shape: torch.randint(low, high, shape, generator=g, device="cuda").float()  # noqa: E731
    W = whole(0, 4, V, d)
    W[:, laws:] = whole(-3, 4, 1, d - laws)
    tops = torch.randperm(V, generator=g, device="cuda")[:laws]
    W[tops, torch.arange(laws, device="cuda")] = 24.0
    at = torch.randint(0, laws, (R,), generator=g, device="cuda")
    h = torch.zeros(R, d, device="cuda")
    h[:, laws:] = whole(-4, 5, R, d - laws)
    h[torch.arange(R, device="cuda"), at] = 64.0
    labels = torch.randint(0, V, (R,), generator=g, device="cuda").to(torch.int32)
    labels[torch.rand(R, generator=g, device="cuda") < 0.2] = -1
    labels[0] = V - 1
    w = 2.0 ** torch.randint(-2, 3, (R,), generator=g, device="cuda").float()
    on = (labels >= 0).double() * w.double()
    G = torch.zeros(R, V, dtype=torch.float64, device="cuda")
    rows = torch.arange(R, device="cuda")
    G[rows, tops[at]] += on
    G[rows, labels.clamp(min=0).long()] -= on
    hit = (on > 0) & (labels == tops[at])  # their term of G is 0 but for e
    spare = torch.zeros_like(G)
    if dtype == "bf16":
        z = (h.double() @ W.double().t().contiguous()).abs().amax(1)
        spare[rows, tops[at]] = hit * w * (z + 1) * 2.0 ** -23 * 1.02  # (the bf16 roundings of G and of the result: 2^-8 each)
    return h.to(KIND[dtype]), W.to(KIND[dtype]), labels, w, G, spare


def _same(got, want, spare, magnitudes, terms, dtype):
    """Equal, but where `spare` is not 0."""
    want = want.float()
    tol = torch.where(spare > 0, spare + 2.0 ** -8 * want.abs().double() + terms * 2.0 ** -24 * magnitudes, 0.0)
    assert bool(((got.double() - want.to(KIND[dtype]).double()).abs() <= tol).all())


def _check(R, d, V, dtype, seed):
    h, W, labels, w, G, spare = _rows(R, d, V, dtype, seed)
    op = fb.HeadCrossEntropyGrad(R, d, V, dtype=dtype)
    op.workspace.fill_(255)
    _, _, gh, gw = op(h, W, labels, w)
    h, W = h.double(), W.double()
    turned = lambda t: t.t().contiguous()  # noqa: E731
    _same(gh, G @ W, spare @ W.abs(), G.abs() @ W.abs(), V, dtype)
    _same(gw, turned(G) @ h, turned(spare) @ h.abs(), turned(G).abs() @ h.abs(), R, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,d,V", [(1, 64, 130), (5, 64, 1000), (16, 1024, 2000), (31, 128, 4001), (33, 192, 515), (64, 320, 1023), (65, 128, 127), (70, 2048, 300),
                                   (129, 256, 1999), (200, 64, 16500), (257, 512, 700), (1030, 128, 129), (40, 64, 70000)])
def test_products(R, d, V, dtype):
    _check(R, d, V, dtype, R + V)


@pytest.mark.parametrize("R,d,V", [(1, 1, 1), (3, 2, 9), (17, 5, 64), (64, 30, 200), (65, 4, 333), (66, 12, 65), (100, 36, 129), (130, 33, 700), (33, 130, 40),
                                   (300, 68, 1001), (9000, 8, 90)])
def test_products_of_any_width(R, d, V):
    _check(R, d, V, "f32", R + V + d)
