"""A thousand steps with states in 8 bits: every bit of the definition in numpy's float32, and how far what is held of sqrt(v) goes from the sums that
64 bits hold, as the header says it."""
import numpy as np
import pytest
import torch

import test_gpu_adamw as one
from paper_2605_14305_amd import binding as fb

F = np.float32
N, STEPS, LR, B1, EPS = 4096, 1000, 1e-4, 0.9, 1e-8


def _gradients(seed=3):
    """Gaussian, with a spread of its own for each element."""
    rng = np.random.default_rng(seed)
    spread = np.exp(rng.standard_normal(N)) * 1e-3
    return ((rng.standard_normal(N) * spread).astype(F) for _ in range(STEPS))


# 1 % and 99 % of 0.83 to 1.20 and of 0.72 to 1.55 times the exact value.  A quantile of 4096 elements is off by sqrt(0.01 0.99 / 4096) over the
# density there, 0.027 over the standard deviation in a normal law: 0.06 standard deviations, which are 0.08 and 0.18 (and twice that
# in the longer tail above).  Four of these, rounded up.
@pytest.mark.parametrize("b2,low,high", [(0.95, 0.83 - 0.02, 1.20 + 0.04), (0.999, 0.72 - 0.05, 1.55 + 0.09)])
def test_how_far_the_second_state_goes(b2, low, high):
    o, exact = one.Oracle(np.zeros(N, F), False, False, True), np.zeros(N)
    for t, g in enumerate(_gradients(), 1):
        o.step(g, t, LR, B1, b2, EPS, 0.0)
        exact = exact * b2 + (1 - b2) * g.astype(np.float64) ** 2
    ratio = one._value(o.v, o.vs) / np.sqrt(exact)
    assert low <= np.quantile(ratio, 0.01) and np.quantile(ratio, 0.99) <= high and 0.9 <= np.median(ratio) <= 1.1


@pytest.mark.gpu
@pytest.mark.parametrize("b2", [0.95, 0.999])
def test_every_bit_of_a_thousand_steps(b2):
    grad = torch.zeros(N, device="cuda")
    op = fb.AdamW([torch.zeros(N, device="cuda")], [grad], lr=LR, betas=(B1, b2), eps=EPS, weight_decay=0.0, states="8bit")
    o = one.Oracle(np.zeros(N, F), False, False, True)
    for t, g in enumerate(_gradients(), 1):
        grad.copy_(torch.from_numpy(g))
        op.step()
        o.step(g, t, LR, B1, b2, EPS, 0.0)
        if t % 100 == 0:
            one._same(op, [o], True)
