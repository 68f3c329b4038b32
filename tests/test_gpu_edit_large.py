"""fef_edit_logits at sizes that take its other kernels: 512 threads x 8 tokens (2^25 logits and more) and 512 x 4 (histories of 16384 and
more), and rows of more than 512 pairs (a second pass of the merge).  Compared with the definition in 64 bits on some of the sequences, with
the tolerance of test_gpu_edit_logits.py."""
import numpy as np
import pytest
import torch

from test_gpu_edit_logits import _check, _inputs, _logits, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K,V,H,n_bias,mask,some", [
    (16, 16, 131101, 300, 40, "slots", (0, 7, 15)), (128, 64, 4097, 100, 9, "sequences", (0, 1, 64, 127)), (8, 16, 262400, 5000, 0, "sequences", (0, 7)),
    (1, 2, 131200, 16384, 600, "slots", (0,)), (2, 1, 264000, 50, 3, None, (0, 1)), (3, 2, 5000, 40000, 0, None, (0, 1, 2))])
def test_large(B, K, V, H, n_bias, mask, some, dtype):
    rng = np.random.default_rng(B + K + V)
    x = _inputs(rng, B, K, V, H, n_bias, mask)
    logits = _logits(rng, B, K, V, dtype)
    out, lse = _run(logits, x, 0.8)
    for b in some:
        _check(logits[b:b + 1], {k: v[b:b + 1] for k, v in x.items()}, 0.8, out[b:b + 1], lse[b:b + 1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_without_edits(dtype):
    """Every logit of 2^25 and more where nothing but the temperature is asked for, and every row's log-sum-exp: fewer than 100 roundings of
    the sum, differences from the maximum (below 100 on average) that are off by a half step each, two more half steps of the result."""
    rng = np.random.default_rng(1)
    logits = _logits(rng, 16, 16, 131101, dtype)
    out, lse = _run(logits, {}, 0.5)
    assert torch.equal(out, logits.float() * 2)
    want = torch.logsumexp(logits.double() * 2, -1)
    assert bool(((lse.double() - want).abs() <= 200 * 2.0 ** -24 + 2.0 ** -23 * want.abs()).all())
