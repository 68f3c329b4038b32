"""A NaN in a hidden state of fef_verify_step: its slot is rejected, whichever half it is in, with a token of the vocabulary; the sequences
beside it keep their results to the bit."""
import numpy as np
import pytest
import torch

from paper_2605_14305_amd import binding as fb
from paper_2605_14305_amd import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which", ["draft", "target"])
@pytest.mark.parametrize("B,K,d,V,dtype,variant", [
    (3, 4, 512, 5000, "bf16", fb.FEF_GEMM_SKINNY), (3, 4, 512, 40000, "bf16", fb.FEF_GEMM_STREAM), (3, 4, 512, 40000, "bf16", fb.FEF_GEMM_ROWSTREAM),
    (20, 4, 512, 9000, "bf16", fb.FEF_GEMM_TILED256), (3, 4, 192, 9000, "f32", fb.FEF_GEMM_F32), (3, 4, 64, 250, "f32", fb.FEF_GEMM_F32)])
def test_a_nan_hidden_state_rejects_its_slot(B, K, d, V, dtype, variant, which):
    W = synth.make_head(V, d, 1)
    hd, _ = synth.make_hidden(B, K, d, 1, 0.9, 3.0 / (0.02 * np.sqrt(d)))
    if dtype == "f32":
        W, hd = W.float(), hd.float()
    W, hd = W.cuda(), hd.cuda()
    ht = hd.clone()                                   # equal laws: every draft is accepted
    vs = fb.VerifyStep(B, K, 2 * K, d, V, dtype=dtype, device="cuda:0", gemm_variant=variant)
    conf = torch.zeros(B, 2 * K, device="cuda")
    want = [t.clone() for t in vs(hd, ht, W, 4, conf=conf)]
    assert want[1].tolist() == [K] * B
    (hd if which == "draft" else ht)[1, 2, 7] = float("nan")
    conf.zero_()
    tok, acc, rem = vs(hd, ht, W, 4, conf=conf)
    assert int(acc[1]) == 2 and 0 <= int(tok[1, 2]) < V and int(tok[1, 3]) == -1
    others = [b for b in range(B) if b != 1]
    for got, ref in zip((tok, acc, rem), want):
        assert torch.equal(got[others], ref[others])
    assert bool(torch.isfinite(conf).all()) and (float(conf[1, 2]) == 0) == (which == "target")
