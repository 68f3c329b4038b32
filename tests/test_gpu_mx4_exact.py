"""fef_mx4_logits on numbers whose sums are exact in any order, in every form of its kernels: the results have to be equal to the last bit.

Hidden states and weights are whole numbers of a unit, and the sum of magnitudes of a logit stays below 2^24 units, so each product and each
partial sum, in whatever order, is a float32 number: a kernel that adds in fewer than 24 bits, loses a part of a float32 hidden
state, a column, a step of its ring or a tile is off.  The sizes reach every kernel of both types: stages of one to four units per slice in
one to eight slices, tiles of every number per wavefront with rings of two and of three pairs that wrap around, and the plain kernel."""
import pytest
import torch

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.gpu
MAGNITUDE = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _dense(codes, scales):
    """[V, d] in float64 on the device."""
    lut = torch.tensor([*MAGNITUDE, *(-m for m in MAGNITUDE)], dtype=torch.float64, device="cuda")
    V, half = codes.shape
    w = torch.empty(V, half, 2, dtype=torch.float64, device="cuda")
    w[:, :, 0] = lut[(codes & 15).long()]
    w[:, :, 1] = lut[(codes >> 4).long()]
    return w.view(V, half // 16, 32).mul_(torch.exp2(scales.double() - 127)[:, :, None]).view(V, 2 * half)


def _equal(R, d, V, dtype, h, codes, scales, tau=0.5):
    out = fb.Mx4Logits(R, d, V, dtype)(h, codes, scales, temperature=tau)
    want = (h.double() @ _dense(codes, scales).t()) / tau
    assert bool((want.float().double() == want).all())
    assert torch.equal(out, want.float())


BF16 = [  # tiles, per 16 M rows x WC columns of TT tiles of tokens
        (20, 4160, 9000), (8, 4160, 50257), (1, 4160, 70000), (31, 4160, 66001), (40, 704, 9000), (48, 640, 60001), (34, 576, 70000), (64, 576, 9000),
        (64, 704, 60001), (49, 576, 70000), (96, 640, 9000), (96, 640, 20001), (96, 640, 66001), (67, 576, 50257), (104, 640, 9000), (104, 640, 17000),
        (104, 576, 33000), (97, 576, 50257), (128, 640, 65001), (300, 576, 20001), (512, 640, 33001),
        # stages: units per slice x slices, 16 and 32 rows
        (8, 256, 50257), (8, 512, 50257), (8, 1024, 151936), (8, 2048, 70000), (5, 384, 50257), (16, 768, 126464), (3, 1536, 70001), (1, 4096, 50257),
        (12, 3584, 20001), (2, 640, 50257), (20, 256, 50257), (32, 512, 50257), (24, 1024, 126464), (17, 2048, 70001), (32, 2560, 30001), (30, 384, 50257),
        (32, 4096, 9001), (300, 2048, 1000), (64, 4064, 3001), (20, 160, 1000), (5, 4128, 2001)]
F32 = [(24, 4160, 9000), (20, 4160, 20001), (17, 64, 70000), (32, 192, 66001), (24, 320, 50257), (50, 4160, 9000), (33, 832, 20001), (50, 704, 33000),
       (40, 4160, 66001), (34, 192, 50257), (40, 576, 60001), (100, 4160, 30001),
       (8, 256, 50257), (8, 512, 50257), (16, 1024, 32000), (40, 1024, 50257), (8, 2048, 70000), (150, 576, 8207), (96, 3584, 9001), (16, 4096, 20001),
       (8, 384, 126464), (64, 2560, 5001), (64, 512, 100001), (64, 4064, 3001), (4, 96, 3001), (8, 4128, 2001)]


@pytest.mark.parametrize("R,d,V,dtype", [(*s, "bf16") for s in BF16] + [(*s, "f32") for s in F32])
def test_whole_numbers(R, d, V, dtype):
    """Weights of up to 48 units (codes of up to 12 halves, scales of 1/2, 1 and 2), mostly positive, so that sums grow."""
    g = torch.Generator(device="cuda").manual_seed(R * 7919 + d * 31 + V)
    codes = torch.randint(0, 256, (V, d // 2), generator=g, device="cuda").to(torch.uint8)
    sign = torch.rand(V, d // 2, generator=g, device="cuda") < 0.8
    codes = torch.where(sign, codes & 0x77, codes)
    scales = torch.randint(126, 129, (V, d // 32), generator=g, device="cuda").to(torch.uint8)
    most = (2 ** 24 - 1) // (48 * d)
    if dtype == "bf16":
        most = min(most, 256)
    h = torch.randint(0, most + 1, (R, d), generator=g, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    _equal(R, d, V, dtype, h, codes, scales)


@pytest.mark.parametrize("R,d,V", F32)
def test_every_bit_of_a_float32_hidden_state(R, d, V):
    """Three weights of 1 or -1 per token, hidden states of 22 bits: all three of their parts count."""
    g = torch.Generator(device="cuda").manual_seed(R * 7919 + d * 31 + V + 1)
    at = torch.randint(0, d, (V, 3), generator=g, device="cuda")
    nibble = torch.where(torch.rand(V, 3, generator=g, device="cuda") < 0.5, 2, 10)
    full = torch.zeros(V, d, dtype=torch.uint8, device="cuda").scatter_(1, at, nibble.to(torch.uint8))
    codes = full[:, 0::2] | (full[:, 1::2] << 4)
    scales = torch.full((V, d // 32), 127, dtype=torch.uint8, device="cuda")
    h = (torch.randint(-2 ** 21, 2 ** 21, (R, d), generator=g, device="cuda") * 2 + 1).float()
    _equal(R, d, V, "f32", h, codes.contiguous(), scales)


ONE_OF_EACH = [(1, 64, 300), (8, 512, 3001), (20, 576, 900), (8, 4096, 1000), (40, 192, 9000), (64, 256, 20000), (130, 320, 9000), (4, 96, 500)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,d,V", ONE_OF_EACH)
def test_subnormal_weights_count(R, d, V, dtype):
    """All weights are 2^-128 times up to 24: most of them subnormal in bf16 and float32."""
    g = torch.Generator(device="cuda").manual_seed(R + d + V)
    codes = torch.randint(0, 256, (V, d // 2), generator=g, device="cuda").to(torch.uint8)
    scales = torch.randint(0, 2, (V, d // 32), generator=g, device="cuda").to(torch.uint8)
    most = min((2 ** 24 - 1) // (24 * d), 256)
    h = (torch.randint(-most, most + 1, (R, d), generator=g, device="cuda").double() * 2.0 ** 100).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    _equal(R, d, V, dtype, h, codes, scales)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,d,V", ONE_OF_EACH)
def test_every_code_with_every_scale(R, d, V, dtype):
    """One column at a time: the logit is the weight itself, infinite from 2^128 on, NaN with a scale of 255."""
    g = torch.Generator(device="cuda").manual_seed(R + d + V)
    codes = torch.randint(0, 256, (V, d // 2), generator=g, device="cuda").to(torch.uint8)
    scales = torch.randint(0, 256, (V, d // 32), generator=g, device="cuda").to(torch.uint8)
    scales[::5] = 254 - (scales[::5] & 7)
    column = torch.randint(0, d, (R,), generator=g, device="cuda")
    h = torch.zeros(R, d, device="cuda").scatter_(1, column[:, None], 1.0).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    got = fb.Mx4Logits(R, d, V, dtype)(h, codes, scales)
    w = _dense(codes, scales)
    none = (scales == 255).any(1)
    w = torch.where((scales == 255)[:, :, None].expand(-1, -1, 32).reshape(V, d), torch.nan, w)
    over = ((w.abs() >= 2.0 ** 128).any(1)) & ~none   # an infinite weight times a hidden state of 0 is NaN
    good = ~(none | over)
    assert bool(good.any()) and bool(torch.isnan(got[:, none]).all())
    assert torch.equal(got[:, good], w[good][:, column].t().float())
    if bool(over.any()):
        assert not bool(torch.isfinite(got[:, over]).any())
