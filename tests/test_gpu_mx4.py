"""fef_mx4_logits against the definition in 64 bits.

Tolerance.  Products of a code times its scale with a bf16 value, or with a bf16 part of a float32 one, are exact in float32 (at most
16 significant bits); d (bf16) or 3 d (float32) of them are added, each addition off by at most 2^-23 of what it adds up to (a unit of
the last place, should the multiplier cut instead of round), and 1 / tau and the multiplication by it round once each.  So a logit is
off by at most (n + 2) 2^-23 sum |h w| / tau.  The sum of magnitudes is taken for every single logit."""
import numpy as np
import pytest
import torch

from paper_2605_14305_amd import binding as fb

pytestmark = pytest.mark.gpu
MAGNITUDE = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def _weights(rng, V, d, low=100, high=135):
    codes = rng.integers(0, 256, (V, d // 2), dtype=np.uint8)
    scales = rng.integers(low, high, (V, d // 32), dtype=np.uint8)
    return codes, scales


def _dense(codes, scales):
    V, half = codes.shape
    q = np.stack((codes & 15, codes >> 4), 2).reshape(V, 2 * half)
    w = np.where(q & 8, -1.0, 1.0) * MAGNITUDE[q & 7]
    return w * np.repeat(np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127)), 32, 1)


def _hidden(rng, R, d, dtype):
    h = rng.standard_normal((R, d)) * np.exp2(rng.integers(-6, 7, (R, d)))  # magnitudes from block to block and inside one
    return torch.from_numpy(h).to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _check(got, h, w, tau, dtype):
    x = h.double().numpy()
    want, size = x @ w.T / tau, np.abs(x) @ np.abs(w).T / tau
    n = h.shape[1] * (1 if dtype == "bf16" else 3) + 2
    err = np.abs(got.cpu().double().numpy() - want)
    assert np.all(err <= n * 2.0 ** -23 * size), float((err / (size + 1e-300)).max())


SIZES = [(1, 32, 1), (1, 64, 17), (1, 512, 5000), (2, 96, 33), (3, 160, 130), (7, 1088, 1000), (8, 4096, 3001), (15, 2560, 777), (16, 128, 4096),
         (17, 576, 515), (31, 1024, 2049), (32, 3584, 1030), (33, 224, 999), (48, 512, 640), (55, 2560, 1003), (64, 1024, 1025), (65, 320, 300),
         (96, 64, 2000), (100, 192, 257), (128, 2048, 515), (129, 256, 800), (200, 1280, 333), (256, 512, 1024), (257, 128, 700), (300, 416, 520),
         (512, 640, 770),
         # runs of every number of tiles per wavefront (some of a round of workgroups are one tile shorter), steps that end in the middle of a pair
         (33, 128, 9000), (40, 192, 20000), (50, 384, 33000), (64, 576, 41003), (70, 64, 17000), (90, 448, 66000), (110, 320, 35001), (128, 704, 40000),
         (20, 64, 50001), (24, 4160, 600), (3, 4224, 333)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,d,V", SIZES)
def test_sizes(R, d, V, dtype):
    rng = np.random.default_rng(R * 7919 + d * 31 + V)
    codes, scales = _weights(rng, V, d)
    h = _hidden(rng, R, d, dtype)
    tau = (1.0, 0.7, 3.0)[V % 3]
    out = fb.Mx4Logits(R, d, V, dtype)(h.cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), temperature=tau)
    _check(out, h, _dense(codes, scales), float(np.float32(tau)), dtype)


# vocabularies and hidden sizes from which on many rows go through tiles; many row blocks through stages
LONG = [(33, 192, 8200), (48, 320, 9001), (64, 256, 8195), (65, 448, 8200), (96, 192, 8333), (100, 128, 8200), (130, 64, 8201), (150, 576, 8207),
        (300, 256, 4001), (17, 192, 16400), (50, 320, 16385), (40, 704, 20001), (40, 4160, 200), (20, 4224, 150), (130, 4352, 97),
        (272, 1024, 333), (528, 128, 2000), (100, 2112, 70), (600, 192, 50),
        # odd numbers of blocks, with every remainder of the vocabulary by four
        (1, 160, 1000), (8, 2080, 1001), (16, 1056, 20002), (17, 3616, 303), (40, 160, 8195), (70, 4064, 97), (300, 992, 150), (5, 96, 9001), (40, 4128, 70)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,d,V", LONG)
def test_sizes_with_many_rows(R, d, V, dtype):
    rng = np.random.default_rng(R * 7919 + d * 31 + V)
    codes, scales = _weights(rng, V, d)
    h = _hidden(rng, R, d, dtype)
    tau = (1.0, 0.7, 3.0)[V % 3]
    out = fb.Mx4Logits(R, d, V, dtype)(h.cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), temperature=tau)
    _check(out, h, _dense(codes, scales), float(np.float32(tau)), dtype)


@pytest.mark.parametrize("dtype,R,V", [("bf16", 40, 8300), ("bf16", 100, 8300), ("bf16", 300, 8301), ("f32", 20, 16400), ("f32", 50, 16401)])
def test_infinities_and_nan_in_tiles(dtype, R, V):
    rng = np.random.default_rng(R)
    d = 192
    codes, scales = _weights(rng, V, d, 120, 130)
    codes |= 0x11
    scales[7, 3] = scales[V - 1, 5] = 255
    h = _hidden(rng, R, d, dtype)
    h[0, 5], h[1, 100] = float("inf"), float("nan")
    whole = torch.full((R + 2, V + 13), -7.0, device="cuda")
    fb.Mx4Logits(R, d, V, dtype)(h.cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), out=whole[1:R + 1, 5:5 + V])
    out = whole[1:R + 1, 5:5 + V].cpu()
    good = torch.ones(V, dtype=torch.bool)
    good[[7, V - 1]] = False
    w = _dense(codes, scales)[good.numpy()]
    assert bool(torch.isnan(out[:, ~good]).all()) and bool(torch.isnan(out[1]).all())
    assert bool((out[0, good].double() == torch.from_numpy(np.sign(w[:, 5])) * float("inf")).all())
    _check(out[2:, good], h[2:], w, 1.0, dtype)
    whole[1:R + 1, 5:5 + V] = -7.0
    assert bool((whole == -7.0).all())


@pytest.mark.parametrize("R,V", [(1, 100), (5, 333), (40, 70), (300, 97)])
def test_output_rows_further_apart_and_nothing_else_written(R, V):
    rng = np.random.default_rng(R)
    codes, scales = _weights(rng, V, 256)
    h = _hidden(rng, R, 256, "bf16")
    whole = torch.full((R + 2, V + 13), -7.0, device="cuda")
    out = whole[1:R + 1, 5:5 + V]
    got = fb.Mx4Logits(R, 256, V)(h.cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), out=out)
    assert got is out
    _check(out, h, _dense(codes, scales), 1.0, "bf16")
    whole[1:R + 1, 5:5 + V] = -7.0
    assert bool((whole == -7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [1, 20, 70, 260])
def test_scales_over_the_whole_range(R, dtype):
    """Scales from 2^-127 on, subnormal weights among them; a scale of 255 makes its own token's logits NaN and nobody else's."""
    rng = np.random.default_rng(R)
    V, d = 150, 192
    codes, scales = _weights(rng, V, d, 0, 60)
    scales[7, 3] = 255
    scales[149, 0] = 255
    h = torch.from_numpy(rng.standard_normal((R, d)) * 2.0 ** 60).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    out = fb.Mx4Logits(R, d, V, dtype)(h.cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()).cpu()
    bad = torch.zeros(V, dtype=torch.bool)
    bad[[7, 149]] = True
    assert bool(torch.isnan(out[:, bad]).all()) and bool(torch.isfinite(out[:, ~bad]).all())
    _check(out[:, ~bad], h, _dense(codes, scales)[~bad.numpy()], 1.0, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [3, 40, 300])
def test_infinite_and_nan_hidden_states_stay_in_their_row(R, dtype):
    rng = np.random.default_rng(R)
    V, d = 90, 128
    codes, scales = _weights(rng, V, d, 120, 130)
    codes |= 0x11                                     # no code is zero: an infinity times any of them is one
    h = _hidden(rng, R, d, dtype)
    h[0, 5], h[1, 100] = float("inf"), float("nan")
    out = fb.Mx4Logits(R, d, V, dtype)(h.cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()).cpu()
    w = _dense(codes, scales)
    assert bool((out[0].double() == torch.from_numpy(np.sign(w[:, 5])) * float("inf")).all())
    assert bool(torch.isnan(out[1]).all())
    _check(out[2:], h[2:], w, 1.0, dtype)


def test_large_float32_values_and_their_low_bits():
    """All 24 bits of a float32 hidden state count: rows that differ in the last bit of one value only."""
    V, d = 64, 64
    codes = np.zeros((V, d // 2), dtype=np.uint8)
    codes[:, 0] = 0x02                                # w[:, 0] = 1, all else 0
    scales = np.full((V, d // 32), 127, dtype=np.uint8)
    x = np.zeros((4, d), dtype=np.float32)
    x[:, 0] = [16777215.0, 16777214.0, 3.4028234e38, -1.17549435e-38]
    out = fb.Mx4Logits(4, d, V, "f32")(torch.from_numpy(x).cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()).cpu()
    assert bool((out == torch.from_numpy(x[:, :1])).all())


@pytest.mark.parametrize("R", [4, 40, 300])
def test_same_bits_again_and_on_another_stream(R):
    rng = np.random.default_rng(R)
    V, d = 2000, 512
    codes, scales = (torch.from_numpy(t).cuda() for t in _weights(rng, V, d))
    h = _hidden(rng, R, d, "bf16").cuda()
    call = fb.Mx4Logits(R, d, V)
    first = call(h, codes, scales).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call.out.fill_(0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = call(h, codes, scales)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, again)


@pytest.mark.parametrize("R", [4, 100])
def test_in_a_graph(R):
    rng = np.random.default_rng(R)
    V, d = 1500, 256
    codes, scales = (torch.from_numpy(t).cuda() for t in _weights(rng, V, d))
    h = _hidden(rng, R, d, "bf16").cuda()
    call, eager = fb.Mx4Logits(R, d, V), fb.Mx4Logits(R, d, V)
    call(h, codes, scales)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(h, codes, scales)
    for i in range(4):
        h.copy_(_hidden(np.random.default_rng(i), R, d, "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(call.out, eager(h, codes, scales))
