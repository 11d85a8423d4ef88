"""Rotary positions against oracle/rotary.py.

The bound on an element: cosine and sine are each off by at most 3 2^-24 (the series' last roundings and its truncation, 2^-25 and
less) and by the angle's: its fp32 rest, 2^-25 of half a quarter turn, below 2^-25; then the magnitude's product (2^-24), the pair's
product and its fused sum (2^-24 each): 8 2^-24 of m (|u| + |v|) covers them.  In fp64 the angle takes two roundings here and one
in the oracle, 2^-53 each, and the oracle's pair is of 64 bits: 2^-51 of the angle times that.  Then half a step of the output's type."""
import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from oracle import rotary as orot

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
LEAST = {"bf16": 1e-38, "f16": 2.0 ** -25, "f32": 1e-38}


def rope_of(freq, interleaved, magnitude=1.0):
    return mdss.Rotary(torch.from_numpy(np.asarray(freq, np.float64)).cuda(), interleaved=interleaved, magnitude=magnitude)


def close(got, x64, freq, pos, interleaved, magnitude, inverse, kind):
    magnitude = float(np.float32(magnitude))
    want = orot.rotate(x64, freq, pos, interleaved, magnitude, inverse)
    near, far = orot.slack(x64, freq, pos, interleaved, magnitude)
    got = got.double().cpu().numpy()
    tol = (8 * 2.0 ** -24 * near + 2.0 ** -51 * far) * 1.01
    tol = tol + (np.abs(want) + tol) * torch.finfo(TYPES[kind]).eps / 2 + LEAST[kind]
    dim = 2 * len(freq)
    assert np.array_equal(got[:, :, dim:], x64[:, :, dim:])
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{bad.sum()} elements, worst {np.nanmax(np.abs(got - want) / tol):.3g} of the bound"


def values(rng, shape, kind):
    t = torch.from_numpy(rng.standard_normal(shape) * np.exp2(rng.integers(-4, 5, shape[1]))[None, :, None]).to(TYPES[kind])
    return t.cuda(), t.double().numpy()


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,dim", [(1, 1, 2, 2), (1, 40, 128, 128), (3, 5, 64, 64), (17, 3, 96, 72), (5, 2, 127, 126), (9, 7, 80, 20),
                                       (2, 3, 576, 64), (33, 1, 10, 4), (130, 9, 256, 128), (7, 2, 40, 40), (4, 2, 24, 24)])
def test_layouts_and_sizes(T, H, D, dim, interleaved, kind):
    rng = np.random.default_rng([T, H, D, dim, interleaved])
    freq = orot.frequencies(dim, 10000.0, 4.0, 2048)
    pos = rng.integers(0, 5000, T).astype(np.int32)
    pos[0] = 0
    x, x64 = values(rng, (T, H, D), kind)
    for inverse in (False, True):
        got = mdss.rotary(x, rope_of(freq, interleaved, 1.125), torch.from_numpy(pos).cuda(), inverse=inverse)
        close(got, x64, freq, pos, interleaved, 1.125, inverse, kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_far_and_negative_positions(kind):
    rng = np.random.default_rng(3)
    freq = np.concatenate((orot.frequencies(64), [0.0, 1.0, 2.5, 6.283185307179586, 1000.0, 1e-9, 3.0, 0.1]))
    pos = np.array([0, 1, -1, 65535, 1 << 20, (1 << 24) + 1, 10 ** 9 + 7, (1 << 31) - 1, -(1 << 31)], np.int32)
    x, x64 = values(rng, (len(pos), 3, 80), kind)
    close(mdss.rotary(x, rope_of(freq, False), torch.from_numpy(pos).cuda()), x64, freq, pos, False, 1.0, False, kind)


@pytest.mark.parametrize("interleaved", [False, True])
def test_quarter_turns(interleaved):
    """Angles at and beside the borders of a quadrant, of all four."""
    rng = np.random.default_rng(4)
    q = np.pi / 2
    freq = np.concatenate([[k * q / 2 + d for d in (0.0, 1e-7, -1e-7, 1e-16)] for k in range(16)])
    pos = np.array([0, 1, 3, 5, 1000001], np.int32)
    x, x64 = values(rng, (len(pos), 2, 128), "f32")
    close(mdss.rotary(x, rope_of(freq, interleaved), torch.from_numpy(pos).cuda()), x64, freq, pos, interleaved, 1.0, False, "f32")


@pytest.mark.parametrize("kind,D,dim", [("bf16", 128, 128), ("f32", 96, 50), ("f16", 64, 32), ("bf16", 63, 62)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_and_in_place(kind, D, dim, interleaved):
    """Heads inside a fused product, other layouts, odd addresses; what lies beside a view stays as it is."""
    rng = np.random.default_rng([D, dim])
    freq, T, H = orot.frequencies(dim), 11, 4
    rope, pos = rope_of(freq, interleaved), rng.integers(0, 9999, T).astype(np.int32)
    p = torch.from_numpy(pos).cuda()
    wide, wide64 = values(rng, (T, 3 * H, D), kind)
    close(mdss.rotary(wide[:, H:2 * H], rope, p), wide64[:, H:2 * H], freq, pos, interleaved, 1.0, False, kind)
    close(mdss.rotary(wide[:, ::3], rope, p), wide64[:, ::3], freq, pos, interleaved, 1.0, False, kind)
    turned = wide.transpose(0, 1).contiguous().transpose(0, 1)  # [heads][T][D] in memory
    out = torch.empty_like(turned)
    assert out.stride() == turned.stride()
    got = mdss.rotary(turned, rope, p, out=out)
    assert got.data_ptr() == out.data_ptr()
    close(got, wide64, freq, pos, interleaved, 1.0, False, kind)
    row = wide[:1, :1].expand(T, H, D)  # one head for all
    close(mdss.rotary(row, rope, p), np.broadcast_to(wide64[:1, :1], (T, H, D)), freq, pos, interleaved, 1.0, False, kind)
    odd = torch.zeros(wide.numel() + 1, dtype=wide.dtype, device="cuda:0")
    odd[1:] = wide.reshape(-1)
    close(mdss.rotary(odd[1:].view(T, 3 * H, D), rope, p), wide64, freq, pos, interleaved, 1.0, False, kind)
    buffer = wide.clone()
    view = buffer[:, H:2 * H]
    assert mdss.rotary(view, rope, p, out=view).data_ptr() == view.data_ptr()
    close(view, wide64[:, H:2 * H], freq, pos, interleaved, 1.0, False, kind)
    assert torch.equal(buffer[:, :H], wide[:, :H]) and torch.equal(buffer[:, 2 * H:], wide[:, 2 * H:])


def test_many_tokens_and_none():
    """More tokens than one thread's share; a token's result does not hang on the others."""
    rng = np.random.default_rng(6)
    freq, T = orot.frequencies(32), 70001
    x, _ = values(rng, (T, 2, 32), "f16")
    pos = torch.from_numpy(rng.integers(0, 1 << 20, T).astype(np.int32)).cuda()
    rope = rope_of(freq, False)
    all_of = mdss.rotary(x, rope, pos)
    some = torch.from_numpy(rng.integers(0, T, 200)).cuda()
    assert torch.equal(all_of[some], mdss.rotary(x[some], rope, pos[some]))
    assert mdss.rotary(x[:0], rope, pos[:0]).shape == (0, 2, 32)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients(interleaved):
    """inverse takes the gradient back: against the formula's transposed map and against differences."""
    rng = np.random.default_rng(7)
    freq, T, H, D, m = orot.frequencies(20), 6, 2, 24, 1.5
    pos = rng.integers(0, 300, T).astype(np.int32)
    rope, p = rope_of(freq, interleaved, m), torch.from_numpy(pos).cuda()
    x, x64 = values(rng, (T, H, D), "f32")
    g, g64 = values(rng, (T, H, D), "f32")
    back = mdss.rotary(g, rope, p, inverse=True)
    close(back, g64, freq, pos, interleaved, m, True, "f32")
    got = back.double().cpu().numpy()
    loss = lambda z: (orot.rotate(z, freq, pos, interleaved, m) * g64).sum(axis=2)  # noqa: E731
    for d in range(D):
        step = np.zeros_like(x64)
        step[:, :, d] = 1e-3
        slope = (loss(x64 + step) - loss(x64 - step)) / 2e-3  # (linear: differences are exact but for rounding)
        np.testing.assert_allclose(got[:, :, d], slope, rtol=0, atol=1e-5 * np.abs(g64).max())
    # there and back: m^2 times what it was
    again = mdss.rotary(mdss.rotary(x, rope, p), rope, p, inverse=True)[:, :, :20].double().cpu().numpy()
    near, _ = orot.slack(x64, freq, pos, interleaved, m * m)
    assert (np.abs(again - m * m * x64[:, :, :20]) <= 2 * 10 * 2.0 ** -24 * 2 * near[:, :, :20]).all()


def test_infinities_and_nan():
    freq = orot.frequencies(8)
    x = torch.ones((4, 1, 12), device="cuda:0")
    x[0, 0, 1] = float("inf")
    x[1, 0, 5] = float("nan")
    x[2, 0, 9] = float("nan")  # past the turned part
    got = mdss.rotary(x, rope_of(freq, False), torch.tensor([3, 2, 1, 0], dtype=torch.int32, device="cuda:0")).cpu()
    hit = ~torch.isfinite(got)
    want = torch.zeros_like(hit)
    want[0, 0, [1, 5]] = want[1, 0, [1, 5]] = want[2, 0, 9] = True
    assert torch.equal(hit, want)
    assert torch.equal(got[3], torch.ones((1, 12)))


def test_another_stream_and_a_graph():
    rng = np.random.default_rng(8)
    rope = rope_of(orot.frequencies(64), True)
    x, _ = values(rng, (50, 3, 64), "bf16")
    pos = torch.arange(50, dtype=torch.int32, device="cuda:0")
    want = mdss.rotary(x, rope, pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = mdss.rotary(x, rope, pos)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = mdss.rotary(x, rope, pos)
    for k in range(3):
        pos.fill_(k)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, mdss.rotary(x, rope, pos))


def test_frequencies():
    for args in (dict(dim=64), dict(dim=2), dict(dim=128, base=500000.0, scale=8.0), dict(dim=96, scale=16.0, original=4096),
                 dict(dim=64, scale=4.0, original=1000, turns=(0.5, 8.0)), dict(dim=8, divisors=[1.0, 2.0, 3.5, 64.0])):
        got = mdss.rotary_frequencies(**args)
        assert got.dtype == torch.float64
        np.testing.assert_allclose(got.numpy(), orot.frequencies(**args), rtol=1e-14)
