"""The beam step against oracle/beam.py.

Parents and tokens are equal wherever the 64-bit totals of neighbouring places differ by more than a total's error:
(x - m) and the two sums after it are rounded once each (2^-24 of |x - m| + |log z| and of the total) and log z is off
by 2^-21 (fp32 sums in chunks, one logarithm).  Ties within a beam are exact: the logits' own order."""
import math

import numpy as np
import pytest
import torch

import paper_2410_18234_amd as mdss
from oracle import beam as ob

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def check(x, scores, done=None, n=None, eos=-1):
    """x: logits in their type, on the CPU or (a strided view) on the GPU."""
    B, W, V = x.shape
    n = W if n is None else n
    status = torch.zeros(B * W, dtype=torch.int32, device="cuda:0")
    d = None if done is None else torch.from_numpy(np.asarray(done, np.uint8)).cuda()
    got = mdss.beam_select(x.cuda(), torch.from_numpy(scores.astype(np.float32)).cuda(), d, n=n, eos=eos, row_status=status)
    torch.cuda.synchronize()
    parent, token, score, ended = (t.cpu().numpy() for t in got)
    x64 = x.double().cpu().numpy()
    wparent, wtoken, wscore, wended, refused = ob.select(x64, scores.astype(np.float32), done, n + 1, eos)
    assert {i for i in range(B * W) if status[i].item()} == refused
    fin = np.isfinite(wscore[:, :n])
    assert np.array_equal(np.isfinite(score), fin)
    big = np.abs(np.where(np.isfinite(x64), x64, 0.0)).max() * 2 + np.abs(np.where(np.isfinite(scores), scores, 0)).max() + 20
    tol = 2.0 ** -21 + 3 * 2.0 ** -24 * big
    assert np.all(np.abs(score - wscore[:, :n])[fin] <= tol)
    for b in range(B):
        for j in range(n):
            near = [i for i in (j - 1, j + 1) if 0 <= i <= n and wparent[b, i] != wparent[b, j] and
                    abs(wscore[b, i] - wscore[b, j]) <= 2 * tol]
            if not near:
                assert (parent[b, j], token[b, j], ended[b, j]) == (wparent[b, j], wtoken[b, j], wended[b, j]), (b, j)
    return parent, token, score, ended


def logits(rng, shape, kind, scale=3.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(TYPES[kind])


def first_scores(rng, B, W):
    return np.sort(-12.0 * rng.random((B, W)), axis=1)[:, ::-1].astype(np.float32).copy()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,W,V", [(1, 1, 1), (2, 3, 2), (3, 4, 7), (1, 4, 1000), (5, 2, 4095), (2, 8, 4097), (3, 5, 50257),
                                   (1, 64, 300), (9, 1, 32000), (70, 8, 16385)])
def test_batches(B, W, V, kind):
    rng = np.random.default_rng([B, W, V])
    check(logits(rng, (B, W, V), kind), first_scores(rng, B, W))


@pytest.mark.parametrize("n", [1, 2, 7, 16, 64])
def test_more_or_fewer_places_than_beams(n):
    rng = np.random.default_rng(n)
    check(logits(rng, (2, 4, 9000), "f32"), first_scores(rng, 2, 4), n=n)
    check(logits(rng, (2, 4, 9), "bf16"), first_scores(rng, 2, 4), n=n)  # more places than candidates


@pytest.mark.parametrize("V", [131072 * 3 + 5, 1 << 21])
def test_long_rows(V):
    """Rows of many chunks, several of them a workgroup's."""
    rng = np.random.default_rng(V)
    check(logits(rng, (1, 2, V), "bf16"), first_scores(rng, 1, 2), n=5)
    check(torch.arange(2 * V, dtype=torch.float32).view(1, 2, V) / V, first_scores(rng, 1, 2), n=5)


def test_equal_logits():
    """Ties go to the lower token, and to the lower beam where the totals tie too."""
    for V in (5, 700, 4096, 20000, 70000):
        x = torch.zeros((1, 3, V))
        parent, token, _, _ = check(x, np.zeros((1, 3), np.float32))
        assert parent.tolist() == [[0, 0, 0]] and token.tolist() == [[0, 1, 2]]
        x = torch.full((2, 2, V), torch.finfo(torch.float32).min)  # a mask of the type's lowest value all over
        x[0, 0, V - 1] = 1.0
        check(x, np.zeros((2, 2), np.float32))
    x = torch.zeros((1, 2, 9000))
    x[0, 1, ::2] = -0.0  # zeros of either sign are one value
    _, token, _, _ = check(x, np.array([[-50.0, 0.0]], np.float32), n=4)
    assert token.tolist() == [[0, 1, 2, 3]]


@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_masks_and_empty_beams(kind):
    rng = np.random.default_rng(31)
    B, W, V = 6, 4, 5000
    x = logits(rng, (B, W, V), kind)
    x[torch.from_numpy(rng.random((B, W, V)) < 0.6)] = -math.inf
    x[0, 0] = -math.inf
    x[1] = -math.inf
    x[2, :] = -math.inf
    x[2, 1, 17] = 0.5
    x[3, 2] = torch.finfo(TYPES[kind]).min
    s = first_scores(rng, B, W)
    s[4] = [0.0, -math.inf, -math.inf, -math.inf]
    s[5] = [math.nan, -1.0, math.inf, -2.0]
    parent, token, score, ended = check(x, s)
    assert (parent[1] == -1).all() and (token[1] == -1).all() and np.isneginf(score[1]).all()
    assert parent[2].tolist() == [1, -1, -1, -1] and token[2, 0] == 17


def test_finished_beams_and_eos():
    rng = np.random.default_rng(32)
    B, W, V = 5, 4, 3000
    x = logits(rng, (B, W, V), "bf16")
    done = np.zeros((B, W), np.uint8)
    done[0, 0] = done[1, 2] = done[2] = 1
    x[3, :, 77] = 40.0  # eos wins
    s = first_scores(rng, B, W)
    s[2, 3] = -math.inf
    x[0, 0] = math.nan  # a finished beam's logits are not read
    parent, token, score, ended = check(x, s, done, eos=77)
    assert parent[2].tolist() == [0, 1, 2, -1] and token[2].tolist() == [77, 77, 77, -1]
    assert ended[2].tolist() == [1, 1, 1, 0] and ended[3].all()


def test_nan_and_infinite_logits_refuse_their_beam():
    rng = np.random.default_rng(33)
    x = logits(rng, (3, 3, 20000), "f32")
    x[0, 1, 19999] = math.nan
    x[1, 0, 3] = math.inf
    x[2] = math.nan
    check(x, first_scores(rng, 3, 3))


def test_strided_rows_and_misaligned_base():
    rng = np.random.default_rng(34)
    for kind in ("f32", "bf16"):
        wide = logits(rng, (4, 3, 1111), kind).cuda()
        for view in (wide[:, :, 1:1000], wide[:, :, 5:], wide[:, :, 3:8]):
            check(view, first_scores(rng, 4, 3))


def test_reorder():
    rng = np.random.default_rng(35)
    parent = np.array([[0, 2, 2, -1], [1, 1, 0, 7]], np.int32)
    for dtype, tail in ((np.int32, (5,)), (np.float64, (3, 2)), (np.uint8, (7,)), (np.int16, (1,)), (np.float32, (4096,)),
                        (np.float32, ())):
        state = (rng.random((2, 3) + tail) * 100).astype(dtype)
        got = mdss.beam_reorder(torch.from_numpy(state).cuda(), torch.from_numpy(parent).cuda())
        np.testing.assert_array_equal(got.cpu().numpy(), ob.reorder(state, parent))


def test_empty_batch():
    x = torch.empty((0, 4, 100), device="cuda:0")
    got = mdss.beam_select(x, torch.empty((0, 4), device="cuda:0"))
    assert all(t.shape == (0, 4) for t in got)


def test_graph_replays():
    rng = np.random.default_rng(36)
    x, s = logits(rng, (2, 4, 32000), "f32").cuda(), torch.from_numpy(first_scores(rng, 2, 4)).cuda()
    want = mdss.beam_select(x, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = mdss.beam_select(x, s)
    for _ in range(3):
        for t in got:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        torch.randn(1000, device="cuda:0").sum().item()
