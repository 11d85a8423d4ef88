"""Refusals of the rotary and shared-prefix calls: bad arguments come back before anything is launched (no GPU needed), and the
Python entry points check types, shapes and devices."""
import ctypes

import pytest
import torch

import paper_2410_18234_amd as mdss
from paper_2410_18234_amd.rotary import _ROPE
from test_abi_cache import BAD_SHAPES, FAKE, ODD, desc

EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE = 1, 2, 3, 5
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    return mdss.load_library()


def rope(freq=0x1000, pairs=32, interleaved=0, magnitude=1.0):
    return _ROPE.pack(freq, pairs, interleaved, magnitude)


BAD_ROPES = [(dict(pairs=0), ESHAPE), (dict(pairs=-1), ESHAPE), (dict(pairs=33), ESHAPE), (dict(pairs=1 << 30), ESHAPE), (dict(magnitude=0.0), EINVAL),
             (dict(magnitude=-1.0), EINVAL), (dict(magnitude=NAN), EINVAL), (dict(magnitude=INF), EINVAL), (dict(freq=0x1004), EINVAL),
             (dict(freq=0), EINVAL)]


def rotary(lib, x=FAKE, xt=128, xh=64, dtype=1, T=4, H=2, D=64, positions=FAKE, r=None, out=ctypes.c_void_p(0x2000), ot=128, oh=64):
    return lib.mdss_rotary(x, xt, xh, dtype, T, H, D, positions, rope() if r is None else r, 0, out, ot, oh, None)


def append(lib, c=None, layer=0, key=FAKE, kst=128, value=FAKE, dtype=1, T=4, starts=FAKE, table=FAKE, width=3, lengths=FAKE, S=2,
           r=None, q=FAKE, qst=256, hq=4, q_out=ctypes.c_void_p(0x2000)):
    return lib.mdss_cache_append_rotary(desc() if c is None else c, layer, key, kst, 64, value, 128, 64, dtype, T, starts, table, width,
                                        lengths, S, rope() if r is None else r, None, q, qst, 64, hq, q_out, None, None)


def shared(lib, c=None, T=4, starts=FAKE, table=FAKE, width=3, lengths=FAKE, S=2, groups=FAKE, G=1, least=0, tokens=FAKE, rows=FAKE):
    return lib.mdss_cache_shared(desc() if c is None else c, T, starts, table, width, lengths, S, groups, G, least, tokens, rows, None)


def attention(lib, c=None, layer=0, q=FAKE, st=256, dtype=1, T=4, hq=4, starts=FAKE, table=FAKE, width=3, lengths=FAKE, S=2, tokens=FAKE,
              rows=FAKE, G=1, most=(0, 0, 0, 0), out=FAKE, ws=FAKE, wsb=1 << 20):
    return lib.mdss_cache_attention_shared(desc() if c is None else c, layer, q, st, 64, dtype, T, hq, starts, table, width, lengths, S,
                                           tokens, rows, G, 0.125, *most, out, None, ws, wsb, None)


@pytest.mark.parametrize("change,code", BAD_SHAPES)
def test_pool_sizes(lib, change, code):
    c = desc(**change)
    for call in (append, shared, attention):
        assert call(lib, c) == code
    assert lib.mdss_workspace_bytes_attention_shared(c, 4, 2, 1, 3, 4, 0, 0, 0, 0, 0) == 0


@pytest.mark.parametrize("change,code", BAD_ROPES)
def test_ropes(lib, change, code):
    r = rope(**change)
    assert rotary(lib, r=r) == code and append(lib, r=r) == code


def test_rotary(lib):
    none = ctypes.c_void_p(None)
    for change, code in ((dict(x=none), EINVAL), (dict(x=ODD), EINVAL), (dict(x=ctypes.c_void_p(0x1002), dtype=0), EINVAL), (dict(out=none), EINVAL),
                         (dict(out=ODD), EINVAL), (dict(positions=none), EINVAL), (dict(r=none), EINVAL), (dict(dtype=3), EUNSUPPORTED),
                         (dict(T=-1), ESHAPE), (dict(T=(1 << 24) + 1), ESHAPE), (dict(H=0), ESHAPE), (dict(D=0), ESHAPE), (dict(D=62), ESHAPE),
                         (dict(D=65537), ESHAPE), (dict(H=1 << 25), ESHAPE), (dict(xt=-1), EINVAL), (dict(xh=-64), EINVAL), (dict(ot=63), EINVAL),
                         (dict(oh=63), EINVAL), (dict(ot=64), EINVAL), (dict(ot=100), EINVAL), (dict(ot=64, oh=255), EINVAL), (dict(ot=127), EINVAL), (dict(out=FAKE, ot=256), EINVAL), (dict(out=FAKE, xh=128), EINVAL)):
        assert rotary(lib, **change) == code, change
    assert rotary(lib, T=0, x=none, out=none, positions=none) == 0
    # (rows that lie apart pass these checks: the next one refuses)
    for apart in (dict(ot=128), dict(ot=64, oh=256), dict(ot=64, T=1), dict(ot=64, H=1, D=64, oh=0)):
        assert rotary(lib, positions=none, **apart) == EINVAL and rotary(lib, dtype=3, **apart) == EUNSUPPORTED


def test_append(lib):
    none = ctypes.c_void_p(None)
    for change, code in ((dict(layer=-1), EINVAL), (dict(layer=2), EINVAL), (dict(key=none), EINVAL), (dict(key=ODD), EINVAL), (dict(value=none), EINVAL),
                         (dict(kst=-1), EINVAL), (dict(dtype=0), EUNSUPPORTED), (dict(T=-1), ESHAPE), (dict(starts=None, T=5), ESHAPE),
                         (dict(table=none), EINVAL), (dict(width=0), ESHAPE), (dict(lengths=none), EINVAL), (dict(S=65536), ESHAPE),
                         (dict(c=desc(k=0)), EINVAL), (dict(r=none), EINVAL), (dict(hq=3), ESHAPE), (dict(hq=-2), ESHAPE), (dict(hq=2 * 1025), ESHAPE),
                         (dict(T=1 << 24, hq=2048), ESHAPE), (dict(q=none), EINVAL), (dict(q=ODD), EINVAL), (dict(q_out=none), EINVAL),
                         (dict(q_out=FAKE), EINVAL), (dict(q_out=ctypes.c_void_p(0x2008)), EINVAL), (dict(qst=-1), EINVAL)):
        assert append(lib, **change) == code, change
    assert append(lib, T=0, key=none, value=none, q=none) == 0 and append(lib, S=0, table=none) == 0


def test_shared(lib):
    none = ctypes.c_void_p(None)
    for change, code in ((dict(T=-1), ESHAPE), (dict(starts=None, T=5), ESHAPE), (dict(table=none), EINVAL), (dict(width=0), ESHAPE), (dict(lengths=none), EINVAL),
                         (dict(S=65536), ESHAPE), (dict(S=65535, width=1 << 20), ESHAPE), (dict(groups=none), EINVAL), (dict(G=-1), ESHAPE), (dict(G=65536), ESHAPE),
                         (dict(least=-1), EINVAL), (dict(tokens=none), EINVAL), (dict(rows=none), EINVAL)):
        assert shared(lib, **change) == code, change
    assert shared(lib, S=0, T=0, G=0, table=none, groups=none, tokens=none, rows=none) == 0


def test_attention(lib):
    none = ctypes.c_void_p(None)
    for change, code in ((dict(layer=2), EINVAL), (dict(q=none), EINVAL), (dict(q=ODD), EINVAL), (dict(st=-1), EINVAL), (dict(dtype=0), EUNSUPPORTED),
                         (dict(hq=3), ESHAPE), (dict(hq=0), ESHAPE), (dict(hq=2 * 1025), ESHAPE), (dict(T=1 << 24, hq=2048), ESHAPE),
                         (dict(starts=None, T=3), ESHAPE), (dict(out=none), EINVAL), (dict(out=ctypes.c_void_p(0x1008)), EINVAL), (dict(lengths=none), EINVAL),
                         (dict(table=none), EINVAL), (dict(tokens=none), EINVAL), (dict(rows=none), EINVAL), (dict(G=-1), ESHAPE), (dict(G=65536), ESHAPE),
                         (dict(S=65536), ESHAPE), *((dict(most=tuple(-1 if i == j else 0 for j in range(4))), EINVAL) for i in range(4)),
                         (dict(ws=none), EWORKSPACE), (dict(wsb=64), EWORKSPACE), (dict(ws=ctypes.c_void_p(0x1010)), EWORKSPACE)):
        assert attention(lib, **change) == code, change
    assert attention(lib, T=0, q=none, out=none) == 0 and attention(lib, S=0) == 0
    need = lib.mdss_workspace_bytes_attention_shared(desc(), 4, 2, 1, 3, 4, 0, 0, 0, 0, 0)
    assert need >= 4 * 4 * 2 * 66 * 4 and attention(lib, wsb=need - 1) == EWORKSPACE


def test_python_arguments():
    """What the Python entry points refuse by themselves (no GPU needed)."""
    f = torch.ones(4, dtype=torch.float64)
    for bad in (dict(frequencies=f), dict(frequencies=f[:0]), dict(frequencies=f.view(2, 2)), dict(frequencies=[1.0])):
        with pytest.raises(ValueError):
            mdss.Rotary(**bad)
    for bad in (dict(dim=3), dict(dim=0), dict(dim=4, base=0.0), dict(dim=4, scale=-1.0), dict(dim=4, scale=INF), dict(dim=4, original=0),
                dict(dim=4, original=10, turns=(2.0, 1.0)), dict(dim=4, divisors=[1.0]), dict(dim=4, divisors=[1.0, 0.0])):
        with pytest.raises(ValueError):
            mdss.rotary_frequencies(**bad)
    with pytest.raises(ValueError):
        mdss.rotary(torch.zeros(2, 2, 8), None, torch.zeros(2, dtype=torch.int32))
    rope = object.__new__(mdss.Rotary)
    for name in ("frequencies", "interleaved", "magnitude", "_ref"):
        with pytest.raises(AttributeError):
            setattr(rope, name, 1)
        with pytest.raises(AttributeError):
            delattr(rope, name)


@pytest.mark.gpu
def test_another_device_than_the_current_one(monkeypatch):
    """(The current device's number is what the calls are told here.)"""
    dev = torch.device("cuda:0")
    i32 = dict(dtype=torch.int32, device=dev)
    rope = mdss.Rotary(torch.ones(4, dtype=torch.float64, device=dev))
    x, pos = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=dev), torch.zeros(3, **i32)
    c = mdss.PagedCache.empty(1, 4, 2, 64, 16, device=dev)
    table, lengths, groups = torch.zeros((3, 1), **i32), torch.ones(3, **i32), torch.tensor([0, 3], **i32)
    shared = mdss.cache_shared(c, 3, None, table, lengths, groups)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in (lambda: mdss.rotary(x, rope, pos), lambda: mdss.cache_append_rotary(c, 0, x, x, None, table, lengths, rope),
                 lambda: mdss.cache_shared(c, 3, None, table, lengths, groups),
                 lambda: mdss.cache_attention_shared(x, c, 0, None, table, lengths, shared)):
        with pytest.raises(ValueError, match="current device"):
            call()


@pytest.mark.gpu
def test_python_arguments_on_the_gpu():
    dev = torch.device("cuda:0")
    i32 = dict(dtype=torch.int32, device=dev)
    rope = mdss.Rotary(torch.ones(4, dtype=torch.float64, device=dev))
    x, pos = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=dev), torch.zeros(3, **i32)
    c = mdss.PagedCache.empty(1, 4, 2, 64, 16, device=dev)
    table, lengths = torch.zeros((3, 1), **i32), torch.ones(3, **i32)
    with pytest.raises(TypeError):
        mdss.Rotary(torch.ones(4, device=dev))
    for magnitude in (0.0, -1.0, NAN, INF):
        with pytest.raises(ValueError):
            mdss.Rotary(torch.ones(4, dtype=torch.float64, device=dev), magnitude=magnitude)
    for bad, error in (((x[0], rope, pos), ValueError), ((x.int(), rope, pos), TypeError), ((x, rope, pos.long()), TypeError), ((x, rope, pos[:2]), ValueError),
                       ((x, None, pos), TypeError), ((x.transpose(1, 2), rope, pos), ValueError), ((x[:, :, :6], rope, pos), mdss.MdssError)):
        with pytest.raises(error):
            mdss.rotary(*bad)
    for out in (x[:2], x.float(), x.cpu(), torch.empty((3, 64, 2), dtype=x.dtype, device=dev).transpose(1, 2), torch.empty((3, 1, 64), dtype=x.dtype, device=dev).expand(3, 2, 64)):
        with pytest.raises((ValueError, mdss.MdssError)):
            mdss.rotary(x, rope, pos, out=out)
    args = (c, 0, x, x, None, table, lengths)
    for more, error in ((dict(rope=None), TypeError), (dict(rope=rope, positions=pos.long()), TypeError), (dict(rope=rope, q=x[:2]), ValueError),
                        (dict(rope=rope, q=x.half()), TypeError), (dict(rope=rope, q=x, q_out=x), mdss.MdssError), (dict(rope=rope, q_out=x), ValueError),
                        (dict(rope=rope, q=x[:, :1]), mdss.MdssError), (dict(rope=rope, q=x, q_out=x[:2]), ValueError)):
        with pytest.raises(error):
            mdss.cache_append_rotary(*args, **more)
    groups = torch.tensor([0, 3], **i32)
    for bad, error in ((groups.long(), TypeError), (groups[:0], ValueError), (groups[None], ValueError)):
        with pytest.raises(error):
            mdss.cache_shared(c, 3, None, table, lengths, bad)
    with pytest.raises(mdss.MdssError):
        mdss.cache_shared(c, 4, None, table, lengths, groups)
    tokens, rows = mdss.cache_shared(c, 3, None, table, lengths, groups)
    for bad, error in (((tokens[:2], rows), ValueError), ((tokens.long(), rows), TypeError), ((tokens, rows[:, :3]), ValueError), ((tokens, rows.long()), TypeError)):
        with pytest.raises(error):
            mdss.cache_attention_shared(x, c, 0, None, table, lengths, bad)
    with pytest.raises(ValueError):
        mdss.cache_attention_shared(x, c, 0, None, table, lengths, (tokens, rows), workspace=torch.zeros(8, dtype=torch.uint8, device=dev))
