"""Refusals of the cache and beam calls: bad arguments come back before anything is launched (no GPU needed), and the
Python entry points check types, shapes and devices."""
import ctypes

import pytest
import torch

import paper_2410_18234_amd as mdss
from paper_2410_18234_amd.cache import _DESC

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: every call below fails validation first
ODD = ctypes.c_void_p(0x1001)
EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE = 1, 2, 3, 5


@pytest.fixture(scope="module")
def lib():
    return mdss.load_library()


def desc(k=0x1000, v=0x1000, pages=8, layers=2, heads=2, d=64, ps=16):
    return _DESC.pack(k, v, 0x1000, 0x1000, pages, layers, heads, d, ps)


BAD_SHAPES = [(dict(pages=0), ESHAPE), (dict(pages=(1 << 24) + 1), ESHAPE), (dict(layers=0), ESHAPE), (dict(heads=0), ESHAPE),
              (dict(heads=1025), ESHAPE), (dict(d=80), EUNSUPPORTED), (dict(d=0), EUNSUPPORTED), (dict(ps=8), EUNSUPPORTED),
              (dict(ps=48), EUNSUPPORTED), (dict(ps=512), EUNSUPPORTED)]


def append(lib, c=None, layer=0, key=FAKE, kst=128, ksh=64, value=FAKE, dtype=1, T=4, starts=FAKE, table=FAKE, width=3,
           lengths=FAKE, S=2):
    return lib.mdss_cache_append(desc() if c is None else c, layer, key, kst, ksh, value, 128, 64, dtype, T, starts, table,
                                 width, lengths, S, None, None)


def attention(lib, c=None, layer=0, q=FAKE, st=256, dtype=1, T=4, hq=4, starts=FAKE, table=FAKE, width=3, lengths=FAKE, S=2,
              new=0, longest=0, out=FAKE, ws=None, wsb=0):
    return lib.mdss_cache_attention(desc() if c is None else c, layer, q, st, 64, dtype, T, hq, starts, table, width, lengths,
                                    S, 0.125, new, longest, out, None, ws, wsb, None)


def fork(lib, c=None, table=FAKE, lengths=FAKE, S=2, width=3, refs=FAKE, parent=FAKE, S_out=2,
         table_out=ctypes.c_void_p(0x2000), lengths_out=ctypes.c_void_p(0x2000), refs_out=FAKE, ws=FAKE, wsb=1 << 20):
    return lib.mdss_cache_fork(desc() if c is None else c, table, lengths, S, width, refs, parent, None, None, S_out,
                               table_out, lengths_out, refs_out, None, ws, wsb, None)


def compact(lib, c=None, table=FAKE, lengths=FAKE, S=2, width=3, refs=FAKE, table_out=FAKE,
            refs_out=ctypes.c_void_p(0x2000), used=FAKE, ws=FAKE, wsb=1 << 20):
    return lib.mdss_cache_compact(desc() if c is None else c, table, lengths, S, width, refs, table_out, refs_out, used, ws,
                                  wsb, None)


@pytest.mark.parametrize("change,code", BAD_SHAPES)
def test_pool_sizes(lib, change, code):
    c = desc(**change)
    for call in (append, attention, fork, compact):
        assert call(lib, c) == code
    assert lib.mdss_cache_copy(c, FAKE, FAKE, 1, None) == code
    assert lib.mdss_workspace_bytes_cache_fork(c, 2) == 0 and lib.mdss_workspace_bytes_cache_compact(c) == 0
    assert lib.mdss_workspace_bytes_attention(c, 4, 2, 3, 4, 0, 0, 0) == 0


def test_append(lib):
    assert append(lib, ctypes.c_void_p(None)) == EINVAL
    for change, code in ((dict(layer=-1), EINVAL), (dict(layer=2), EINVAL), (dict(key=None), EINVAL), (dict(key=ODD), EINVAL),
                         (dict(value=None), EINVAL), (dict(kst=-1), EINVAL), (dict(ksh=-64), EINVAL), (dict(dtype=0), EUNSUPPORTED),
                         (dict(dtype=7), EUNSUPPORTED), (dict(T=-1), ESHAPE), (dict(T=(1 << 24) + 1), ESHAPE),
                         (dict(starts=None, T=5), ESHAPE), (dict(table=None), EINVAL), (dict(width=0), ESHAPE),
                         (dict(width=1 << 31), ESHAPE), (dict(S=65535, width=1 << 20), ESHAPE), (dict(lengths=None), EINVAL),
                         (dict(S=-1), ESHAPE), (dict(S=65536), ESHAPE), (dict(c=desc(k=0)), EINVAL), (dict(c=desc(v=0x1008)), EINVAL)):
        assert append(lib, **change) == code, change
    assert append(lib, T=0, key=None, value=None) == 0 and append(lib, S=0, table=None) == 0


def test_attention(lib):
    for change, code in ((dict(layer=2), EINVAL), (dict(q=None), EINVAL), (dict(q=ODD), EINVAL), (dict(st=-1), EINVAL),
                         (dict(dtype=0), EUNSUPPORTED), (dict(hq=3), ESHAPE), (dict(hq=0), ESHAPE), (dict(hq=2 * 1025), ESHAPE),
                         (dict(T=1 << 24, hq=2048), ESHAPE), (dict(starts=None, T=3), ESHAPE), (dict(new=-1), EINVAL),
                         (dict(longest=-1), EINVAL), (dict(out=None), EINVAL), (dict(out=ctypes.c_void_p(0x1008)), EINVAL),
                         (dict(lengths=None), EINVAL), (dict(S=65536), ESHAPE)):
        assert attention(lib, **change) == code, change
    assert attention(lib, T=0, q=None, out=None) == 0 and attention(lib, S=0) == 0
    # a call that is split needs its workspace
    need = lib.mdss_workspace_bytes_attention(desc(), 4, 2, 5000, 4, 0, 0, 0)
    assert need > 0
    assert attention(lib, width=5000) == EWORKSPACE
    assert attention(lib, width=5000, ws=FAKE, wsb=need - 1) == EWORKSPACE
    assert attention(lib, width=5000, ws=ctypes.c_void_p(0x1010), wsb=need) == EWORKSPACE


def test_fork_and_compact(lib):
    same = ctypes.c_void_p(0x1000)
    for change, code in ((dict(refs=None), EINVAL), (dict(refs_out=None), EINVAL), (dict(table=None), EINVAL),
                         (dict(lengths=None), EINVAL), (dict(table_out=None), EINVAL), (dict(lengths_out=None), EINVAL),
                         (dict(table_out=same), EINVAL), (dict(lengths_out=same), EINVAL), (dict(parent=None, S_out=3), EINVAL),
                         (dict(width=0), ESHAPE), (dict(S_out=65536), ESHAPE), (dict(ws=None), EWORKSPACE),
                         (dict(wsb=64), EWORKSPACE), (dict(ws=ctypes.c_void_p(0x1010)), EWORKSPACE)):
        assert fork(lib, **change) == code, change
    for change, code in ((dict(refs=None), EINVAL), (dict(refs_out=FAKE), EINVAL), (dict(refs_out=None), EINVAL),
                         (dict(used=None), EINVAL), (dict(table_out=None), EINVAL), (dict(S=-1), ESHAPE),
                         (dict(ws=None), EWORKSPACE), (dict(wsb=64), EWORKSPACE)):
        assert compact(lib, **change) == code, change
    assert lib.mdss_cache_copy(desc(), None, FAKE, 1, None) == EINVAL
    assert lib.mdss_cache_copy(desc(), FAKE, FAKE, -1, None) == ESHAPE
    assert lib.mdss_cache_copy(desc(), None, None, 0, None) == 0


def test_beams(lib):
    need = lib.mdss_workspace_bytes_beam(2, 3, 1000, 4)
    assert need > 0 and lib.mdss_workspace_bytes_beam(0, 3, 1000, 4) == 0
    assert lib.mdss_workspace_bytes_beam(2, 65, 1000, 4) == 0 and lib.mdss_workspace_bytes_beam(2, 3, 0, 4) == 0

    def call(logits=FAKE, dtype=0, stride=1000, scores=FAKE, B=2, W=3, V=1000, n=4, eos=-1, parent=FAKE, done_out=FAKE,
             ws=FAKE, wsb=need):
        return lib.mdss_beam_select(logits, dtype, stride, scores, None, B, W, V, n, eos, parent, FAKE, FAKE, done_out, None,
                                    ws, wsb, None)

    for change, code in ((dict(logits=None), EINVAL), (dict(logits=ODD), EINVAL), (dict(dtype=3), EUNSUPPORTED),
                         (dict(stride=999), ESHAPE), (dict(scores=None), EINVAL), (dict(B=-1), ESHAPE), (dict(B=65536), ESHAPE),
                         (dict(B=30000), ESHAPE), (dict(W=0), ESHAPE), (dict(W=65), ESHAPE), (dict(n=0), ESHAPE), (dict(n=65), ESHAPE),
                         (dict(V=0), ESHAPE), (dict(V=(1 << 23) + 1, stride=1 << 24), ESHAPE), (dict(eos=-2), EINVAL),
                         (dict(eos=1000), EINVAL), (dict(parent=None), EINVAL), (dict(done_out=None), EINVAL),
                         (dict(ws=None), EWORKSPACE), (dict(wsb=need - 1), EWORKSPACE)):
        assert call(**change) == code, change
    assert call(B=0, logits=None, ws=None) == 0
    r = lib.mdss_beam_reorder
    other = ctypes.c_void_p(0x2000)
    assert r(FAKE, FAKE, 2, 3, 4, 8, FAKE, None) == EINVAL and r(None, FAKE, 2, 3, 4, 8, other, None) == EINVAL
    assert r(FAKE, FAKE, 2, 3, 4, -1, other, None) == ESHAPE and r(FAKE, FAKE, 2, 99, 4, 8, other, None) == ESHAPE
    assert r(None, None, 2, 3, 4, 0, None, None) == 0


def test_python_checks():
    x = torch.zeros((1, 2, 10))
    with pytest.raises(ValueError):
        mdss.beam_select(x, torch.zeros((1, 2)))
    with pytest.raises(ValueError):
        mdss.beam_reorder(x, torch.zeros((1, 2), dtype=torch.int32))
    k = torch.zeros((1, 2, 1, 1, 4, 16, 16), dtype=torch.uint8)
    with pytest.raises(ValueError):
        mdss.PagedCache(k, torch.zeros((1, 2, 1, 1, 64, 16), dtype=torch.uint8), torch.zeros((1, 2, 1), dtype=torch.int8),
                        torch.zeros((1, 2, 1), dtype=torch.int8))
    with pytest.raises(ValueError):
        mdss.PagedCache.empty(1, 2, 1, 64, 20, device="cpu")


@pytest.mark.gpu
def test_python_checks_on_the_gpu():
    c = mdss.PagedCache.empty(1, 4, 2, 64, 16)
    i32 = dict(dtype=torch.int32, device="cuda:0")
    table, lengths, starts, refs = torch.zeros((2, 3), **i32), torch.ones(2, **i32), torch.zeros(3, **i32), torch.zeros(4, **i32)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda:0")
    with pytest.raises(TypeError):
        mdss.cache_attention(q.float(), c, 0, starts, table, lengths)
    with pytest.raises(ValueError):
        mdss.cache_attention(q[:, :, :32], c, 0, starts, table, lengths)
    with pytest.raises(ValueError):
        mdss.cache_attention(q.transpose(1, 2).contiguous().transpose(1, 2), c, 0, starts, table, lengths)
    with pytest.raises(ValueError):
        mdss.cache_attention(q, c, 0, starts[:2], table, lengths)
    with pytest.raises(TypeError):
        mdss.cache_attention(q, c, 0, starts, table.long(), lengths)
    with pytest.raises(mdss.MdssError):
        mdss.cache_attention(q[:, :3], c, 0, starts, table, lengths)
    with pytest.raises(mdss.MdssError):
        mdss.cache_attention(q, c, 1, starts, table, lengths)
    with pytest.raises(ValueError):
        mdss.cache_append(c, 0, q, q, starts, table, lengths)
    with pytest.raises(TypeError):
        mdss.cache_append(c, 0, q[:, :2], q[:, :2].half(), starts, table, lengths)
    with pytest.raises(ValueError):
        mdss.cache_fork(c, table, lengths, refs[:3])
    with pytest.raises(TypeError):
        mdss.cache_fork(c, table, lengths, refs, parent=torch.zeros(2, dtype=torch.int64, device="cuda:0"))
    with pytest.raises(ValueError):
        mdss.cache_copy(c, refs, refs[:2])
    x = torch.zeros((1, 2, 10), device="cuda:0")
    with pytest.raises(TypeError):
        mdss.beam_select(x.double(), torch.zeros((1, 2), device="cuda:0"))
    with pytest.raises(ValueError):
        mdss.beam_select(x, torch.zeros((2, 1), device="cuda:0"))
    with pytest.raises(ValueError):
        mdss.beam_select(x.transpose(1, 2), torch.zeros((1, 10), device="cuda:0"))
    with pytest.raises(mdss.MdssError):
        mdss.beam_select(x, torch.zeros((1, 2), device="cuda:0"), n=65)
