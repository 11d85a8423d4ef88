"""The scratch of calls: what a caller may pass, and whose the library's own buffers are."""
import pytest
import torch

from paper_2410_18234_amd import binding

CPU = torch.device("cpu")


@pytest.mark.parametrize("bad", [torch.zeros(1, dtype=torch.uint8).expand(4096), torch.zeros(8192, dtype=torch.uint8)[::2],
                                 torch.zeros((64, 128), dtype=torch.uint8).t(), torch.zeros(1024), torch.zeros(1023, dtype=torch.uint8)])
def test_a_workspace_is_one_piece_of_bytes(bad):
    """(A view whose elements lie elsewhere than behind its first one would have the kernels write past its memory.)"""
    with pytest.raises(ValueError):
        binding._ws_arg(CPU, 1024, bad)
    good = torch.zeros(1024, dtype=torch.uint8)
    assert binding._ws_arg(CPU, 1024, good) is good
    assert binding._ws_arg(CPU, 1024, good.view(4, 256)).data_ptr() == good.data_ptr()


@pytest.mark.gpu
def test_calls_refuse_it():
    import paper_2410_18234_amd as mdss
    dev = torch.device("cuda:0")
    bad = torch.zeros(1, dtype=torch.uint8, device=dev).expand(1 << 24)
    p = torch.full((2, 32), 1 / 32, device=dev)
    c = mdss.PagedCache.empty(1, 4, 2, 64, 16, device=dev)
    i32 = dict(dtype=torch.int32, device=dev)
    table, lengths, refs = torch.zeros((2, 3), **i32), torch.ones(2, **i32), torch.zeros(4, **i32)
    long = torch.zeros((1, 5000), **i32)
    q = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device=dev)
    calls = [lambda: mdss.induced_dist(p, p, 2, workspace=bad), lambda: mdss.cache_fork(c, table, lengths, refs, workspace=bad),
             lambda: mdss.cache_compact(c, table, lengths, refs, workspace=bad),
             lambda: mdss.cache_attention(q, c, 0, None, long, lengths[:1], workspace=bad),
             lambda: mdss.beam_select(p[None], torch.zeros((1, 2), device=dev), workspace=bad),
             lambda: mdss.accept_or_resample(p, p, torch.zeros(2, **i32), workspace=bad)]
    for call in calls:
        with pytest.raises(ValueError):
            call()


def test_threads_have_buffers_of_their_own(monkeypatch):
    """Two host threads on one stream: a call of one may launch between the launches of the other's."""
    import threading
    monkeypatch.setattr(binding, "_stream", lambda device: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    both, got = threading.Barrier(2, timeout=20), {}

    def work(i):
        first = binding._workspace(CPU, 1000)
        both.wait()
        again = binding._workspace(CPU, 500)
        larger = binding._workspace(CPU, 5000)
        got[i] = (first, again, larger)
        both.wait()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert got[0][0].data_ptr() != got[1][0].data_ptr() and got[0][2].data_ptr() != got[1][2].data_ptr()
    for first, again, larger in got.values():  # one thread's calls share a buffer, which grows
        assert first.data_ptr() == again.data_ptr() and larger.numel() == 5000
    monkeypatch.setattr(binding, "_stream", lambda device: 1)
    assert binding._workspace(CPU, 10).data_ptr() == binding._workspace(CPU, 10).data_ptr()
