"""PagedCache goes by its tensors' addresses: it cannot come to hold other tensors than those, and its copies go by their own."""
import copy
import pickle

import pytest
import torch

import paper_2410_18234_amd as mdss


def test_its_attributes_stay():
    cache = object.__new__(mdss.PagedCache)  # (no GPU needed)
    for name in ("k", "v", "k_exp", "v_exp", "layers", "pages", "heads", "head_dim", "page_size", "device", "_ref"):
        with pytest.raises(AttributeError):
            setattr(cache, name, torch.zeros(1))
        with pytest.raises(AttributeError):
            delattr(cache, name)


@pytest.mark.gpu
@pytest.mark.parametrize("duplicate", [copy.copy, copy.deepcopy, lambda c: pickle.loads(pickle.dumps(c))])
def test_copies_go_by_their_own_tensors(duplicate):
    cache = mdss.PagedCache.empty(2, 4, 2, 64, 16)
    other = duplicate(cache)
    apart = other.k.data_ptr() != cache.k.data_ptr()
    i32 = dict(dtype=torch.int32, device="cuda:0")
    x = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda:0")
    args = (1, x, x, None, torch.zeros((1, 1), **i32), torch.full((1,), 3, **i32))
    assert (other.layers, other.pages, other.heads, other.head_dim, other.page_size) == (2, 4, 2, 64, 16)
    mdss.cache_append(other, *args)
    for n in ("k", "v"):
        assert getattr(other, n).any() and bool(getattr(cache, n).any()) != apart
    assert int(other.k_exp[1, 0, 0]) == -8 and (int(cache.k_exp[1, 0, 0]) == -40) == apart
