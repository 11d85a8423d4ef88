"""Shared by the tests of the paged cache: pools on both sides, ragged batches, and random tables."""
import numpy as np
import torch

import paper_2410_18234_amd as mdss

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def to_gpu(pool):
    return mdss.PagedCache(*(torch.from_numpy(pool[n].copy()).cuda() for n in ("k", "v", "k_exp", "v_exp")))


def to_pool(cache):
    torch.cuda.synchronize()
    return {n: getattr(cache, n).cpu().numpy() for n in ("k", "v", "k_exp", "v_exp")}


def same_pool(cache, pool):
    got = to_pool(cache)
    for name, want in pool.items():
        np.testing.assert_array_equal(got[name], want, err_msg=name)


def ids(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda:0")


def starts_of(new):
    return np.concatenate(([0], np.cumsum(new))).astype(np.int32)


def tables(lengths, ps, pages, rng, extra=1):
    """Rows of distinct pages in random order."""
    per = [(x + ps - 1) // ps for x in lengths]
    order = rng.permutation(pages)
    out, at = np.full((len(lengths), max(per + [0]) + extra), -1, np.int32), 0
    for s, n in enumerate(per):
        out[s, :n] = order[at:at + n]
        at += n
    assert at <= pages
    return out


def values(rng, shape, kind, outliers=True):
    """Values as the type holds them, on the GPU and in 64 bits: heads of unlike size, some tokens that stand out."""
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-6, 7, shape[1]))[None, :, None]
    if outliers:
        x *= np.where(rng.random((shape[0], 1, 1)) < 0.1, 40.0, 1.0)
    t = torch.from_numpy(x).to(TYPES[kind])
    return t.cuda(), t.double().numpy()
