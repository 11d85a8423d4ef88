"""What the cache and beam operators are timed on: attention over a paged cache held in 8 bits, appending to
that cache, forking and compacting its pages, and beam search's selection with the reordering of its states.

The cache.  A pool of pages for all layers, a page being `ps` tokens (a multiple of 16) of every head:
  k      [layers][pages][heads][ps / 16][d / 16][16 tokens][16 of d]   e4m3 codes
  v      [layers][pages][heads][ps / 16][d][16 tokens]                 e4m3 codes
  k_exp, v_exp [layers][pages][heads] int8: a value is code * 2^exp, one exponent for a page and head
A sequence is a row of `table` (page ids, -1 where there is none) and a length; `refs` counts how many rows hold
a page (0: free).  New tokens come ragged: sequence s has tokens starts[s] .. starts[s + 1] - 1.

Inputs are synthetic: normal keys and values, pages in random order, logits as in a language model's head.
Lengths and parents follow fixed patterns of the case, so that its work is known without its data.
"""
import math

import torch

own = False

_F64 = torch.float64
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_F8 = torch.float8_e4m3fn
_EMIN, _EMAX = -40, 40  # range of the cache's exponents


def _attn(name, S, n, length, heads, group, d, ps, dtype, ragged=False):
    """S sequences of up to `length` cached tokens, the last up to `n` of them new (the queries)."""
    return {"name": name, "op": "attention", "S": S, "n": n, "length": length, "heads": heads, "group": group, "d": d,
            "ps": ps, "dtype": dtype, "ragged": ragged}


def _append(name, S, n, length, heads, d, ps, dtype, ragged=False):
    """Up to `n` new tokens for each of S sequences, which hold up to `length` with them."""
    return {"name": name, "op": "append", "S": S, "n": n, "length": length, "heads": heads, "group": 1, "d": d,
            "ps": ps, "dtype": dtype, "ragged": ragged}


def _fork(name, B, W, length, layers, heads, d, ps, grow):
    """B groups of W beams over a shared prompt, every beam replaced by a parent's copy and grown by `grow`."""
    return {"name": name, "op": "fork", "B": B, "W": W, "length": length, "layers": layers, "heads": heads, "d": d,
            "ps": ps, "grow": grow}


def _compact(name, S, length, layers, heads, d, ps, hole):
    """S sequences whose pages lie scattered over a pool; `hole`: the share of them that has to move."""
    return {"name": name, "op": "compact", "S": S, "length": length, "layers": layers, "heads": heads, "d": d,
            "ps": ps, "hole": hole}


def _beam(name, B, W, V, dtype, history, masked=0.0, done=False):
    """B groups of W beams, logits over V tokens (a share `masked` of them -inf), `history` tokens reordered."""
    return {"name": name, "op": "beam", "B": B, "W": W, "V": V, "dtype": dtype, "history": history, "masked": masked,
            "done": done}


def listed():
    return [
        # One sequence, one token, a short chat: latency.
        _attn("attn_one_1x300", 1, 1, 300, 8, 4, 128, 16, "bf16"),
        # A serving batch that verifies 0 to 5 tokens for each sequence (one is a plain decode step), lengths
        # from a quarter of 4096 up.
        _attn("attn_batch_64x4096", 64, 5, 4096, 8, 4, 128, 64, "bf16", True),
        # Few sequences of 131072 tokens, one new token each: the cache's bandwidth, and the largest cache.
        _attn("attn_long_4x131072", 4, 1, 131072, 8, 8, 128, 32, "f16"),
        # Prompts in chunks of up to 1024 tokens over what is cached of them: matrix products.
        _attn("attn_prompt_4x1024", 4, 1024, 5000, 8, 4, 128, 64, "bf16", True),
        # One decode step's keys and values, in one layer.
        _append("append_256x1", 256, 1, 2000, 8, 128, 16, "bf16"),
        # The prompts of a batch, odd lengths, half precision.
        _append("append_prompt_16x2048", 16, 2048, 2500, 8, 128, 64, "f16", True),
        # A beam step of a small batch and model.
        _fork("fork_4x4", 4, 4, 300, 4, 4, 64, 16, 1),
        # A beam step of a large batch: partly filled pages are copied in 12 layers.
        _fork("fork_64x8", 64, 8, 700, 12, 8, 128, 16, 1),
        # Defragmenting a small pool, and a large one.
        _compact("compact_small", 8, 200, 4, 4, 64, 16, 0.3),
        _compact("compact_large", 96, 1000, 6, 8, 128, 32, 0.4),
        # Beam search of one prompt over 32000 tokens, 32-bit logits.
        _beam("beam_1x4x32000", 1, 4, 32000, "f32", 64),
        # A large batch and vocabulary, half of the groups with a finished beam.
        _beam("beam_64x8x128256", 64, 8, 128256, "bf16", 512, 0.02, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["decode", "decode", "verify", "prompt", "append", "append", "fork", "fork", "compact", "beam",
                     "beam"])
    d = rng.choice([64, 96, 128, 128, 128, 256])
    ps = rng.choice([16, 16, 32, 64, 128])
    heads = rng.choice([1, 2, 4, 8, 8])
    dtype = rng.choice(["bf16", "f16"])
    if op in ("decode", "verify"):
        n = 1 if op == "decode" else rng.randint(2, 16)
        length = _log_int(rng, max(n, 16), 100000)
        group = rng.choice([1, 2, 4, 5, 8, 16])
        S = _log_int(rng, 1, max(1, min(256, 120000000 // (length * heads * d), 400000000 // (length * heads * group * n))))
        c = _attn("", S, n, length, heads, group, d, ps, dtype, rng.random() < 0.5)
    elif op == "prompt":
        n = _log_int(rng, 20, 1500)
        length = n + _log_int(rng, 1, 4000)
        group = rng.choice([1, 2, 4, 8])
        S = rng.randint(1, max(1, min(8, 250000000 // (length * heads * group * n))))
        c = _attn("", S, n, length, heads, group, d, ps, dtype, rng.random() < 0.5)
    elif op == "append":
        n = rng.choice([1, 1, _log_int(rng, 2, 3000)])
        length = n + _log_int(rng, 1, 2000)
        S = _log_int(rng, 1, max(1, min(512, 24000000 // (n * heads * d))))
        c = _append("", S, n, length, heads, d, ps, dtype, rng.random() < 0.5)
        while _pool_bytes(c) > 1.5e9:
            c["S"] = max(1, c["S"] // 2)
    elif op == "fork":
        B, W = _log_int(rng, 1, 64), rng.randint(2, 8)
        c = _fork("", B, W, _log_int(rng, 20, 800), rng.randint(1, 16), heads, d, rng.choice([16, 16, 32]), rng.choice([1, 1, 4, 40]))
        while _pool_bytes(c) > 1.5e9:
            c["layers"] = max(1, c["layers"] // 2)
            c["B"] = max(1, c["B"] // 2)
    elif op == "compact":
        c = _compact("", _log_int(rng, 1, 128), _log_int(rng, 20, 1500), rng.randint(1, 16), heads, d, ps, round(rng.uniform(0.02, 0.5), 2))
        while _pool_bytes(c) > 1.5e9:
            c["layers"] = max(1, c["layers"] // 2)
            c["S"] = max(1, c["S"] // 2)
    else:
        V = _log_int(rng, 64, 130000)
        W = rng.choice([1, 2, 3, 4, 5, 8, 16])
        B = _log_int(rng, 1, max(1, min(128, 50000000 // (W * V))))
        c = _beam("", B, W, V, rng.choice(["bf16", "f16", "f32"]), _log_int(rng, 8, 1000), rng.choice([0.0, 0.0, 0.02, 0.5]),
                  rng.random() < 0.5)
    del c["name"]
    return c


# --------------------------------------------------------------------------- patterns of a case
def _lengths(case):
    """(new tokens, length) of every sequence.  Ragged: 0 .. n new ones, lengths from a quarter of the most."""
    S, n, L = case["S"], case["n"], case["length"]
    if not case["ragged"]:
        return [n] * S, [L] * S
    new = [(n - (s * 37) % (n + 1)) for s in range(S)]
    share = [1.0 - 0.75 * ((s * 0.6180339887) % 1.0) for s in range(S)]
    return new, [max(a, int(L * f)) for a, f in zip(new, share)]


def _up(a, b):
    return -(-a // b)


def _fork_rows(case):
    """(lengths, pages that a group shares, parents) of the beams: a prompt's whole pages are shared, what comes
    after them is each beam's own; children of one parent are common, and the last beam of a third group has ended."""
    B, W, ps = case["B"], case["W"], case["ps"]
    lengths, shared, parent = [], [], []
    for b in range(B):
        L = max(1, int(case["length"] * (1.0 - 0.6 * ((b * 0.6180339887) % 1.0))))
        whole = (L * 3 // 4) // ps
        shared.append(whole)
        for w in range(W):
            lengths.append(L)
            parent.append(-1 if w == W - 1 and b % 3 == 2 else b * W + (w * w + b) % W)
    return lengths, shared, parent


def _fork_counts(case):
    """Pages held before, pages copied, and pages taken."""
    lengths, shared, parent = _fork_rows(case)
    B, W, ps = case["B"], case["W"], case["ps"]
    held = sum(shared[b] + W * (_up(lengths[b * W], ps) - shared[b]) for b in range(B))
    copied = taken = 0
    for b in range(B):
        rows = [p for p in parent[b * W:(b + 1) * W] if p >= 0]
        L = lengths[b * W]
        if L % ps:
            copied += len(rows) - len(set(rows))
        taken += len(rows) * (_up(L + case["grow"], ps) - _up(L, ps))
    return held, copied, copied + taken


def _pages(case):
    if case["op"] == "fork":
        held, _, more = _fork_counts(case)
        return held + more + 8
    per = [_up(L, case["ps"]) for L in ([case["length"]] * case["S"] if case["op"] == "compact" else _lengths(case)[1])]
    if case["op"] == "compact":
        return 2 * sum(per) + 3
    return sum(per) + sum(per) // 8 + 2


def _page_bytes(case):
    return 2 * case["ps"] * case["heads"] * case["d"]


def _pool_bytes(case):
    return _pages(case) * case.get("layers", 1) * _page_bytes(case)


def _moved(case):
    used = case["S"] * _up(case["length"], case["ps"])
    return min(used, max(1, int(used * case["hole"])))


# ------------------------------------------------------------------------------------- inputs
def _pool(case, g):
    """A filled pool: codes of normal values, exponents of a few octaves."""
    L, N, H, d, ps = case.get("layers", 1), _pages(case), case["heads"], case["d"], case["ps"]

    def codes(*shape):
        out = torch.empty(shape, dtype=torch.uint8, device="cuda")
        flat = out.view(-1)
        for at in range(0, flat.numel(), 1 << 27):
            part = flat[at:at + (1 << 27)]
            part.copy_((torch.randn(part.shape, generator=g, device="cuda") * 70.0).clamp_(-448.0, 448.0).to(_F8).view(torch.uint8))
        return out

    def exps():
        return torch.randint(-7, -4, (L, N, H), generator=g, device="cuda", dtype=torch.int8)

    return {"k": codes(L, N, H, ps // 16, d // 16, 16, 16), "v": codes(L, N, H, ps // 16, d, 16), "k_exp": exps(),
            "v_exp": exps()}


def _dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def _table(counts, ids, width):
    """Rows of page ids, taken in order from `ids` (on the GPU), -1 after a row's own."""
    n = _dev(counts)
    at = torch.arange(width, device="cuda", dtype=torch.int32)[None]
    first = torch.cumsum(n, 0) - n
    where = (first[:, None] + at).clamp(max=max(ids.numel() - 1, 0)).long()
    return torch.where(at < n[:, None], ids[where].int(), torch.full_like(where, -1).int()).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    st = {"case": case}
    if op in ("attention", "append"):
        new, length = _lengths(case)
        T, H, d, ps = sum(new), case["heads"], case["d"], case["ps"]
        st.update(_pool(case, g))
        ids = torch.randperm(_pages(case), generator=g, device="cuda")
        per = [_up(x, ps) for x in length]
        starts = [0]
        for x in new:
            starts.append(starts[-1] + x)
        st.update(table=_table(per, ids, max(per) + 2), lengths=_dev(length), starts=_dev(starts))
        kind = _TYPES[case["dtype"]]
        if op == "attention":
            st["q"] = torch.randn((T, H * case["group"], d), generator=g, device="cuda").to(kind)
        else:
            # heads of unlike magnitude, now and then a token that stands out
            size = torch.exp2(torch.randint(-3, 4, (1, H, 1), generator=g, device="cuda").float())
            for name in ("key", "value"):
                x = torch.randn((T, H, d), generator=g, device="cuda") * size
                x *= 1.0 + 30.0 * (torch.rand((T, 1, 1), generator=g, device="cuda") < 0.01)
                st[name] = x.to(kind)
    elif op == "fork":
        lengths, shared, parent = _fork_rows(case)
        B, W, ps = case["B"], case["W"], case["ps"]
        N = _pages(case)
        st.update(_pool(case, g))
        ids = torch.randperm(N, generator=g, device="cuda").int()
        rows, at, width = [], 0, max(_up(x + case["grow"], ps) for x in lengths) + 1
        for b in range(B):
            own_pages = _up(lengths[b * W], ps) - shared[b]
            for w in range(W):
                first = at + shared[b] + w * own_pages
                rows.append(list(range(at, at + shared[b])) + list(range(first, first + own_pages)) +
                            [-1] * (width - shared[b] - own_pages))
            at += shared[b] + W * own_pages
        rows = _dev(rows)
        st["table"] = torch.where(rows >= 0, ids[rows.clamp(min=0).long()], rows)
        st["refs"] = torch.zeros(N, dtype=torch.int32, device="cuda")
        st["refs"].scatter_add_(0, st["table"][rows >= 0].long(), torch.ones_like(st["table"][rows >= 0]))
        st.update(lengths=_dev(lengths), parent=_dev(parent), grow=torch.full((B * W,), case["grow"], dtype=torch.int32, device="cuda"))
    elif op == "compact":
        S, ps = case["S"], case["ps"]
        per, N, moved = _up(case["length"], ps), _pages(case), _moved(case)
        used = S * per
        st.update(_pool(case, g))
        low = torch.randperm(used, generator=g, device="cuda")[:used - moved]
        high = used + torch.randperm(N - used, generator=g, device="cuda")[:moved]
        ids = torch.cat((low, high))[torch.randperm(used, generator=g, device="cuda")]
        st["table"] = _table([per] * S, ids, per + 1)
        st["refs"] = torch.zeros(N, dtype=torch.int32, device="cuda")
        st["refs"][ids] = 1
        st["lengths"] = _dev([case["length"]] * S)
    else:
        B, W, V = case["B"], case["W"], case["V"]
        x = 3.0 * torch.randn((B, W, V), generator=g, device="cuda")
        if case["masked"]:
            x.masked_fill_(torch.rand((B, W, V), generator=g, device="cuda") < case["masked"], -math.inf)
            if B > 1:
                x[1, 0] = -math.inf  # a constraint that leaves a beam nothing
        st["logits"] = x.to(_TYPES[case["dtype"]])
        st["scores"] = torch.sort(-12.0 * torch.rand((B, W), generator=g, device="cuda"), dim=1, descending=True).values
        st["done"] = torch.zeros((B, W), dtype=torch.uint8, device="cuda")
        if case["done"] and W > 1:
            st["done"][::2, 1] = 1
        st["eos"] = V // 2
        st["history"] = torch.randint(0, V, (B, W, case["history"]), generator=g, device="cuda", dtype=torch.int32)
    return st


# ---------------------------------------------------------------------------------- the calls
def _f8(x):
    return x.view(_F8)


def _pools(st):
    return {"k": _f8(st["k"]), "v": _f8(st["v"]), "k_exp": st["k_exp"], "v_exp": st["v_exp"]}


def run(state):
    c, st = state["case"], state
    op = c["op"]
    if own:
        import paper_2410_18234_amd as mdss
        if op == "beam":
            parent, token, score, done = mdss.beam_select(st["logits"], st["scores"], st["done"], eos=st["eos"])
            return {"parent": parent, "token": token, "score": score, "done": done,
                    "history": mdss.beam_reorder(st["history"], parent)}
        cache = mdss.PagedCache(st["k"], st["v"], st["k_exp"], st["v_exp"])
        if op == "attention":
            return mdss.cache_attention(st["q"], cache, 0, st["starts"], st["table"], st["lengths"], max_new=c["n"],
                                        max_length=c["length"])
        if op == "append":
            mdss.cache_append(cache, 0, st["key"], st["value"], st["starts"], st["table"], st["lengths"])
            return _pools(st)
        if op == "fork":
            table, lengths, refs = mdss.cache_fork(cache, st["table"], st["lengths"], st["refs"], st["parent"],
                                                   grow=st["grow"])
            return {"table": table, "lengths": lengths, "refs": refs, **_pools(st)}
        table, refs, used = mdss.cache_compact(cache, st["table"], st["lengths"], st["refs"])
        return {"table": table, "refs": refs, "used": used, **_pools(st)}
    return {"attention": _plain_attention, "append": _plain_append, "fork": _plain_fork, "compact": _plain_compact,
            "beam": _plain_beam}[op](st)


# ------------------------------------------------------------------------------ the plain forms
def _rows(st):
    """For every new token its sequence, its place among the sequence's new ones, and its position."""
    starts, lengths = st["starts"].long(), st["lengths"].long()
    n = starts[1:] - starts[:-1]
    T = (st["q"] if "q" in st else st["key"]).shape[0]
    t = torch.arange(T, device="cuda")
    s = torch.searchsorted(starts, t, right=True) - 1
    i = t - starts[s]
    return s, i, lengths[s] - n[s] + i


def _plain_attention(st):
    c = st["case"]
    q, table, lengths = st["q"], st["table"].long(), st["lengths"].long()
    T, S, H, G, d, ps = q.shape[0], c["S"], c["heads"], c["group"], c["d"], c["ps"]
    s, i, pos = _rows(st)
    pages = table[:, :_up(c["length"], ps)].clamp(min=0)
    L = pages.shape[1] * ps
    ks = torch.exp2(st["k_exp"][0].float())[pages][..., None, None, None, None]  # [S][pages][H]
    vs = torch.exp2(st["v_exp"][0].float())[pages][..., None, None, None]
    k = (_f8(st["k"][0][pages]).float() * ks).permute(0, 2, 1, 3, 5, 4, 6).reshape(S, H, L, d)
    v = (_f8(st["v"][0][pages]).float() * vs).permute(0, 2, 1, 3, 5, 4).reshape(S, H, L, d)
    v = v * (torch.arange(L, device="cuda") < lengths[:, None])[:, None, :, None]
    n = c["n"]
    qs = torch.zeros((S, n, H, G, d), device="cuda")
    qs[s, i] = q.float().view(T, H, G, d)
    last = torch.full((S, n), -1, device="cuda")
    last[s, i] = pos
    qs = qs.permute(0, 2, 1, 3, 4).reshape(S, H, n * G, d)
    a = torch.matmul(qs, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    hidden = torch.arange(L, device="cuda") > last[:, :, None]
    a.view(S, H, n, G, L).masked_fill_(hidden[:, None, :, None, :], -math.inf)
    m = a.amax(3, keepdim=True).clamp(min=-3e38)
    e = torch.exp(a - m)
    z = e.sum(3, keepdim=True)
    out = torch.matmul(e, v) / torch.where(z > 0, z, torch.ones_like(z))
    return out.view(S, H, n, G, d).permute(0, 2, 1, 3, 4)[s, i].reshape(T, H * G, d).to(q.dtype)


def _exponent(amax):
    """The least e with amax <= 448 * 2^e, within the exponents' range."""
    m, x = torch.frexp(amax)
    e = torch.where(m <= 0.875, x - 9, x - 8)
    return torch.where(amax > 0, e, torch.full_like(e, _EMIN)).clamp(_EMIN, _EMAX)


def _plain_append(st):
    c = st["case"]
    ps, H, N = c["ps"], c["heads"], st["k"].shape[1]
    s, i, pos = _rows(st)
    page, slot = st["table"].long()[s, pos // ps], pos % ps
    first = torch.full((N,), ps, device="cuda").scatter_reduce_(0, page, slot, "amin")
    touched = torch.unique(page)
    unit, at = slot // 16, slot % 16
    for name, x in (("k", st["key"].float()), ("v", st["value"].float())):
        codes, exps = st[name][0], st[name + "_exp"][0]
        amax = torch.zeros((N, H), device="cuda").scatter_reduce_(0, page[:, None].expand(-1, H), x.abs().amax(2), "amax")
        e, old = _exponent(amax), exps.int()
        e = torch.where(first[:, None] > 0, torch.maximum(e, old), e)
        # what such a page holds already goes to its new exponent
        held = codes[touched]
        shift = torch.exp2((old - e)[touched].float())
        again = _f8(held).float() * (shift[:, :, None, None, None, None] if name == "k" else shift[:, :, None, None, None])
        here = torch.arange(ps, device="cuda").view(ps // 16, 16) < first[touched][:, None, None]
        here = here[:, None, :, None, :, None] if name == "k" else here[:, None, :, None, :]
        codes[touched] = torch.where(here, again.to(_F8).view(torch.uint8), held)
        new = (x * torch.exp2(-e[page].float())[:, :, None]).clamp(-448.0, 448.0).to(_F8).view(torch.uint8)
        if name == "k":
            codes.permute(0, 2, 4, 1, 3, 5)[page, unit, at] = new.view(-1, H, c["d"] // 16, 16)
        else:
            codes.permute(0, 2, 4, 1, 3)[page, unit, at] = new
        exps[touched] = e[touched].to(torch.int8)
    return _pools(st)


def _plain_fork(st):
    c = st["case"]
    ps, table, lengths, refs = c["ps"], st["table"].long(), st["lengths"].long(), st["refs"].long()
    N, width = refs.numel(), table.shape[1]
    at = torch.arange(width, device="cuda")[None]
    parent, grow = st["parent"].long(), st["grow"].long()
    L = torch.where(parent >= 0, lengths[parent.clamp(min=0)], torch.zeros_like(parent))
    pages = (L + ps - 1) // ps
    t = torch.where(at < pages[:, None], table[parent.clamp(min=0)], torch.full((1, 1), -1, device="cuda"))
    before = table[at < ((lengths + ps - 1) // ps)[:, None]]
    after = t[t >= 0]
    now = refs.scatter_add(0, before, torch.full_like(before, -1)).scatter_add_(0, after, torch.ones_like(after))
    grow = torch.where(parent >= 0, grow, torch.zeros_like(grow))
    # a partly filled page that others hold too is copied by each that writes to it, but for the last where all do
    i = torch.arange(parent.numel(), device="cuda")
    part = (grow > 0) & (L % ps != 0)
    page = t.gather(1, (L // ps).clamp(max=width - 1)[:, None])[:, 0].clamp(min=0)
    writers = torch.zeros(N, dtype=torch.long, device="cuda").scatter_add_(0, page, part.long())
    keeper = torch.full((N,), -1, device="cuda").scatter_reduce_(0, page, torch.where(part, i, torch.full_like(i, -1)), "amax")
    copy = part & (now[page] > 1) & ~((writers[page] == now[page]) & (keeper[page] == i))
    more = (L + grow + ps - 1) // ps - pages
    need = more + copy
    first = torch.cumsum(need, 0) - need
    free = (refs == 0).nonzero()[:, 0]
    src, dst = page[copy], free[first[copy]]
    t[copy, (L // ps)[copy]] = dst
    added = (at >= pages[:, None]) & (at < (pages + more)[:, None])
    t = torch.where(added, free[((first + copy)[:, None] + at - pages[:, None]).clamp(0, free.numel() - 1)], t)
    now.scatter_add_(0, src, torch.full_like(src, -1))
    now[dst] = 1
    now[t[added]] = 1
    for name in ("k", "v", "k_exp", "v_exp"):
        st[name][:, dst] = st[name][:, src]
    return {"table": t.int(), "lengths": (L + grow).int(), "refs": now.int(), **_pools(st)}


def _plain_compact(st):
    table, refs = st["table"].long(), st["refs"]
    held = refs > 0
    used = held.sum()
    ids = torch.arange(refs.numel(), device="cuda")
    src = torch.flip(ids[held & (ids >= used)], (0,))  # the highest page goes to the lowest hole
    dst = ids[~held & (ids < used)]
    to = ids.clone()
    to[src] = dst
    for name in ("k", "v", "k_exp", "v_exp"):
        st[name][:, dst] = st[name][:, src]
    now = torch.zeros_like(refs)
    now[to[held]] = refs[held]
    return {"table": torch.where(table >= 0, to[table.clamp(min=0)], table).int(), "refs": now, "used": used.int(), **_pools(st)}


def _plain_beam(st):
    x, scores, done, eos = st["logits"].float(), st["scores"], st["done"].bool(), st["eos"]
    B, W, V = x.shape
    m = x.amax(2, keepdim=True)
    m = torch.where(m > -math.inf, m, torch.zeros_like(m))
    logp = (x - m) - torch.log(torch.exp(x - m).sum(2, keepdim=True))
    # a beam's candidates by their logit, then the lower token; all by their total, then the lower beam
    top = torch.sort(x, dim=2, descending=True, stable=True).indices[:, :, :W]
    total = logp.gather(2, top) + scores[:, :, None]
    total = torch.where(torch.isnan(total), torch.full_like(total, -math.inf), total)
    only = torch.full_like(total, -math.inf)
    only[:, :, 0] = scores
    total = torch.where(done[:, :, None], only, total)
    top = torch.where(done[:, :, None], torch.full_like(top, eos), top)
    n = top.shape[2]
    best = torch.sort(total.view(B, W * n), dim=1, descending=True, stable=True)
    score, at = best.values[:, :W], best.indices[:, :W]
    parent, token = at // n, top.reshape(B, W * n).gather(1, at)
    none = score == -math.inf
    ended = done.gather(1, parent) | (token == eos)
    parent, token = parent.masked_fill(none, -1), token.masked_fill(none, -1)
    rows = st["history"].gather(1, parent.clamp(min=0)[:, :, None].expand(-1, -1, st["history"].shape[2]))
    return {"parent": parent.int(), "token": token.int(), "score": score, "done": (ended & ~none).to(torch.uint8),
            "history": rows.masked_fill(none[:, :, None], 0)}


def work(case):
    op = case["op"]
    if op in ("attention", "append"):
        new, length = _lengths(case)
        T, H, d, e = sum(new), case["heads"], case["d"], 2
        if op == "append":
            return {"bytes": 2 * T * H * d * (e + 1), "flops": 0}
        hq = H * case["group"]
        seen = sum(n * (L - n) + n * (n + 1) // 2 for n, L in zip(new, length))
        cached = sum(L for n, L in zip(new, length) if n)
        return {"bytes": cached * H * d * 2 + 2 * T * hq * d * e, "flops": 4 * hq * d * seen}
    if op == "fork":
        held, copied, _ = _fork_counts(case)
        rows = case["B"] * case["W"]
        width = max(_up(x + case["grow"], case["ps"]) for x in _fork_rows(case)[0]) + 1
        return {"bytes": 2 * copied * case["layers"] * _page_bytes(case) + 8 * rows * width + 8 * _pages(case), "flops": 0}
    if op == "compact":
        return {"bytes": 2 * _moved(case) * case["layers"] * _page_bytes(case) + 8 * case["S"] * _up(case["length"], case["ps"]) +
                8 * _pages(case), "flops": 0}
    B, W, V = case["B"], case["W"], case["V"]
    rows = B * W - (_up(B, 2) if case["done"] and W > 1 else 0)
    size = 4 if case["dtype"] == "f32" else 2
    return {"bytes": rows * V * size + 8 * B * W * case["history"], "flops": 4 * rows * V}


# --------------------------------------------------------------------------- 64-bit counterparts
def _value64(codes):
    """e4m3 codes as 64-bit numbers, from their bits."""
    c = codes.to(_F64)
    sign, low = torch.floor(c / 128.0), torch.remainder(c, 128.0)
    x, m = torch.floor(low / 8.0), torch.remainder(low, 8.0)
    mag = torch.where(x > 0, (8.0 + m) * torch.exp2(x - 10.0), m * 2.0 ** -9)
    return torch.where(sign > 0, -mag, mag)


def _round64(x):
    """The nearest e4m3 value, ties to the even code (|x| <= 448)."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3.0)
    return torch.round(x / step) * step


def _exact_attention(case, st):
    new, length = _lengths(case)
    H, G, d, ps = case["heads"], case["group"], case["d"], case["ps"]
    if 4.0 * H * G * d * sum(a * b for a, b in zip(new, length)) > 4e12:
        return None
    out = torch.zeros(st["q"].shape, dtype=_F64, device="cuda")
    at = 0
    for s, (n, L) in enumerate(zip(new, length)):
        if n:
            pages = st["table"][s, :_up(L, ps)].long()
            pos = torch.arange(L, device="cuda") - (L - n)
            for h in range(H):
                k = _value64(st["k"][0, pages, h]) * torch.exp2(st["k_exp"][0, pages, h].to(_F64))[:, None, None, None, None]
                v = _value64(st["v"][0, pages, h]) * torch.exp2(st["v_exp"][0, pages, h].to(_F64))[:, None, None, None]
                k = k.permute(0, 1, 3, 2, 4).reshape(-1, d)[:L]
                v = v.permute(0, 1, 3, 2).reshape(-1, d)[:L].contiguous()
                q = st["q"][at:at + n, h * G:(h + 1) * G].to(_F64).reshape(n * G, d)
                a = (q @ k.t().contiguous()) / math.sqrt(d)
                a = a.view(n, G, L).masked_fill(pos[None, None, :] > torch.arange(n, device="cuda")[:, None, None], -math.inf)
                out[at:at + n, h * G:(h + 1) * G] = torch.matmul(torch.softmax(a, 2), v)
        at += n
    return out


def _exact_append(case, st):
    ps, H = case["ps"], case["heads"]
    new, length = _lengths(case)
    table = st["table"].tolist()
    out = {}
    for name, x in (("k", st["key"].to(_F64)), ("v", st["value"].to(_F64))):
        val, exps = _value64(st[name]), st[name + "_exp"].clone()
        flat = val[0].permute(0, 2, 4, 1, 3, 5) if name == "k" else val[0].permute(0, 2, 4, 1, 3)  # [N][unit][16][H]..
        at = 0
        top = x.abs().amax(2).cpu()
        olds, gains = exps[0].cpu(), exps[0].cpu().clone()
        jobs = []
        for n, L, row in zip(new, length, table):
            p = L - n
            while p < L:
                m = min(L - p, ps - p % ps)
                a = top[at + p - (L - n):at + p - (L - n) + m].amax(0).tolist()
                page, o = row[p // ps], p % ps
                for h in range(H):
                    e = _EMIN
                    while a[h] > 448.0 * 2.0 ** e and e < _EMAX:
                        e += 1
                    gains[page, h] = max(e, int(olds[page, h])) if o else e
                jobs.append((page, o, m, at + p - (L - n)))
                p += m
            at += n
        exps[0] = gains.cuda()
        shift = torch.exp2((olds - gains).to(_F64)).cuda()
        scale = torch.exp2(-gains.to(_F64)).cuda()
        page_of = torch.cat([torch.full((m,), pg) for pg, _, m, _ in jobs]).cuda()
        slot = torch.cat([torch.arange(o, o + m) for _, o, m, _ in jobs]).cuda()
        row = torch.cat([torch.arange(r, r + m) for _, _, m, r in jobs]).cuda()
        fill = torch.zeros((flat.shape[0],), dtype=torch.long)
        for pg, o, _, _ in jobs:
            fill[pg] = o
        fill = fill.cuda()
        tok = torch.arange(ps, device="cuda").view(ps // 16, 16)
        keep = (tok[None] < fill[:, None, None])[:, :, :, None, None]
        grown = shift[:, None, None, :, None]
        if name == "k":
            keep, grown = keep[..., None], grown[..., None]
        flat.copy_(torch.where(keep, _round64(flat * grown), flat))
        xs = _round64((x[row] * scale[page_of][:, :, None]).clamp(-448.0, 448.0))
        flat[page_of, slot // 16, slot % 16] = xs.view(-1, H, case["d"] // 16, 16) if name == "k" else xs
        out[name], out[name + "_exp"] = val, exps
    return out


def _moved64(st, pairs):
    src = torch.tensor([a for a, _ in pairs], dtype=torch.long, device="cuda")
    dst = torch.tensor([b for _, b in pairs], dtype=torch.long, device="cuda")
    out = {}
    for name in ("k", "v"):
        val = _value64(st[name])
        if pairs:
            val.index_copy_(1, dst, val.index_select(1, src))
        out[name], out[name + "_exp"] = val, st[name + "_exp"].index_copy(1, dst, st[name + "_exp"].index_select(1, src))
    return out


def _exact_fork(case, st):
    ps, grow = case["ps"], case["grow"]
    lengths, _, parent = _fork_rows(case)
    table, refs = st["table"].tolist(), st["refs"].tolist()
    free = [p for p, r in enumerate(refs) if r == 0]
    rows = [table[p][:_up(lengths[p], ps)] if p >= 0 else [] for p in parent]
    holders = {}
    for i, row in enumerate(rows):
        for page in row:
            holders.setdefault(page, []).append(i)
    pairs, take = [], 0
    for i, row in enumerate(rows):
        if parent[i] < 0:
            continue
        L = lengths[parent[i]]
        if L % ps and len(holders[row[-1]]) > 1:  # in order, each but the last to hold it takes a copy
            holders[row[-1]].remove(i)
            pairs.append((row[-1], free[take]))
            row[-1] = free[take]
            take += 1
        while len(row) < _up(L + grow, ps):
            row.append(free[take])
            take += 1
    now = [0] * len(refs)
    for row in rows:
        for page in row:
            now[page] += 1
    width = len(table[0])
    return {"table": _dev([r + [-1] * (width - len(r)) for r in rows]),
            "lengths": _dev([lengths[p] + grow if p >= 0 else 0 for p in parent]), "refs": _dev(now), **_moved64(st, pairs)}


def _exact_compact(case, st):
    refs, table = st["refs"].tolist(), st["table"].tolist()
    held = [p for p, r in enumerate(refs) if r > 0]
    used = len(held)
    to, hole = {p: p for p in held}, 0
    pairs = []
    for p in reversed(held):
        while hole < used and refs[hole] > 0:
            hole += 1
        if hole >= used or p < used:
            break
        to[p] = hole
        pairs.append((p, hole))
        hole += 1
    now = [0] * len(refs)
    for p in held:
        now[to[p]] = refs[p]
    return {"table": _dev([[to[p] if p >= 0 else -1 for p in row] for row in table]), "refs": _dev(now),
            "used": torch.tensor(used, dtype=torch.int32), **_moved64(st, pairs)}


def _exact_beam(case, st):
    B, W, V = case["B"], case["W"], case["V"]
    n = min(W, V)
    score = torch.full((B, W), -math.inf, dtype=_F64, device="cuda")
    for b in range(B):
        x = st["logits"][b].to(_F64)
        logp = x - torch.logsumexp(x, 1, keepdim=True)
        total = torch.topk(torch.nan_to_num(logp, nan=-math.inf), n, dim=1).values + st["scores"][b].to(_F64)[:, None]
        for w in range(W):
            if st["done"][b, w]:
                total[w] = -math.inf
                total[w, 0] = st["scores"][b, w].to(_F64)
        score[b] = torch.topk(total.reshape(-1), W).values
    return {"parent": None, "token": None, "score": score, "done": None, "history": None}


def exact(case, seed):
    st = prepare(case, seed)
    return {"attention": _exact_attention, "append": _exact_append, "fork": _exact_fork, "compact": _exact_compact,
            "beam": _exact_beam}[case["op"]](case, st)
