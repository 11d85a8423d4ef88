"""What the position and shared-prefix operators are timed on: rotary positions of queries and keys, appending to the
paged 8-bit cache with the keys rotated on the way, finding what rows of the cache share, and attention that goes over
a shared prefix once for all the rows that share it.

Rotation.  A head's first 2 P elements are P pairs, (x_i, x_{i + P}) or, interleaved, (x_{2i}, x_{2i+1}).  At position t
a pair (u, v) becomes m (u cos a - v sin a, u sin a + v cos a) with a = t f_i (64 bits); inverse: a = -t f_i.

The cache is the pool that perf/operators.py describes: pages of `ps` tokens, e4m3 codes of keys
[layers][pages][heads][ps / 16][d / 16][16 tokens][16 of d] and values [..][ps / 16][d][16 tokens], one int8 exponent for a
page and head.  New tokens come ragged: sequence s has tokens starts[s] .. starts[s + 1] - 1, the last of its lengths[s].
An appended page's exponent of keys is that of the larger of its largest magnitude in the part of the head that is not
rotated, and sqrt(2) m (in 32 bits) times that of the part that is, before it is rotated: no angle passes it.

Groups.  Rows groups[g] .. groups[g + 1] - 1 of the table may share leading pages.  Of those that hold `least` tokens (at
least one) before their new ones, the shared tokens are the pages that are the same in all, up to the fewest tokens that one
of them holds before its new ones, in whole multiples of max(64, ps); none where fewer than two take part, or where it is
less than `least`.  `tokens` [S]: what a sequence shares (0: it takes no part); `rows` [G][4]: a group's first new token, its
new tokens, its first row that takes part (-1: none) and its shared tokens.

Inputs are synthetic: normal keys, values and queries, pages in random order.  Lengths follow fixed patterns of the case,
so that its work is known without its data.
"""
import math

import torch

own = False

_F64 = torch.float64
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_F8 = torch.float8_e4m3fn
_EMIN, _EMAX = -40, 40  # range of the cache's exponents


def _rotary(name, T, H, of, D, dim, dtype, interleaved, far, scaled, inverse=False):
    """T tokens of H heads of D that lie among `of` heads; `dim` elements of a head are rotated; positions below `far`."""
    return {"name": name, "op": "rotary", "T": T, "H": H, "of": of, "D": D, "dim": dim, "dtype": dtype,
            "interleaved": interleaved, "far": far, "scaled": scaled, "inverse": inverse}


def _append(name, S, n, length, heads, group, d, dim, ps, dtype, interleaved, scaled, ragged=False, tree=False):
    """Up to `n` new tokens for each of S sequences, which hold up to `length` with them; `group` query heads a key
    head go along; `tree`: positions are given (drafts that branch), not counted."""
    return {"name": name, "op": "append", "S": S, "n": n, "length": length, "heads": heads, "group": group, "d": d,
            "dim": dim, "ps": ps, "dtype": dtype, "interleaved": interleaved, "scaled": scaled, "ragged": ragged,
            "tree": tree}


def _shared(op, name, G, W, n, prefix, own_tokens, heads, group, d, ps, dtype, ragged=False):
    """G groups of up to W sequences over a common prefix of up to `prefix` tokens, each with up to `own_tokens` more,
    the last up to `n` of them new."""
    return {"name": name, "op": op, "G": G, "W": W, "n": n, "prefix": prefix, "own": own_tokens, "heads": heads,
            "group": group, "d": d, "ps": ps, "dtype": dtype, "ragged": ragged}


def listed():
    return [
        # A decode step's queries and keys (32 and 8 heads inside a fused product of 48), in one layer: latency.
        _rotary("rotary_step_64x40", 64, 40, 48, 128, 128, "bf16", False, 100000, False),
        # Prompts of a batch, pairs side by side, frequencies for a long context.
        _rotary("rotary_prompt_8192x40", 8192, 40, 40, 128, 128, "f16", True, 1000000, True),
        # The gradient of it in 32 bits, three quarters of an uneven number of heads rotated, an odd number of tokens.
        _rotary("rotary_gradient_4001x33", 4001, 33, 33, 96, 72, "f32", False, 20000, False, True),
        # A decode step of a batch: keys and values into the cache, queries rotated.
        _append("append_256x1", 256, 1, 2000, 8, 4, 128, 128, 16, "bf16", False, False),
        # Drafts to verify, branching: up to 5 tokens a sequence at given positions.
        _append("append_drafts_64x5", 64, 5, 1500, 8, 4, 128, 128, 64, "bf16", False, True, True, True),
        # Prompts, odd lengths, half of the head rotated, pairs side by side.
        _append("append_prompt_16x2048", 16, 2048, 2500, 8, 4, 128, 64, 64, "f16", True, False, True),
        # What the beams of a small batch share.
        _shared("prefix", "prefix_4x4", 4, 4, 1, 300, 40, 1, 1, 64, 16, "bf16"),
        # What 1024 beams with long prompts share, in small pages.
        _shared("prefix", "prefix_128x8", 128, 8, 1, 8192, 100, 1, 1, 64, 16, "bf16", True),
        # Four beams of one prompt: latency.
        _shared("attention", "shared_1x4x1000", 1, 4, 1, 1000, 24, 8, 4, 128, 16, "bf16"),
        # Eight beams each of 16 prompts, lengths from a quarter of 6000 up.
        _shared("attention", "shared_16x8x6000", 16, 8, 1, 6000, 150, 8, 4, 128, 64, "bf16", True),
        # Four drafts of up to 5 tokens for each of 32 sequences.
        _shared("attention", "shared_drafts_32x4x5", 32, 4, 5, 4000, 40, 8, 4, 128, 16, "f16", True),
        # A batch under one long instruction: 256 sequences, up to 1000 tokens of their own.
        _shared("attention", "shared_batch_256x8192", 1, 256, 1, 8192, 1000, 8, 8, 128, 64, "bf16", True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "rotary", "append", "append", "append", "prefix", "beams", "drafts", "batch", "long"])
    interleaved, scaled = rng.random() < 0.5, rng.random() < 0.5
    dtype = rng.choice(["bf16", "f16"])
    heads, group = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 4, 5, 8])
    d, ps = rng.choice([64, 96, 128, 128, 128, 256]), rng.choice([16, 16, 32, 64, 128])
    ragged = rng.random() < 0.5
    if op == "rotary":
        D = rng.choice([32, 40, 64, 80, 96, 127, 128, 128, 192, 256])
        dim = rng.choice([D - D % 2, D // 4 * 2, 2 * rng.randint(1, D // 2)])
        H = rng.randint(1, 48)
        T = _log_int(rng, 1, min(20000, 40000000 // (H * D)))
        c = _rotary("", T, H, H + rng.choice([0, 0, 1, 8]), D, dim, rng.choice(["bf16", "f16", "f32"]), interleaved,
                    _log_int(rng, 100, 10000000), scaled, rng.random() < 0.3)
    elif op == "append":
        n = rng.choice([1, 1, rng.randint(2, 9), _log_int(rng, 10, 3000)])
        length = n + _log_int(rng, 1, 2000)
        S = _log_int(rng, 1, max(1, min(512, 24000000 // (n * heads * (2 + group) * d) * 2)))
        c = _append("", S, n, length, heads, group, d, rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)]), ps, dtype,
                    interleaved, scaled, ragged, rng.random() < 0.3)
        while _pool_bytes(c) > 1.5e9:
            c["S"] = max(1, c["S"] // 2)
    elif op == "prefix":
        c = _shared("prefix", "", _log_int(rng, 1, 128), rng.randint(1, 16), rng.randint(1, 6), _log_int(rng, 20, 8000),
                    rng.randint(8, 200), 1, 1, 64, ps, dtype, ragged)
        while _pool_bytes(c) > 1e9:
            c["G"] = max(1, c["G"] // 2)
    else:
        if op == "beams":
            G, W, n, prefix, more = _log_int(rng, 1, 32), rng.randint(2, 16), 1, _log_int(rng, 64, 8000), rng.randint(1, 300)
        elif op == "drafts":
            n = rng.randint(2, 8)
            G, W, prefix, more = _log_int(rng, 1, 32), rng.randint(2, 8), _log_int(rng, 64, 8000), rng.randint(n, 60)
        elif op == "batch":
            G, W, n, prefix, more = rng.randint(1, 3), _log_int(rng, 16, 256), 1, _log_int(rng, 200, 8000), _log_int(rng, 8, 1000)
        else:
            G, W, n, prefix, more = 1, rng.randint(2, 8), rng.randint(1, 4), _log_int(rng, 8000, 100000), rng.randint(8, 100)
        c = _shared("attention", "", G, W, n, prefix, more, heads, group, d, ps, dtype, ragged)
        top = work(listed()[-1])
        while True:
            w, rows = work(c), c["heads"] * c["group"] * c["n"] * c["G"] * c["W"]
            if (w["flops"] <= top["flops"] and w["bytes"] <= top["bytes"] and _pool_bytes(c) < 1.5e9 and
                    rows * (c["prefix"] + c["own"]) < 150000000):
                break
            if c["W"] > 2:
                c["W"] //= 2
            elif c["G"] > 1:
                c["G"] //= 2
            else:
                c["prefix"] //= 2
    del c["name"]
    return c


# --------------------------------------------------------------------------- patterns of a case
def _up(a, b):
    return -(-a // b)


def _lengths(case):
    """Append: (new tokens, length) of every sequence.  Ragged: 0 .. n new ones, lengths from a quarter of the most."""
    S, n, L = case["S"], case["n"], case["length"]
    if not case["ragged"]:
        return [n] * S, [L] * S
    new = [(n - (s * 37) % (n + 1)) for s in range(S)]
    share = [1.0 - 0.75 * ((s * 0.6180339887) % 1.0) for s in range(S)]
    return new, [max(a, int(L * f)) for a, f in zip(new, share)]


def _group_rows(case):
    """Groups: for each its prefix, and for each of its sequences (new tokens, tokens of its own, new ones among them).
    Ragged: prefixes from a quarter of the most, groups of down to half of W rows, 0 .. n new tokens, and in every third
    group one row that holds nothing (a beam that was given up)."""
    out = []
    for g in range(case["G"]):
        f = (g * 0.6180339887) % 1.0
        prefix = max(1, int(case["prefix"] * (1.0 - 0.75 * f))) if case["ragged"] else case["prefix"]
        W = case["W"] - (g * 5) % (case["W"] // 2 + 1) if case["ragged"] else case["W"]
        rows = []
        for w in range(W):
            n, more = case["n"], case["own"]
            if case["ragged"]:
                n -= (w * 3 + g) % (n + 1) if n > 1 else 0
                more = max(n, int(more * (1.0 - 0.9 * ((w * 0.7548776662 + f) % 1.0))))
            rows.append((n, more))
        gone = case["ragged"] and g % 3 == 2 and W > 2
        out.append((prefix, rows, W // 2 if gone else -1))
    return out


def _least(case):
    return 64 if case["ragged"] else 0


def _group_tokens(case):
    """For each group (first row, rows, first new token, new tokens, first row that takes part, shared tokens), and for
    each sequence (group, new tokens, length, shared tokens, takes part in)."""
    unit, groups, seqs, row, token = max(64, case["ps"]), [], [], 0, 0
    for prefix, rows, gone in _group_rows(case):
        held = prefix // case["ps"] * case["ps"]  # pages that all have: what comes after them is each one's own
        length = [0 if w == gone else prefix + more for w, (_, more) in enumerate(rows)]
        before = [L - n for L, (n, _) in zip(length, rows)]
        part = [b >= max(1, _least(case)) for b in before]
        common = held if sum(part) > 1 else 0
        common = min([common] + [b for b, p in zip(before, part) if p]) // unit * unit
        if common < _least(case):
            common = 0
        first = row + part.index(True) if any(part) else -1
        n_all = sum(n for n, _ in rows)
        groups.append((row, len(rows), token, n_all, first, common, held))
        seqs += [(len(groups) - 1, n, L, common if p else 0) for (n, _), L, p in zip(rows, length, part)]
        row, token = row + len(rows), token + n_all
    return groups, seqs


def _pages(case):
    if case["op"] == "append":
        per = [_up(L, case["ps"]) for L in _lengths(case)[1]]
        return sum(per) + sum(per) // 8 + 2
    groups, seqs = _group_tokens(case)
    ps = case["ps"]
    spare = max(g[6] for g in groups) // ps + 2  # copies of shared pages that some rows have (prefix)
    return sum(g[6] // ps for g in groups) + sum(max(0, _up(L, ps) - groups[g][6] // ps) for g, _, L, _ in seqs) + spare


def _pool_bytes(case):
    return _pages(case) * 2 * case["ps"] * case["heads"] * case["d"]


def _frequencies(case, dim):
    """dim / 2 frequencies; scaled, for contexts 8 times as long: those that turn less than once over 4096 positions are
    divided by 8, those that turn over 32 times stay, linearly between by the turns; and the magnitude of the rotation."""
    i = torch.arange(dim // 2, dtype=_F64)
    f = torch.pow(torch.tensor(10000.0, dtype=_F64), -2.0 * i / dim)
    if not case["scaled"]:
        return f, 1.0
    keep = ((4096.0 * f / (2.0 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
    return f * (keep + (1.0 - keep) / 8.0), 0.1 * math.log(8.0) + 1.0


# ------------------------------------------------------------------------------------- inputs
def _pool(case, g):
    """A filled pool: codes of normal values, exponents of a few octaves."""
    N, H, d, ps = _pages(case), case["heads"], case["d"], case["ps"]

    def codes(*shape):
        out = torch.empty(shape, dtype=torch.uint8, device="cuda")
        flat = out.view(-1)
        for at in range(0, flat.numel(), 1 << 27):
            part = flat[at:at + (1 << 27)]
            part.copy_((torch.randn(part.shape, generator=g, device="cuda") * 70.0).clamp_(-448.0, 448.0).to(_F8).view(torch.uint8))
        return out

    def exps():
        return torch.randint(-7, -4, (1, N, H), generator=g, device="cuda", dtype=torch.int8)

    return {"k": codes(1, N, H, ps // 16, d // 16, 16, 16), "v": codes(1, N, H, ps // 16, d, 16), "k_exp": exps(),
            "v_exp": exps()}


def _dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def _starts(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return _dev(out)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": case}
    if case["op"] == "rotary":
        kind = _TYPES[case["dtype"]]
        x = torch.randn((case["T"], case["of"], case["D"]), generator=g, device="cuda").to(kind)
        f, st["magnitude"] = _frequencies(case, case["dim"])
        st.update(x=x[:, case["of"] - case["H"]:], frequencies=f.cuda(),
                  positions=torch.randint(0, case["far"], (case["T"],), generator=g, device="cuda", dtype=torch.int32))
        return st
    st.update(_pool(case, g))
    ids = torch.randperm(_pages(case), generator=g, device="cuda").int()
    if case["op"] == "append":
        new, length = _lengths(case)
        T, H, d, ps = sum(new), case["heads"], case["d"], case["ps"]
        per = [_up(x, ps) for x in length]
        width = max(per) + 2
        n = _dev(per)
        at = torch.arange(width, device="cuda", dtype=torch.int32)[None]
        where = (torch.cumsum(n, 0)[:, None] - n[:, None] + at).clamp(max=ids.numel() - 1).long()
        st["table"] = torch.where(at < n[:, None], ids[where], torch.full_like(where, -1).int()).contiguous()
        st.update(lengths=_dev(length), starts=_starts(new))
        kind = _TYPES[case["dtype"]]
        # heads of unlike magnitude, now and then a token that stands out; queries beside them, as a fused product leaves them
        size = torch.exp2(torch.randint(-3, 4, (1, H, 1), generator=g, device="cuda").float())
        qkv = torch.randn((T, (case["group"] + 2) * H, d), generator=g, device="cuda")
        qkv[:, case["group"] * H:] *= torch.cat((size, size), 1)
        qkv[:, case["group"] * H:] *= 1.0 + 30.0 * (torch.rand((T, 1, 1), generator=g, device="cuda") < 0.01)
        qkv = qkv.to(kind)
        st["q"], st["key"], st["value"] = qkv.split((case["group"] * H, H, H), 1)
        f, st["magnitude"] = _frequencies(case, case["dim"])
        st["frequencies"] = f.cuda()
        st["positions"] = None
        if case["tree"]:
            s, i, pos = _rows(st, T)
            st["positions"] = (pos - (i * 3 + s) % 4 * (i > 0)).clamp(min=0).int()
        return st
    groups, seqs = _group_tokens(case)
    ps = case["ps"]
    width = max([_up(L, ps) for _, _, L, _ in seqs] + [1]) + 2
    rows, at, base = [], 0, 0
    starts_of = []
    for _, _, _, _, _, _, held in groups:
        starts_of.append(base)
        base += held // ps
    for gi, _, L, _ in seqs:
        common = min(groups[gi][6] // ps, _up(L, ps))
        mine = _up(L, ps) - common
        rows.append([starts_of[gi], common, base + at, mine])
        at += mine
    r = _dev(rows).long()
    j = torch.arange(width, device="cuda")[None]
    where = torch.where(j < r[:, 1:2], r[:, 0:1] + j, r[:, 2:3] + j - r[:, 1:2])
    st["table"] = torch.where(j < (r[:, 1] + r[:, 3])[:, None], ids[where.clamp(max=ids.numel() - 1)],
                              torch.full_like(where, -1).int()).contiguous()
    st.update(lengths=_dev([x[2] for x in seqs]), starts=_starts([x[1] for x in seqs]))
    T = sum(x[1] for x in seqs)
    st["T"] = T
    if case["op"] == "prefix":
        st["groups"] = _dev([x[0] for x in groups] + [len(seqs)])
        # one row of a group went its own way earlier: it has copies of the last of the prefix's pages, up to a quarter
        u = torch.rand((2, len(groups)), generator=g, device="cuda")
        count = _dev([x[1] for x in groups])
        odd = st["groups"][:-1] + (u[0] * count).int().clamp(max=count - 1)
        held = _dev([x[6] // ps for x in groups])
        from_page = held - (u[1] * (held // 4 + 1)).int()
        group = torch.repeat_interleave(torch.arange(len(groups), device="cuda"), count)
        mine = (torch.arange(len(seqs), device="cuda", dtype=torch.int32) == odd[group])[:, None] & (st["lengths"] > 0)[:, None]
        copied = mine & (j >= from_page[group][:, None]) & (j < held[group][:, None])
        st["table"] = torch.where(copied, ids[-width:][None], st["table"])
    else:
        st["tokens"] = _dev([x[3] for x in seqs])
        st["rows"] = _dev([[a, b, row, P] for _, _, a, b, row, P, _ in groups])
        st["q"] = torch.randn((T, case["heads"] * case["group"], case["d"]), generator=g, device="cuda").to(_TYPES[case["dtype"]])
        # what a program knows of its lengths on the host
        st["most"] = {"max_new": case["n"], "max_group": max(x[3] for x in groups), "max_shared": max(x[5] for x in groups),
                      "max_own": max([L - P for _, _, L, P in seqs])}
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
        if op in ("rotary", "append"):
            rope = mdss.Rotary(st["frequencies"], interleaved=c["interleaved"], magnitude=st["magnitude"])
            if op == "rotary":
                return mdss.rotary(st["x"], rope, st["positions"], inverse=c["inverse"])
        cache = mdss.PagedCache(st["k"], st["v"], st["k_exp"], st["v_exp"])
        if op == "append":
            q = mdss.cache_append_rotary(cache, 0, st["key"], st["value"], st["starts"], st["table"], st["lengths"], rope,
                                         positions=st["positions"], q=st["q"])
            return {"q": q, **_pools(st)}
        if op == "prefix":
            tokens, rows = mdss.cache_shared(cache, st["T"], st["starts"], st["table"], st["lengths"], st["groups"],
                                             least=_least(c))
            return {"tokens": tokens, "rows": rows}
        return mdss.cache_attention_shared(st["q"], cache, 0, st["starts"], st["table"], st["lengths"],
                                           (st["tokens"], st["rows"]), **st["most"])
    return {"rotary": _plain_rotary, "append": _plain_append, "prefix": _plain_prefix, "attention": _plain_attention}[op](st)


# ------------------------------------------------------------------------------ the plain forms
def _rows(st, T):
    """For every new token its sequence, its place among the sequence's new ones, and its position."""
    starts, lengths = st["starts"].long(), st["lengths"].long()
    n = starts[1:] - starts[:-1]
    t = torch.arange(T, device="cuda")
    s = torch.searchsorted(starts, t, right=True) - 1
    i = t - starts[s]
    return s, i, lengths[s] - n[s] + i


def _rotate(x, frequencies, magnitude, positions, interleaved, inverse):
    """x [T][H][D] in 32 bits, its pairs turned."""
    P = frequencies.numel()
    a = positions.to(_F64)[:, None] * frequencies
    c = (torch.cos(a) * magnitude).float()[:, None]
    s = (torch.sin(a) * (-magnitude if inverse else magnitude)).float()[:, None]
    if interleaved:
        u, v = x[:, :, 0:2 * P:2], x[:, :, 1:2 * P:2]
        turned = torch.stack((u * c - v * s, u * s + v * c), 3).flatten(2)
    else:
        u, v = x[:, :, :P], x[:, :, P:2 * P]
        turned = torch.cat((u * c - v * s, u * s + v * c), 2)
    return torch.cat((turned, x[:, :, 2 * P:]), 2)


def _plain_rotary(st):
    c = st["case"]
    return _rotate(st["x"].float(), st["frequencies"], st["magnitude"], st["positions"], c["interleaved"],
                   c["inverse"]).to(st["x"].dtype)


def _exponent(amax):
    """The least e with amax <= 448 * 2^e, within the exponents' range."""
    m, x = torch.frexp(amax)
    e = torch.where(m <= 0.875, x - 9, x - 8)
    return torch.where(amax > 0, e, torch.full_like(e, _EMIN)).clamp(_EMIN, _EMAX)


def _plain_append(st):
    c = st["case"]
    ps, H, N, dim = c["ps"], c["heads"], st["k"].shape[1], c["dim"]
    s, i, pos = _rows(st, st["key"].shape[0])
    page, slot = st["table"].long()[s, pos // ps], pos % ps
    at_pos = pos if st["positions"] is None else st["positions"]
    first = torch.full((N,), ps, device="cuda").scatter_reduce_(0, page, slot, "amin")
    touched = torch.unique(page)
    unit, at = slot // 16, slot % 16
    key, value = st["key"].float(), st["value"].float()
    bound = torch.full((), math.sqrt(2.0) * torch.tensor(st["magnitude"], dtype=torch.float32).item(), device="cuda")
    limit = key[:, :, :dim].abs().amax(2) * bound
    if dim < c["d"]:
        limit = torch.maximum(limit, key[:, :, dim:].abs().amax(2))
    turn = (st["frequencies"], st["magnitude"], at_pos, c["interleaved"], False)
    for name, x, top in (("k", _rotate(key, *turn), limit), ("v", value, value.abs().amax(2))):
        codes, exps = st[name][0], st[name + "_exp"][0]
        amax = torch.zeros((N, H), device="cuda").scatter_reduce_(0, page[:, None].expand(-1, H), top, "amax")
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
    return {"q": _rotate(st["q"].float(), *turn).to(st["q"].dtype), **_pools(st)}


def _plain_prefix(st):
    c = st["case"]
    ps, unit, least = c["ps"], max(64, c["ps"]), _least(c)
    table, lengths, starts, groups = st["table"].long(), st["lengths"].long(), st["starts"].long(), st["groups"].long()
    S, width = table.shape
    G = groups.numel() - 1
    rows = torch.arange(S, device="cuda")
    g = torch.searchsorted(groups, rows, right=True) - 1
    before = lengths.clamp(max=width * ps) - (starts[1:] - starts[:-1])
    part = before >= max(1, least)
    none = torch.full((G,), S, device="cuda")
    first = none.scatter_reduce(0, g[part], rows[part], "amin")
    lead = first[g].clamp(max=S - 1)
    same = (table == table[lead]) & (table >= 0) & (table < st["k"].shape[1])
    pages = torch.cumprod(same.long(), 1).sum(1)
    common = torch.minimum(pages * ps, before)
    shared = torch.full((G,), width * ps, device="cuda").scatter_reduce(0, g[part], common[part], "amin") // unit * unit
    count = torch.zeros((G,), dtype=torch.long, device="cuda").scatter_add_(0, g, part.long())
    shared = torch.where((count > 1) & (shared >= least), shared, torch.zeros_like(shared))
    a, b = starts[groups[:-1]], starts[groups[1:]]
    lead = torch.where(first < S, first, torch.full_like(first, -1))
    return {"tokens": torch.where(part, shared[g], torch.zeros_like(before)).int(),
            "rows": torch.stack((a, b - a, lead, shared), 1).int()}


def _read(st, pages):
    """Keys and values [..][heads][tokens][d] in 32 bits of lists of pages [..][n]."""
    H, d = st["case"]["heads"], st["case"]["d"]
    lead = pages.shape[:-1]
    flat = pages.reshape(-1, pages.shape[-1])
    ks = torch.exp2(st["k_exp"][0].float())[flat][..., None, None, None, None]
    vs = torch.exp2(st["v_exp"][0].float())[flat][..., None, None, None]
    k = (_f8(st["k"][0][flat]).float() * ks).permute(0, 2, 1, 3, 5, 4, 6).reshape(*lead, H, -1, d)
    v = (_f8(st["v"][0][flat]).float() * vs).permute(0, 2, 1, 3, 5, 4).reshape(*lead, H, -1, d)
    return k, v


def _products(q, k, v, hidden, d):
    """(maximum, sum, weighted values) of rows q over keys k and values v, `hidden` ones left out."""
    a = torch.matmul(q, k.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(d))
    a.masked_fill_(hidden, -math.inf)
    m = a.amax(-1, keepdim=True).clamp(min=-3e38)
    e = a.sub_(m).exp_()
    return m, e.sum(-1, keepdim=True), torch.matmul(e, v)


def _plain_attention(st):
    c = st["case"]
    q, table, lengths, starts = st["q"], st["table"].long(), st["lengths"].long(), st["starts"].long()
    tokens, rows = st["tokens"].long(), st["rows"].long()
    T, S, G, H, K, d, ps, n = q.shape[0], table.shape[0], rows.shape[0], c["heads"], c["group"], c["d"], c["ps"], c["n"]
    most = st["most"]
    s, i, pos = _rows(st, T)
    g = torch.searchsorted(rows[:, 0].contiguous(), torch.arange(T, device="cuda"), right=True) - 1
    at = torch.arange(T, device="cuda") - rows[g, 0]
    # the shared tokens: the new tokens of a group are the rows of one product
    N, P = most["max_group"], most["max_shared"]
    qf = q.float().view(T, H, K, d)
    none = (torch.full((T, H, K, 1), -3e38, device="cuda"), torch.zeros((T, H, K, 1), device="cuda"), torch.zeros((T, H, K, d), device="cuda"))
    if P > 0:
        qs = torch.zeros((G, N, H, K, d), device="cuda")
        qs[g, at] = qf
        k, v = _read(st, table[rows[:, 2].clamp(min=0)][:, :P // ps].clamp(min=0))
        hidden = (torch.arange(P, device="cuda") >= rows[:, 3:4])[:, None, None, :]
        m, z, o = _products(qs.permute(0, 2, 1, 3, 4).reshape(G, H, N * K, d), k, v, hidden, d)
        both = [x.view(G, H, N, K, -1).permute(0, 2, 1, 3, 4)[g, at] for x in (m, z, o)]
        takes = (tokens[s] > 0)[:, None, None, None]
        m0, z0, o0 = (torch.where(takes, x, y) for x, y in zip(both, none))
    else:
        m0, z0, o0 = none
    # the tokens of a sequence's own
    count = _up(most["max_own"], ps)
    j = (tokens // ps)[:, None] + torch.arange(count, device="cuda")
    k, v = _read(st, table.gather(1, j.clamp(max=table.shape[1] - 1)).clamp(min=0))
    place = tokens[:, None] + torch.arange(count * ps, device="cuda")
    v = v * (place < lengths[:, None])[:, None, :, None]
    qs = torch.zeros((S, n, H, K, d), device="cuda")
    qs[s, i] = qf
    last = torch.full((S, n), -1, device="cuda")
    last[s, i] = pos
    hidden = (place[:, None, :] > last[:, :, None])[:, None, :, None, :].expand(S, 1, n, K, place.shape[1]).reshape(S, 1, n * K, -1)
    m, z, o = _products(qs.permute(0, 2, 1, 3, 4).reshape(S, H, n * K, d), k, v, hidden, d)
    m1, z1, o1 = (x.view(S, H, n, K, -1).permute(0, 2, 1, 3, 4)[s, i] for x in (m, z, o))
    top = torch.maximum(m0, m1)
    w0, w1 = torch.exp(m0 - top), torch.exp(m1 - top)
    z = z0 * w0 + z1 * w1
    out = (o0 * w0 + o1 * w1) / torch.where(z > 0, z, torch.ones_like(z))
    return out.reshape(T, H * K, d).to(q.dtype)


def work(case):
    op = case["op"]
    if op == "rotary":
        size = case["T"] * case["H"] * case["D"]
        return {"bytes": 2 * size * (4 if case["dtype"] == "f32" else 2) + 4 * case["T"], "flops": 3 * case["T"] * case["H"] * case["dim"]}
    if op == "append":
        T, H, d = sum(_lengths(case)[0]), case["heads"], case["d"]
        return {"bytes": T * H * d * (2 * 3 + 4 * case["group"]), "flops": 3 * T * H * (1 + case["group"]) * case["dim"]}
    groups, seqs = _group_tokens(case)
    if op == "prefix":
        return {"bytes": sum(3 * (P // case["ps"]) for _, _, _, P in seqs) + 12 * len(seqs) + 24 * len(groups), "flops": 0}
    H, hq, d = case["heads"], case["heads"] * case["group"], case["d"]
    T = sum(n for _, n, _, _ in seqs)
    cached = sum(g[5] for g in groups) + sum(L - P for _, n, L, P in seqs if n)
    seen = sum(n * max(0, L - n) + (n * (n + 1) // 2 if L else 0) for _, n, L, _ in seqs)
    return {"bytes": cached * H * d * 2 + 4 * T * hq * d, "flops": 4 * hq * d * seen}


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


def _turned64(x, case, st, positions, inverse):
    """The pairs as complex numbers times e^(i a)."""
    x = x.to(_F64)
    P = case["dim"] // 2
    head = x[..., :2 * P]
    z = torch.view_as_complex((head.unflatten(-1, (P, 2)) if case["interleaved"] else
                               torch.stack((head[..., :P], head[..., P:]), -1)).contiguous())
    a = torch.outer(positions.to(_F64), st["frequencies"])
    z = torch.view_as_real(z * torch.polar(torch.full_like(a, st["magnitude"]), -a if inverse else a)[:, None])
    head = z.flatten(-2) if case["interleaved"] else torch.cat((z[..., 0], z[..., 1]), -1)
    return torch.cat((head, x[..., 2 * P:]), -1)


def _exact_append(case, st):
    ps, H = case["ps"], case["heads"]
    new, length = _lengths(case)
    table = st["table"].tolist()
    spots = [(row[p // ps], p % ps, p, r) for row, n, L, r in
             zip(table, new, length, st["starts"].tolist()) for r, p in zip(range(r, r + n), range(L - n, L))]
    page, slot, pos = (torch.tensor([x[i] for x in spots], dtype=torch.long, device="cuda") for i in range(3))
    at = pos if st["positions"] is None else st["positions"]
    out = {"q": _turned64(st["q"], case, st, at, False)}
    begun = {}
    for pg, o, _, _ in spots:
        begun.setdefault(pg, o)
    ids = torch.tensor(sorted(begun), dtype=torch.long, device="cuda")
    fill = torch.zeros((st["k"].shape[1],), dtype=torch.long, device="cuda")
    fill[ids] = torch.tensor([begun[p] for p in sorted(begun)], device="cuda")
    plain, turned = st["key"].to(_F64).abs(), torch.zeros((len(spots), H), dtype=_F64, device="cuda")
    dim = case["dim"]
    if dim < case["d"]:
        turned = plain[:, :, dim:].amax(2)
    turned = torch.maximum(turned, plain[:, :, :dim].amax(2) * math.sqrt(2.0) * st["magnitude"])
    steps = 448.0 * torch.exp2(torch.arange(_EMIN, _EMAX, dtype=_F64, device="cuda"))
    for name, x, top in (("k", _turned64(st["key"], case, st, at, False), turned),
                         ("v", st["value"].to(_F64), st["value"].to(_F64).abs().amax(2))):
        val, exps = _value64(st[name]), st[name + "_exp"].clone()
        most = torch.zeros((st["k"].shape[1], H), dtype=_F64, device="cuda").index_reduce_(0, page, top, "amax")
        e = _EMIN + (most[..., None] > steps).sum(-1)
        old = exps[0].long()
        e = torch.where(fill[:, None] > 0, torch.maximum(e, old), e)
        gains = old.clone()
        gains[ids] = e[ids]
        exps[0] = gains.to(torch.int8)
        shift, scale = torch.exp2((old - gains).to(_F64)), torch.exp2(-gains.to(_F64))
        flat = val[0].permute(0, 2, 4, 1, 3, 5) if name == "k" else val[0].permute(0, 2, 4, 1, 3)  # [N][unit][16][H]..
        keep = (torch.arange(ps, device="cuda").view(ps // 16, 16)[None] < fill[:, None, None])[:, :, :, None, None]
        grown = shift[:, None, None, :, None]
        if name == "k":
            keep, grown = keep[..., None], grown[..., None]
        flat.copy_(torch.where(keep, _round64(flat * grown), flat))
        xs = _round64((x * scale[page][:, :, None]).clamp(-448.0, 448.0))
        flat[page, slot // 16, slot % 16] = xs.view(-1, H, case["d"] // 16, 16) if name == "k" else xs
        out[name], out[name + "_exp"] = val, exps
    return out


def _exact_prefix(case, st):
    """From the tables, row by row."""
    ps, unit, least = case["ps"], max(64, case["ps"]), _least(case)
    table, lengths, starts, groups = (st[x].tolist() for x in ("table", "lengths", "starts", "groups"))
    tokens, rows = [], []
    for a, b in zip(groups[:-1], groups[1:]):
        held = [lengths[s] - (starts[s + 1] - starts[s]) for s in range(a, b)]
        part = [s for s, x in zip(range(a, b), held) if x >= max(1, least)]
        n = 0
        if len(part) > 1:
            while n < len(table[a]) and len({table[s][n] for s in part}) == 1 and table[part[0]][n] >= 0:
                n += 1
            n = min([n * ps] + [held[s - a] for s in part]) // unit * unit
        n = n if n >= least else 0
        tokens += [n if s in part else 0 for s in range(a, b)]
        rows.append([starts[a], starts[b] - starts[a], part[0] if part else -1, n])
    return {"tokens": _dev(tokens), "rows": _dev(rows)}


def _exact_attention(case, st):
    """Sequence by sequence, over its own table from its first token on."""
    H, K, d, ps = case["heads"], case["group"], case["d"], case["ps"]
    starts, lengths = st["starts"].tolist(), st["lengths"].tolist()
    out = torch.zeros(st["q"].shape, dtype=_F64, device="cuda")
    for s, L in enumerate(lengths):
        a, n = starts[s], starts[s + 1] - starts[s]
        if n == 0 or L == 0:
            continue
        pages = st["table"][s, :_up(L, ps)].long()
        k = _value64(st["k"][0, pages]) * torch.exp2(st["k_exp"][0, pages].to(_F64))[..., None, None, None, None]
        v = _value64(st["v"][0, pages]) * torch.exp2(st["v_exp"][0, pages].to(_F64))[..., None, None, None]
        k = k.permute(1, 0, 2, 4, 3, 5).reshape(H, -1, d)[:, :L]
        v = v.permute(1, 0, 2, 4, 3).reshape(H, -1, d)[:, :L].contiguous()
        q = st["q"][a:a + n].to(_F64).view(n, H, K, d).permute(1, 0, 2, 3).reshape(H, n * K, d)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        late = torch.arange(L, device="cuda")[None, :] > torch.arange(L - n, L, device="cuda")[:, None]
        x = torch.softmax(x.view(H, n, K, L).masked_fill(late[None, :, None, :], -math.inf), 3).view(H, n * K, L)
        out[a:a + n] = torch.matmul(x, v).view(H, n, K, d).permute(1, 0, 2, 3).reshape(n, H * K, d)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rotary":
        return _turned64(st["x"], case, st, st["positions"], case["inverse"])
    return {"append": _exact_append, "prefix": _exact_prefix, "attention": _exact_attention}[case["op"]](case, st)
