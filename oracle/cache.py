"""64-bit counterparts of the paged 8-bit cache's calls, on numpy arrays and Python lists.

A pool is a dict of k [L][N][H][U][C][16][16], v [L][N][H][U][D][16] (uint8 e4m3 codes) and k_exp, v_exp
[L][N][H] (int8); see the layout in include/mdss.h.  Nothing here is shared with the library.
"""
from __future__ import annotations

import math

import numpy as np

EXP_MIN, EXP_MAX = -40, 40


def decode(codes: np.ndarray) -> np.ndarray:
    """e4m3 codes as numbers: sign, 4 bits of exponent (bias 7), 3 of fraction; 0x7f and 0xff are NaN."""
    c = codes.astype(np.int64)
    x, m = (c >> 3) & 15, c & 7
    mag = np.where(x > 0, (8 + m) * np.exp2(x - 10.0), m * 2.0 ** -9)
    mag = np.where((c & 127) == 127, np.nan, mag)
    return np.where(c & 128, -mag, mag)


def encode(x: np.ndarray) -> np.ndarray:
    """The nearest code, ties to the even one; beyond 448 the largest; non-finite: NaN of its sign."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.minimum(np.abs(x), 448.0), 0.0)
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    q = np.rint(a / np.exp2(e - 3)).astype(np.int64)  # 8 .. 16 (below 8: subnormal)
    e = np.where(q == 16, e + 1, e).astype(np.int64)
    q = np.where(q == 16, 8, q)
    code = np.where(q >= 8, ((e + 7) << 3) | (q & 7), q)
    code = np.where(np.isfinite(x), code, 127)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def exponent(amax: float) -> int:
    e = EXP_MIN
    while e < EXP_MAX and amax > 448.0 * 2.0 ** e:
        e += 1
    return e


def new_pool(layers, pages, heads, d, ps, rng=None):
    """Zeros, or any bytes (NaN codes among them) from rng."""
    shapes = {"k": (layers, pages, heads, ps // 16, d // 16, 16, 16), "v": (layers, pages, heads, ps // 16, d, 16)}
    pool = {n: np.zeros(s, np.uint8) if rng is None else rng.integers(0, 256, s, dtype=np.uint8)
            for n, s in shapes.items()}
    for n in ("k_exp", "v_exp"):
        pool[n] = (np.full((layers, pages, heads), EXP_MIN, np.int8) if rng is None else
                   rng.integers(EXP_MIN, EXP_MAX + 1, (layers, pages, heads), dtype=np.int8))
    return pool


def tokens_of(pool, name, layer, page, head):
    """The codes of a page and head as a view [tokens][d]."""
    x = pool[name][layer, page, head]
    if name == "k":  # unit, chunk, token, element
        return x.transpose(0, 2, 1, 3).reshape(x.shape[0] * 16, -1)
    return x.transpose(0, 2, 1).reshape(x.shape[0] * 16, -1)


def put_tokens(pool, name, layer, page, head, codes):
    x = pool[name][layer, page, head]
    if name == "k":
        x[...] = codes.reshape(x.shape[0], 16, x.shape[1], 16).transpose(0, 2, 1, 3)
    else:
        x[...] = codes.reshape(x.shape[0], 16, x.shape[1]).transpose(0, 2, 1)


def append(pool, layer, key, value, starts, table, lengths):
    """key, value [T][H][D] (float64).  Changes the pool; returns the rows without a page."""
    ps, pages, H = pool["v"].shape[3] * 16, pool["k"].shape[1], pool["k"].shape[2]
    missing = set()
    for s in range(len(lengths)):
        n, L = int(starts[s + 1] - starts[s]), int(lengths[s])
        if n == 0:
            continue
        if L - n < 0 or L > table.shape[1] * ps:
            missing.add(s)
            continue
        p = L - n
        while p < L:
            o = p % ps
            m = min(ps - o, L - p)
            page = int(table[s, p // ps])
            if not 0 <= page < pages:
                missing.add(s)
                p += m
                continue
            at = int(starts[s]) + p - (L - n)
            for name, x in (("k", key), ("v", value)):
                for h in range(H):
                    new = np.asarray(x[at:at + m, h], np.float64)
                    mags = np.abs(new[np.isfinite(new)])
                    e = exponent(float(mags.max()) if mags.size else 0.0)
                    codes = tokens_of(pool, name, layer, page, h).copy()
                    if o:
                        old = int(pool[name + "_exp"][layer, page, h])
                        e = max(e, old)
                        if e > old:
                            held = codes[:o]
                            codes[:o] = np.where((held & 127) == 127, held, encode(decode(held) * 2.0 ** (old - e)))
                    codes[o:o + m] = encode(new * 2.0 ** -e)
                    put_tokens(pool, name, layer, page, h, codes)
                    pool[name + "_exp"][layer, page, h] = e
            p += m
    return missing


def sequence(pool, name, layer, row, length, head):
    """Dequantised tokens [length][d] of a row, and which of them have a page."""
    ps, pages = pool["v"].shape[3] * 16, pool["k"].shape[1]
    d = pool["v"].shape[4]
    out, ok = np.zeros((length, d)), np.zeros(length, bool)
    for j in range((length + ps - 1) // ps):
        page = int(row[j])
        m = min(ps, length - j * ps)
        if 0 <= page < pages:
            ok[j * ps:j * ps + m] = True
            out[j * ps:j * ps + m] = (decode(tokens_of(pool, name, layer, page, head)[:m]) *
                                      2.0 ** int(pool[name + "_exp"][layer, page, head]))
    return out, ok


def attention(pool, layer, q, starts, table, lengths, scale):
    """(out, lse, mag, slack) in float64 for q [T][heads_q][D]: mag = sum_j p_j |v_j|, slack = max_j |scale| |q| . |k_j|,
    the magnitudes that a rounding of the weights and of the scores is relative to."""
    ps, H = pool["v"].shape[3] * 16, pool["k"].shape[2]
    T, hq, d = q.shape
    G = hq // H
    out, lse = np.full((T, hq, d), np.nan), np.full((T, hq), np.nan)
    mag, slack = np.zeros((T, hq, d)), np.zeros((T, hq))
    for s in range(len(lengths)):
        a, n = int(starts[s]), int(starts[s + 1] - starts[s])
        L = max(0, min(int(lengths[s]), table.shape[1] * ps))
        for h in range(H):
            k, ok = sequence(pool, "k", layer, table[s], L, h)
            v, _ = sequence(pool, "v", layer, table[s], L, h)
            for i in range(n):
                upto = max(0, min(L, int(lengths[s]) - n + i + 1))
                see = ok[:upto]
                rows = slice(h * G, (h + 1) * G)
                if not see.any():
                    out[a + i, rows], lse[a + i, rows] = 0.0, -math.inf
                    continue
                kk, vv = k[:upto][see], v[:upto][see]
                qq = np.asarray(q[a + i, rows], np.float64)
                with np.errstate(invalid="ignore"):
                    x = (qq @ kk.T) * scale
                    m = x.max(axis=1, keepdims=True)
                    e = np.exp(x - m)
                    z = e.sum(axis=1, keepdims=True)
                    out[a + i, rows] = (e / z) @ vv
                    lse[a + i, rows] = (m + np.log(z))[:, 0]
                    mag[a + i, rows] = (e / z) @ np.abs(vv)
                    slack[a + i, rows] = (np.abs(qq) @ np.abs(kk).T).max(axis=1) * abs(scale)
    return out, lse, mag, slack


def fork(pool, table, lengths, refs, parent=None, keep=None, grow=None):
    """(table, lengths, refs, flagged rows); the pool's copied pages change in place."""
    ps, pages = pool["v"].shape[3] * 16, pool["k"].shape[1]
    S, width = table.shape
    parent = list(range(S)) if parent is None else [int(x) for x in parent]
    now = [int(x) for x in refs]
    free = [p for p in range(pages) if now[p] == 0]
    good = lambda p: 0 <= p < pages  # noqa: E731
    count = lambda s: (max(0, min(int(lengths[s]), width * ps)) + ps - 1) // ps  # noqa: E731
    for s in range(S):
        for p in table[s, :count(s)]:
            if good(p):
                now[p] -= 1
    rows, lens, more, flagged = [], [], [], set()
    for i, p in enumerate(parent):
        L = 0
        if 0 <= p < S:
            L = max(0, min(int(lengths[p]), width * ps))
            if keep is not None:
                L = min(L, max(0, int(keep[i])))
        row = [int(x) if good(x) else -1 for x in table[p, :(L + ps - 1) // ps]] if L else []
        for x in row:
            if x >= 0:
                now[x] += 1
        g = max(0, int(grow[i])) if grow is not None and 0 <= p < S else 0
        if L + g > width * ps:
            flagged.add(i)
            g = 0
        rows.append(row)
        lens.append(L)
        more.append(g)
    # rows that grow on a page which others hold take a copy, in order, the last holder none
    left, copies = list(now), []
    for i, row in enumerate(rows):
        if more[i] and lens[i] % ps and row[-1] >= 0 and left[row[-1]] > 1:
            copies.append(i)
            left[row[-1]] -= 1
    need = len(copies) + sum((L + g + ps - 1) // ps - (L + ps - 1) // ps for L, g in zip(lens, more))
    out = np.full((len(parent), width), -1, np.int32)
    if need > len(free):
        flagged |= {i for i, g in enumerate(more) if g}
        more = [0] * len(more)
        copies = []
    take = iter(free)
    moved = []
    for i, row in enumerate(rows):
        if i in copies:
            p = next(take)
            moved.append((row[-1], p))
            now[row[-1]] -= 1
            now[p] = 1
            row[-1] = p
        for _ in range((lens[i] + more[i] + ps - 1) // ps - (lens[i] + ps - 1) // ps):
            p = next(take)
            now[p] = 1
            row.append(p)
        out[i, :len(row)] = row
    for name in ("k", "v", "k_exp", "v_exp"):
        for a, b in moved:
            pool[name][:, b] = pool[name][:, a]
    return out, np.array([L + g for L, g in zip(lens, more)], np.int32), np.array(now, np.int32), flagged


def compact(pool, table, lengths, refs):
    """(table, refs, used); the pool's moved pages change in place."""
    ps = pool["v"].shape[3] * 16
    held = [p for p in range(len(refs)) if refs[p] > 0]
    used = len(held)
    holes = [p for p in range(used) if refs[p] <= 0]
    to = {p: p for p in held}
    for a, b in zip([p for p in reversed(held) if p >= used], holes):
        to[a] = b
        for name in ("k", "v", "k_exp", "v_exp"):
            pool[name][:, b] = pool[name][:, a]
    now = np.zeros(len(refs), np.int32)
    for p in held:
        now[to[p]] = refs[p]
    out = np.full(table.shape, -1, np.int32)
    for s in range(table.shape[0]):
        for j in range(min((max(int(lengths[s]), 0) + ps - 1) // ps, table.shape[1])):
            out[s, j] = to.get(int(table[s, j]), -1)
    return out, now, used
