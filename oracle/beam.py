"""64-bit counterpart of the beam step."""
from __future__ import annotations

import math

import numpy as np


def select(logits, scores, done=None, n=None, eos=-1):
    """(parent, token, score, done, refused beams) for float64 logits [B][W][V] and scores [B][W]."""
    B, W, V = logits.shape
    n = W if n is None else n
    parent, token = np.full((B, n), -1, np.int32), np.full((B, n), -1, np.int32)
    score, ended = np.full((B, n), -math.inf), np.zeros((B, n), np.uint8)
    refused = set()
    for b in range(B):
        found = []  # (-total, beam, rank in the beam, token)
        for w in range(W):
            s = float(scores[b, w])
            if not math.isfinite(s):
                continue
            if done is not None and done[b, w]:
                found.append((-s, w, 0, eos))
                continue
            x = np.asarray(logits[b, w], np.float64)
            if np.isnan(x).any() or (x == math.inf).any():
                refused.add(b * W + w)
                continue
            if (x == -math.inf).all():
                continue
            m = x.max()
            z = math.log(np.exp(x - m).sum())
            order = np.argsort(-x, kind="stable")[:n]
            found += [(-((x[v] - m) - z + s), w, r, int(v)) for r, v in enumerate(order) if x[v] > -math.inf]
        for j, (t, w, _, v) in enumerate(sorted(found)[:n]):
            parent[b, j], token[b, j], score[b, j] = w, v, -t
            ended[b, j] = bool(done is not None and done[b, w]) or v == eos
    return parent, token, score, ended, refused


def reorder(state, parent):
    B, n = parent.shape
    out = np.zeros((B, n) + state.shape[2:], state.dtype)
    for b in range(B):
        for j in range(n):
            if 0 <= parent[b, j] < state.shape[1]:
                out[b, j] = state[b, parent[b, j]]
    return out
