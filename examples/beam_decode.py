"""Beam search over the paged 8-bit cache: python examples/beam_decode.py [--groups 4 --beams 4 --tokens 32]

A decoder with random weights.  Prompts of unlike length are appended to the cache and attended over in one ragged call;
every step then selects continuations, forks the beams' pages (children share their parents' pages, a partly filled one is
copied when they write to it), and runs the new tokens.  At the end the pool is compacted.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_18234_amd as mdss  # noqa: E402


class Decoder:
    """Layers of attention over the cache and a gated product, in bf16."""

    def __init__(self, vocab=1000, layers=2, heads=2, group=4, head_dim=64, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        width = heads * group * head_dim
        self.layers, self.heads, self.group, self.head_dim, self.width = layers, heads, group, head_dim, width

        def weight(rows, cols):
            return (torch.randn((rows, cols), generator=g, device=device) / rows ** 0.5).bfloat16()

        self.embed = torch.randn((vocab, width), generator=g, device=device).bfloat16()
        self.place = (0.3 * torch.randn((4096, width), generator=g, device=device)).bfloat16()
        self.qkv = [weight(width, width + 2 * heads * head_dim) for _ in range(layers)]
        self.proj = [weight(width, width) for _ in range(layers)]
        self.up = [weight(width, 4 * width) for _ in range(layers)]
        self.down = [weight(2 * width, width) for _ in range(layers)]
        self.head = weight(width, vocab) * 3.0

    def __call__(self, cache, tokens, positions, starts, table, lengths, max_new, max_length):
        """Hidden states of the new tokens, whose keys and values go into the cache."""
        norm = torch.nn.functional.layer_norm
        x = (self.embed[tokens] + self.place[positions]).float()
        nq, nk = self.heads * self.group, self.heads
        for i in range(self.layers):
            h = norm(x, (self.width,)).bfloat16() @ self.qkv[i]
            q, k, v = h.view(h.shape[0], nq + 2 * nk, self.head_dim).split((nq, nk, nk), 1)
            mdss.cache_append(cache, i, k, v, starts, table, lengths)
            a = mdss.cache_attention(q, cache, i, starts, table, lengths, max_new=max_new, max_length=max_length)
            x = x + (a.view(a.shape[0], -1) @ self.proj[i]).float()
            u, w = (norm(x, (self.width,)).bfloat16() @ self.up[i]).chunk(2, 1)
            x = x + ((torch.nn.functional.silu(u) * w) @ self.down[i]).float()
        return norm(x, (self.width,)).bfloat16()

    def logits(self, h):
        return h @ self.head


def decode(model, cache, prompts, beams, tokens, eos=-1):
    """Beam search from `prompts` (lists of token ids).  Returns a dict: history [B][beams][tokens] int32, score and done
    [B][beams], and the table, lengths and refs of the beams after the pool's compaction."""
    if not prompts or not all(prompts):
        raise ValueError("every prompt must hold a token")
    dev = cache.device
    B, W, ps = len(prompts), beams, cache.page_size

    def i32(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    longest = max(len(p) for p in prompts)
    width = (longest + tokens + ps - 1) // ps
    # the prompts: empty rows grow to their lengths, and one ragged call fills them
    table, lengths = torch.full((B, width), -1, dtype=torch.int32, device=dev), i32([0] * B)
    refs = torch.zeros(cache.pages, dtype=torch.int32, device=dev)
    status = torch.zeros(B * W, dtype=torch.int32, device=dev)
    table, lengths, refs = mdss.cache_fork(cache, table, lengths, refs, grow=i32([len(p) for p in prompts]),
                                           row_status=status[:B])
    ends = torch.tensor([len(p) for p in prompts], device=dev).cumsum(0)
    starts = torch.cat((ends.new_zeros(1), ends)).int()
    flat = torch.tensor([t for p in prompts for t in p], device=dev)
    positions = torch.tensor([i for p in prompts for i in range(len(p))], device=dev)
    h = model(cache, flat, positions, starts, table, lengths, longest, longest)
    logits = model.logits(h[ends - 1])[:, None]
    # the first step: W continuations of one row a group
    score = torch.zeros((B, 1), device=dev)
    done = torch.zeros((B, 1), dtype=torch.uint8, device=dev)
    history = torch.zeros((B, 1, tokens), dtype=torch.int32, device=dev)
    group = torch.arange(B, device=dev, dtype=torch.int32)[:, None]
    grow = torch.ones(B * W, dtype=torch.int32, device=dev)
    for step in range(tokens):
        from_rows = logits.shape[1]
        parent, token, score, done = mdss.beam_select(logits, score, done, n=W, eos=eos)
        history = mdss.beam_reorder(history, parent)
        history[:, :, step] = token
        rows = torch.where(parent >= 0, group * from_rows + parent, parent).view(-1)
        # (a beam that has ended keeps its place and is run on, its logits are not looked at)
        table, lengths, refs = mdss.cache_fork(cache, table, lengths, refs, rows, grow=grow, row_status=status)
        at = (lengths - 1).clamp(min=0).long()
        h = model(cache, token.view(-1).clamp(min=0).long(), at, None, table, lengths, 1, longest + step + 1)
        logits = model.logits(h).view(B, W, -1)
    table, refs, used = mdss.cache_compact(cache, table, lengths, refs)
    if bool((status != 0).any()):
        raise RuntimeError("the pool has too few pages")
    return {"history": history, "score": score, "done": done, "table": table, "lengths": lengths, "refs": refs,
            "used": used}


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--groups", type=int, default=4)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=32)
    args = ap.parse_args()
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, 1000, (20 + 13 * b,), generator=g).tolist() for b in range(args.groups)]
    model = Decoder()
    pages = sum(len(p) // 16 + 1 + args.beams * (args.tokens // 16 + 3) for p in prompts)
    cache = mdss.PagedCache.empty(model.layers, pages, model.heads, model.head_dim, 16)
    out = decode(model, cache, prompts, args.beams, args.tokens, eos=7)
    print(f"{int(out['used'])} of {pages} pages in use")
    for b in range(args.groups):
        print(f"group {b}: score {out['score'][b, 0].item():.3f}, tokens {out['history'][b, 0].tolist()}")


if __name__ == "__main__":
    main()
