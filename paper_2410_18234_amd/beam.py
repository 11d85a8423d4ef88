"""Beam search's step: the best continuations over beams and vocabulary, and the reordering of states by parent."""
from __future__ import annotations

import math
from typing import Optional

import torch

from .binding import _check, _need, _ptr, _stream, load_library
from .cache import _scratch

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def beam_select(logits: torch.Tensor, scores: torch.Tensor, done: Optional[torch.Tensor] = None,
                n: Optional[int] = None, eos: int = -1, row_status: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None):
    """(parent, token, score, done), each ``[B][n]``: the n best of ``scores[b][w] + log softmax(logits[b][w])[v]``.

    ``logits`` is ``[B][W][V]`` (fp32, bf16 or fp16; rows may be strided, evenly), ``n`` defaults to W.  Equal totals go to
    the lower beam, then the larger logit, then the lower token.  A beam with ``done`` continues with ``eos`` at its own
    score; places without a candidate hold parent and token -1 and score -inf."""
    lib = load_library()
    if logits.dim() != 3:
        raise ValueError("logits must be [B][W][V]")
    if logits.device.type != "cuda":
        raise ValueError("logits must be a GPU tensor")
    if logits.dtype not in _DTYPES:
        raise TypeError(f"logits must be float32, bfloat16 or float16, got {logits.dtype}")
    B, W, V = logits.shape
    dev = logits.device
    stride = logits.stride(1) if W > 1 else logits.stride(0) if B > 1 else V
    if logits.numel() and (logits.stride(2) != 1 or (B > 1 and W > 1 and logits.stride(0) != W * stride)):
        raise ValueError("logits' rows must be contiguous and evenly strided")
    _need(scores, "scores", torch.float32, (B, W), dev)
    if done is not None:
        _need(done, "done", torch.uint8, (B, W), dev)
    if row_status is not None:
        _need(row_status, "row_status", torch.int32, (B * W,), dev)
    n = W if n is None else n
    parent = torch.empty_strided((B, n), (n, 1), dtype=torch.int32, device=dev)
    token = torch.empty_like(parent)
    score = torch.empty_strided((B, n), (n, 1), dtype=torch.float32, device=dev)
    done_out = torch.empty_strided((B, n), (n, 1), dtype=torch.uint8, device=dev)
    workspace = _scratch(dev, lib.mdss_workspace_bytes_beam(B, W, V, n), workspace)
    _check("mdss_beam_select",
           lib.mdss_beam_select(_ptr(logits), _DTYPES[logits.dtype], stride, _ptr(scores), _ptr(done), B, W, V, n, eos,
                                _ptr(parent), _ptr(token), _ptr(score), _ptr(done_out), _ptr(row_status),
                                _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream(dev)))
    return parent, token, score, done_out


def beam_reorder(state: torch.Tensor, parent: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``out[b][j] = state[b][parent[b][j]]`` for a state ``[B][W][...]`` of any type; zeros where the parent is -1."""
    lib = load_library()
    shape = state.shape
    if len(shape) < 2 or parent.dim() != 2:
        raise ValueError("state must be [B][W][...] and parent [B][n]")
    if not state.is_cuda:
        raise ValueError("state must be a GPU tensor")
    if not state.is_contiguous():
        raise ValueError("state must be contiguous")
    B, W, n = shape[0], shape[1], parent.shape[1]
    _need(parent, "parent", torch.int32, (B, n), state.device)
    if out is None:
        out = torch.empty_like(state) if n == W else torch.empty((B, n) + shape[2:], dtype=state.dtype, device=state.device)
    else:
        _need(out, "out", state.dtype, (B, n) + shape[2:], state.device)
    row = state.element_size() * math.prod(shape[2:])
    _check("mdss_beam_reorder",
           lib.mdss_beam_reorder(_ptr(state), _ptr(parent), B, W, n, row, _ptr(out), _stream(state.device)))
    return out
