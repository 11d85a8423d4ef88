"""Rotary positions: frequencies, and the call that turns queries and keys (or takes their gradients back)."""
from __future__ import annotations

import math
import struct
from typing import Optional, Sequence

import torch

from .binding import _check, _here, _need, _ptr, _stream, load_library

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

# mdss_rope of the C ABI: frequencies, pairs, interleaved, magnitude
_ROPE = struct.Struct("Piif4x")


def rotary_frequencies(dim: int, base: float = 10000.0, scale: float = 1.0, original: Optional[int] = None,
                       turns: Sequence[float] = (1.0, 32.0), divisors: Optional[Sequence[float]] = None) -> torch.Tensor:
    """``[dim / 2]`` float64 (on the CPU): ``base ** (-2 i / dim)`` radians per position, for contexts ``scale`` times as long.

    Without ``original`` all of them are divided by ``scale`` (positions are interpolated, arXiv 2306.15595).  With the context's
    ``original`` length they are divided by parts (arXiv 2309.00071): those that turn less than ``turns[0]`` times over it are divided
    by ``scale``, those that turn more than ``turns[1]`` times are kept, and between them the part kept grows with the turns
    (that paper's magnitude is ``0.1 * log(scale) + 1``).  ``divisors`` (one for each pair) divide them besides."""
    if dim < 2 or dim % 2:
        raise ValueError("dim must be even, 2 or more")
    if not (base > 0.0 and scale > 0.0 and math.isfinite(base) and math.isfinite(scale)):
        raise ValueError("base and scale must be positive")
    f = torch.pow(torch.tensor(float(base), dtype=torch.float64), torch.arange(dim // 2, dtype=torch.float64) * (-2.0 / dim))
    if original is None:
        f = f / scale
    else:
        low, high = turns
        if original < 1 or not 0.0 <= low < high:
            raise ValueError("original must be positive and turns ascending")
        keep = ((original * f / (2.0 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / scale)
    if divisors is not None:
        by = torch.as_tensor(divisors, dtype=torch.float64)
        if by.shape != f.shape or not bool((by > 0).all()):
            raise ValueError(f"divisors must be {dim // 2} positive numbers")
        f = f / by
    return f


class Rotary:
    """How a head's elements are turned: the pairs' frequencies ``[pairs]`` (float64, on the GPU), whether pairs are neighbours
    (``interleaved``) or half of the turned part apart, and the magnitude that turned elements are multiplied by.

    The calls go by the address that the tensor had here: the attributes cannot be set anew, and the tensor is not to be
    given other memory."""

    __slots__ = ("frequencies", "interleaved", "magnitude", "device", "_ref")

    def __init__(self, frequencies: torch.Tensor, interleaved: bool = False, magnitude: float = 1.0):
        if not isinstance(frequencies, torch.Tensor) or frequencies.dim() != 1 or not frequencies.numel():
            raise ValueError("frequencies must be a tensor [pairs]")
        if not frequencies.is_cuda:
            raise ValueError("frequencies must be a GPU tensor")
        _need(frequencies, "frequencies", torch.float64, tuple(frequencies.shape), frequencies.device)
        if not 0.0 < magnitude <= 65536.0:
            raise ValueError("magnitude must be positive, 65536 at most")
        ref = _ROPE.pack(frequencies.data_ptr(), frequencies.numel(), bool(interleaved), magnitude)
        for name, x in zip(self.__slots__, (frequencies, bool(interleaved), float(magnitude), frequencies.device, ref)):
            object.__setattr__(self, name, x)

    def __setattr__(self, name, value):
        raise AttributeError(f"a Rotary keeps its {name}: make another one")

    def __delattr__(self, name):
        raise AttributeError(f"a Rotary keeps its {name}")

    def __reduce__(self):  # copies go by their own tensor's address
        return Rotary, (self.frequencies, self.interleaved, self.magnitude)


def _rope(rope: Rotary, device: torch.device):
    if not isinstance(rope, Rotary):
        raise TypeError("rope must be a Rotary")
    if rope.device != device:
        raise ValueError(f"rope must be on {device}, got {rope.device}")
    return rope._ref


def rotary(x: torch.Tensor, rope: Rotary, positions: torch.Tensor, inverse: bool = False,
           out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``x [T][heads][head_dim]`` (float32, bfloat16 or float16; the last dimension contiguous) turned by ``positions [T]`` int32.

    ``inverse`` turns back: it takes gradients of the result to those of x (with the magnitude, as they need it).  ``out`` may
    be ``x`` itself; otherwise it must not overlap it, and may be a view whose last dimension is contiguous."""
    lib = load_library()
    if x.dim() != 3:
        raise ValueError("x must be [T][heads][head_dim]")
    if not x.is_cuda:
        raise ValueError("x must be a GPU tensor")
    _here(x.device)
    if x.dtype not in _DTYPES:
        raise TypeError(f"x must be float32, bfloat16 or float16, got {x.dtype}")
    T, heads, d = x.shape
    if x.stride(2) != 1 and d > 1 and x.numel():
        raise ValueError("x's last dimension must be contiguous")
    _need(positions, "positions", torch.int32, (T,), x.device)
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    elif out.shape != x.shape or out.dtype != x.dtype or out.device != x.device:
        raise ValueError("out must have x's shape, type and device")
    elif out.stride(2) != 1 and d > 1 and x.numel():
        raise ValueError("out's last dimension must be contiguous")
    _check("mdss_rotary",
           lib.mdss_rotary(_ptr(x), x.stride(0), x.stride(1), _DTYPES[x.dtype], T, heads, d, _ptr(positions),
                           _rope(rope, x.device), inverse, _ptr(out), out.stride(0), out.stride(1), _stream(x.device)))
    return out
