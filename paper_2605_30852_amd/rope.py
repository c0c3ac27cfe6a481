"""Rotary positions: frequencies, scaled for contexts longer than the trained one, and the tables of cosines and sines that
`cache.PagedCache.append` and `append_heads` take.

Frequencies are few and live on the host; a table is computed on the device's current stream, in one launch."""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional, Tuple

import torch

from . import binding as B

_KINDS = {"linear": B.SPD_ROPE_LINEAR, "ntk": B.SPD_ROPE_BASE, "parts": B.SPD_ROPE_PARTS}


@dataclass(frozen=True)
class RopeScaling:
    """kind "linear": all frequencies / factor; "ntk": the base grows with factor, so that the highest frequency stays and the
    lowest is divided by it; "parts": frequencies that turn `low` times or less over the original context are divided by
    factor, those that turn `high` times or more stay, with a passage between them that is linear in the turns. (Where a
    checkpoint's passage is linear in the pair's index, its frequencies are the caller's to compute: `rope_table` takes any.)"""

    kind: str
    factor: float
    original: int = 0
    low: float = 1.0
    high: float = 32.0


def rope_frequencies(dims: int, base: float, scaling: Optional[RopeScaling] = None) -> torch.Tensor:
    """base^(-2i / dims), i < dims / 2, scaled: float64, on the host."""
    s = None
    if scaling is not None:
        if scaling.kind not in _KINDS:
            raise ValueError(f"scaling must be one of {sorted(_KINDS)}")
        if not 0 <= scaling.original < 1 << 31:  # ctypes would cut it to 32 bits
            raise ValueError("original must be in [0, 2^31)")
        s = B.spd_rope_scaling(_KINDS[scaling.kind], scaling.original, scaling.factor, scaling.low, scaling.high)
    if not 0 <= dims < 1 << 31:
        raise ValueError("dims must be in [0, 2^31)")
    return torch.frombuffer(B.spd_rope_frequencies(dims, base, s), dtype=torch.float64)


def rope_table(freq: torch.Tensor, positions: int, first: int = 0, amplitude: float = 1.0,
               out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, device="cuda") -> Tuple[torch.Tensor, torch.Tensor]:
    """(cos, sin), float32 [positions][pairs], of positions first .. first + positions - 1, times amplitude; into `out`, or new
    tensors on `device`. Angles are those of the frequencies in 64 bits, at any position; each value is rounded once."""
    if freq.dtype is not torch.float64 or freq.dim() != 1 or freq.is_cuda or not freq.is_contiguous():
        raise ValueError("freq must be a contiguous float64 tensor of one dimension on the host")
    if not 0 <= positions < 1 << 31:
        raise ValueError("positions must not be negative, nor 2^31 or more")
    if abs(first) > 1 << 30:
        raise ValueError("first must lie within 2^30 of 0")
    pairs = freq.shape[0]
    if out is None:
        cos = torch.empty((positions, pairs), dtype=torch.float32, device=device)
        sin = torch.empty_like(cos)
        if not cos.is_cuda:
            raise ValueError("a table is made on a GPU")
    else:
        cos, sin = out
        for x in out:
            if x.dtype is not torch.float32 or x.shape != (positions, pairs) or not x.is_cuda or not x.is_contiguous() or \
                    x.get_device() != cos.get_device():
                raise ValueError("out must be two contiguous float32 tensors [positions][pairs] on one GPU")
    i = cos.get_device()

    def call():
        B.spd_rope_table(freq.data_ptr(), pairs, first, positions, amplitude, cos.data_ptr(), sin.data_ptr(),
                         torch._C._cuda_getCurrentRawStream(i))

    if torch._C._cuda_getDevice() == i:  # the library launches on the current device
        call()
    else:
        with torch.cuda.device(i):
            call()
    return cos, sin
