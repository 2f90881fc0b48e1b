"""Helpers of the tests of the operators around the tiled layers: buffers with guards on both sides, bounds by rounding steps."""
from __future__ import annotations

import numpy as np
import torch

GUARD = 64          # elements: keeps the base 16-byte aligned for every type


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


FP32 = half_step(torch.float32)


class Guarded:
    """An output [shape] of `fill` inside a larger buffer; intact() says whether what surrounds it was left alone."""

    def __init__(self, shape, dtype, fill=float("nan"), device="cuda"):
        n = int(np.prod(shape))
        self.whole = torch.full((n + 2 * GUARD,), 77, dtype=dtype, device=device)
        self.t = self.whole[GUARD:GUARD + n].view(shape)
        self.t.fill_(fill)

    def intact(self):
        n = self.t.numel()
        return bool((self.whole[:GUARD] == 77).all()) and bool((self.whole[GUARD + n:] == 77).all())


def guarded_workspace(nbytes, device="cuda"):
    """nbytes of noise, with a guard behind."""
    g = Guarded((max(16, nbytes),), torch.uint8, 0, device)
    g.t.random_(0, 256)
    return g


def to64(t):
    return t.detach().cpu().double().numpy()


def bf16(shape, g, std=1.0, mean=0.0):
    return (mean + std * torch.randn(shape, generator=g)).to(torch.bfloat16)


def check(name, got, want, mag, steps):
    """|got - want| <= half a step of got's type at |want|, if that is rounded from fp32, + steps half steps of fp32 at
    the magnitude of what was added up (and the smallest normal number, below which bf16 and fp32 have fixed steps)."""
    rounding = half_step(got.dtype) if got.dtype != torch.float32 else 0.0
    arithmetic = steps * FP32 * mag
    bound = rounding * (np.abs(want) + arithmetic) + arithmetic + 2.0 ** -126
    off = np.abs(to64(got) - want)
    assert np.isfinite(to64(got)).all(), name
    worst = float(np.max(off / bound)) if off.size else 0.0
    assert worst <= 1.0, f"{name}: {worst:.3g} of the bound"
