"""Clipping by factors that fp32 holds with fewer bits or not at all."""
import math

import numpy as np
import pytest
import torch

from oracle import step_oracle as O
from paper_2506_13996_amd import binding as B
from tests import step_util as U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("value,max_norm", [(2e38, 1.0), (1e34, 1e-6), (1e30, 1e-14), (1e36, 1e-20), (3e36, 2e-38), (1e30, 1e-30), (2e38, 2e-40)])
def test_factors_below_the_normal_numbers(value, max_norm, fp32):
    """Factors of 2^-126 to 2^-259: the factor's rounding and the product's, half a step of fp32 each."""
    g = torch.Generator().manual_seed(3)
    rows = (value / 250) * torch.randn(30003, generator=g)        # norm about 0.7 value
    grads = [t.to(torch.float32 if fp32 else torch.bfloat16) for t in (rows[:20000], rows[20000:])]      # (whole chunks of 16 KB, and parts)
    dev = [t.cuda() for t in grads]
    outs, norm = [torch.empty(t.numel() + 8, dtype=t.dtype, device="cuda") for t in dev], torch.empty(1, device="cuda")
    outs = [outs[0][:20000], outs[1][1:1 + dev[1].numel()]]          # (the second one's outputs at another 16-byte phase)
    h = B.GradTensors(dev, outs)
    B.alst_grad_norm_clip(h, max_norm, norm_out=norm, workspace=B.alloc_grad_norm_workspace(h))
    max_norm = float(np.float32(max_norm))
    _, total, want = O.grad_norm_clip([U.to64(t) for t in grads], max_norm)
    assert math.isfinite(float(norm)) and max_norm / total < 2.0 ** -126
    for k, (o, w) in enumerate(zip(outs, want)):
        # (below 2^-126 the types have fixed steps of 2^-149 and 2^-133)
        step = 2.0 ** -149 if fp32 else 2.0 ** -133
        bound = np.abs(w) * (2 * U.FP32 + (0.0 if fp32 else U.half_step(torch.bfloat16) * (1 + 2 * U.FP32))) + step
        off = np.abs(U.to64(o) - w)
        assert (off <= bound).all(), (k, float((off / bound).max()))
