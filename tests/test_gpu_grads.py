"""The global gradient norm and clipping against 64 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import step_oracle as O
from paper_2506_13996_amd import binding as B
from tests import step_util as U

pytestmark = pytest.mark.gpu


def _tensors(sizes, seed=0, std=1.0):
    """(size, fp32, offset in elements): views at that offset of buffers of their own."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for n, f, at in sizes:
        whole = torch.randn(n + at + 3, generator=g).mul_(std).to(torch.float32 if f else torch.bfloat16).cuda()
        out.append(whole[at:at + n])
    return out


def _all(grads, outs, max_norm):
    """The fused call, then the split ones; both results have to be the same bits."""
    h = B.GradTensors(grads, outs)
    ws = U.guarded_workspace(B.alst_grad_norm_workspace_bytes(len(h)))
    S, norm = torch.full((1,), -1.0, dtype=torch.float64, device="cuda"), torch.full((1,), -1.0, device="cuda")
    B.alst_grad_norm_clip(h, max_norm, sumsq_out=S, norm_out=norm, workspace=ws.t)
    fused = [S.clone(), norm.clone()] + [o.clone() for o in outs]
    ws.t.random_(0, 256)
    S.fill_(-1); norm.fill_(-1)
    for o in outs:
        o.zero_()
    B.alst_grad_norm(h, sumsq_out=S, norm_out=norm, workspace=ws.t)
    again = torch.empty_like(norm)
    B.alst_grad_clip(h, S, max_norm, norm_out=again)
    torch.cuda.synchronize()
    assert ws.intact()
    bits = lambda t: t.contiguous().view(torch.uint8)  # noqa: E731
    for a, b in zip(fused, [S, norm] + outs):
        assert torch.equal(bits(a), bits(b))
    assert torch.equal(bits(again), bits(norm))
    return float(S), float(norm)


def _check(grads, outs, S, norm, max_norm):
    wS, wn, want = O.grad_norm_clip([U.to64(g) for g in grads], max_norm)
    # fp64: fewer than 2^12 additions one behind the other, in 2^-53 steps, far below the bound; norm is
    # rounded to fp32 once
    assert abs(S - wS) <= 1e-12 * wS
    assert abs(norm - wn) <= U.FP32 * wn * (1 + 1e-6)
    for k, (o, w, g) in enumerate(zip(outs, want, grads)):
        if wn <= max_norm:
            assert torch.equal(o, g)
        else:                                 # the factor rounded, the product rounded
            U.check(f"out {k}", o, w, np.abs(w), 2)


SIZES = {
    "one element": [(1, False, 0)],
    "one fp32 element": [(1, True, 1)],
    "short": [(7, False, 0), (8, False, 0), (9, False, 0), (3, True, 0), (4, True, 0), (5, True, 0)],
    "every phase": [(1000 + k, False, k) for k in range(8)] + [(1000 + k, True, k) for k in range(4)],
    "short at every phase": [(3, False, k) for k in range(8)] + [(2, True, k) for k in range(4)],
    "chunk edges": [(8192 * k + d, False, 0) for d in (-1, 0, 1) for k in (1, 2)] + [(4096 * k + d, True, 0) for d in (-1, 0, 1) for k in (1, 2)]
    + [(8192 - 3, False, 3), (8192 - 3, False, 5), (4096 - 1, True, 1)],
    "empty ones": [(0, False, 0), (5, False, 0), (0, True, 0), (0, False, 0), (70000, True, 0), (0, True, 0)],
    "many": [(1 + 37 * k, k % 3 == 0, k % 5) for k in range(200)],
    "large": [(5_000_001, False, 1), (3_000_000, True, 0), (11, False, 0)],
}


@pytest.mark.parametrize("name", list(SIZES))
@pytest.mark.parametrize("clipped", [True, False])
def test_norm_and_clip(name, clipped):
    grads = _tensors(SIZES[name], 3)
    total = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    max_norm = float(np.float32(0.37 * total if clipped else 1.5 * total))
    outs = [torch.empty(g.numel() + 16, dtype=g.dtype, device="cuda")[:g.numel()] for g in grads]
    S, norm = _all(grads, outs, max_norm)
    _check(grads, outs, S, norm, max_norm)
    # outputs at the gradients' own phase, between guards
    rooms = [U.Guarded((g.numel() + 16,), g.dtype, 77) for g in grads]
    outs = []
    for g, r in zip(grads, rooms):
        at = g.storage_offset()
        outs.append(r.t[at:at + g.numel()])
    S2, norm2 = _all(grads, outs, max_norm)
    assert (S, norm) == (S2, norm2)
    _check(grads, outs, S2, norm2, max_norm)
    for g, r in zip(grads, rooms):
        at, n = g.storage_offset(), g.numel()
        assert r.intact() and (r.t[:at] == 77).all() and (r.t[at + n:] == 77).all()
    # in place
    inside = _tensors(SIZES[name], 3)
    B.alst_grad_norm_clip(inside, max_norm, workspace=B.alloc_grad_norm_workspace(inside))
    assert all(torch.equal(a, b) for a, b in zip(inside, outs))


def test_more_tensors_than_a_launch_lists_with_empty_ones_between():
    sizes = [(0 if k % 2 else 20000 + k, k % 4 == 0, 0) for k in range(300)]
    grads = _tensors(sizes, 5)
    outs = [torch.empty_like(g) for g in grads]
    S, norm = _all(grads, outs, 1.0)
    _check(grads, outs, S, norm, 1.0)
    outs = [torch.empty_like(g) for g in grads[1::2]]         # nothing at all
    S, norm = _all(grads[1::2], outs, 1.0)
    assert S == 0 and norm == 0


def test_extreme_values():
    big, small = torch.full((4000,), 3e38, device="cuda"), torch.full((4000,), 1e-30, device="cuda")
    for g in (big / 1e6, small, small.to(torch.bfloat16)):
        outs = [torch.empty_like(g)]
        max_norm = float(g[0].double())
        S, norm = _all([g], outs, max_norm)
        _check([g], outs, S, norm, max_norm)
    zero = torch.zeros(100, device="cuda")
    outs = [torch.empty_like(zero)]
    S, norm = _all([zero], outs, 1.0)
    assert S == 0 and norm == 0 and (outs[0] == 0).all()
    g = torch.ones(100, device="cuda")
    outs = [torch.empty_like(g)]
    S, norm = _all([g], outs, float("inf"))
    assert norm == 10 and torch.equal(outs[0], g)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_gradients_of_a_norm_that_is_not_finite_are_left(bad):
    grads = _tensors([(1000, False, 1), (50000, True, 0)], 9)
    grads[1][777] = bad
    outs = [torch.empty_like(g) for g in grads]
    h = B.GradTensors(grads, outs)
    norm = torch.zeros(1, device="cuda")
    B.alst_grad_norm_clip(h, 1.0, norm_out=norm, workspace=B.alloc_grad_norm_workspace(h))
    assert not math.isfinite(float(norm))
    for g, o in zip(grads, outs):
        assert torch.equal(g.view(torch.uint8) if g.storage_offset() == 0 else g.clone().view(torch.uint8), o.view(torch.uint8))
    # a finite sum whose root fp32 cannot hold
    g = torch.full((4000,), 3e38, device="cuda")
    keep = g.clone()
    B.alst_grad_norm_clip([g], 1.0, norm_out=norm, workspace=B.alloc_grad_norm_workspace([g]))
    assert math.isinf(float(norm)) and torch.equal(g, keep)


def test_ranks_that_add_their_sums():
    """Two ranks' gradients, clipped by the sum of both ranks' sums, as after an all-reduce."""
    parts = [_tensors([(5000, True, 0), (300, False, 3)], seed) for seed in (1, 2)]
    sums = [torch.empty(1, dtype=torch.float64, device="cuda") for _ in parts]
    for g, s in zip(parts, sums):
        B.alst_grad_norm(g, sumsq_out=s, workspace=B.alloc_grad_norm_workspace(g))
    both = sums[0] + sums[1]
    want = O.grad_norm_clip([U.to64(g) for p in parts for g in p], 2.0)[2]
    for p in parts:
        B.alst_grad_clip(p, both, 2.0)
    for k, g in enumerate(g for p in parts for g in p):
        U.check(f"gradient {k}", g, want[k], np.abs(want[k]), 2)


def test_captured_calls_follow_their_inputs():
    sizes = [(30000, False, 1), (9000, True, 0), (17, False, 0)]
    sets = [_tensors(sizes, seed, std) for seed, std in ((1, 1.0), (2, 1e-3), (3, 5.0))]
    grads, outs = _tensors(sizes, 0), [torch.empty(n, dtype=torch.float32 if f else torch.bfloat16, device="cuda") for n, f, _ in sizes]
    h = B.GradTensors(grads, outs)
    ws, norm = B.alloc_grad_norm_workspace(h), torch.zeros(1, device="cuda")
    B.alst_grad_norm_clip(h, 1.0, norm_out=norm, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.alst_grad_norm_clip(h, 1.0, norm_out=norm, workspace=ws)
    for s in sets + sets[:2]:
        for a, b in zip(grads, s):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = [norm.clone()] + [o.clone() for o in outs]
        B.alst_grad_norm_clip(h, 1.0, norm_out=norm, workspace=ws)
        assert all(torch.equal(a, b) for a, b in zip(got, [norm] + outs))
        _check(grads, outs, O.grad_norm_clip([U.to64(g) for g in grads], 1.0)[0], float(norm), 1.0)
