"""Backward block norms do not go by what the header says that they do not need: whatever it holds, the gradients are the same bits."""
import itertools

import pytest
import torch

from paper_2506_13996_amd import binding as B
from tests import step_util as U
from tests.test_gpu_block_norm import _check_backward, _dev, _inputs

pytestmark = pytest.mark.gpu
SHAPES = [(37, 200), (9, 1600), (5, 8200)]


def _backward(x, fp32, residual_out, branch, **kw):
    """Gradients of the parts that x has, with these tensors as the forward's residual_out and branch."""
    N, H = x["du"].shape
    rows, bf16 = torch.float32 if fp32 else torch.bfloat16, torch.bfloat16
    d = _dev(x)
    out = {"d_residual": U.Guarded((N, H), rows), "d_branch": U.Guarded((N, H), bf16)}
    if x["gate"] is not None:
        out["d_gate"] = U.Guarded(tuple(x["gate"].shape), bf16)
    for w, dw in (("w_post", "dw_post"), ("w_pre", "dw_pre")):
        if x[w] is not None:
            out[dw] = U.Guarded((H,), torch.float32)
    B.alst_block_norm_backward(residual_out, branch=branch, w_post=d["w_post"], gate=d["gate"], w_pre=d["w_pre"], d_normed=d["dn"],
                               d_residual_out=d["du"], **{k: v.t for k, v in out.items()}, workspace=B.alloc_block_norm_workspace(N, H),
                               flags=B.ALST_FLAG_DW_FP32 | (B.ALST_FLAG_RESIDUAL_FP32 if fp32 else 0), **kw)
    torch.cuda.synchronize()
    assert all(o.intact() for o in out.values())
    return {k: v.t for k, v in out.items()}


def _spoiled(t):
    """t on the device, all NaN, and with single elements that are not finite."""
    t = t.cuda()
    yield torch.full_like(t, float("nan"))
    for bad in (float("nan"), float("inf"), -float("inf")):
        s = t.clone()
        s[1, 3] = s[t.shape[0] - 1, t.shape[1] - 1] = bad
        yield s


@pytest.mark.parametrize("N,H", SHAPES)
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("post,gate", list(itertools.product([False, True], ["none", "row", "element"])))
def test_the_stream_without_a_norm_before_the_next_block(N, H, fp32, post, gate):
    x = _inputs(N, H, post, gate, False, fp32)
    branch = x["b"].cuda()
    want = _backward(x, fp32, None, branch)
    assert torch.equal(want["d_residual"].cpu(), x["du"])
    _check_backward(x, want)
    for r in (x["r"].cuda(), *_spoiled(x["r"])):
        got = _backward(x, fp32, r, branch)
        assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.parametrize("N,H", SHAPES)
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("pre", [False, True])
def test_the_branch_without_a_norm_and_a_gate_behind_it(N, H, fp32, pre):
    x = _inputs(N, H, False, "none", pre, fp32)
    r = x["r"].cuda() if pre else None
    want = _backward(x, fp32, r, None, branch_scale=0.5)
    _check_backward(x, want, scale=0.5)
    for b in (x["b"].cuda(), *_spoiled(x["b"])):
        got = _backward(x, fp32, r, b, branch_scale=0.5)
        assert all(torch.equal(got[k], want[k]) for k in want)
