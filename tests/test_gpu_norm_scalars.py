"""Block norms do not go by a scale or an offset of parts that are absent, whatever it is."""
import pytest
import torch

from paper_2506_13996_amd import binding as B
from tests.test_gpu_block_norm import _dev, _inputs, _run_backward, _run_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,H", [(37, 200), (5, 8200)])
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_scalars_of_absent_parts(N, H, fp32, bad):
    """branch_scale without a branch, weight_offset without weights."""
    x = _inputs(N, H, False, "none", True, fp32)
    x["b"] = None
    _, want = _run_forward(x, fp32)
    _, got = _run_forward(x, fp32, branch_scale=bad)
    assert torch.equal(got, want)
    want, got = _run_backward(x, fp32), _run_backward(x, fp32, branch_scale=bad)
    assert all(torch.equal(got[k], want[k]) for k in want)
    for gate in ("none", "row", "element"):
        x = _inputs(N, H, False, gate, False, fp32)
        want, got = _run_forward(x, fp32)[0], _run_forward(x, fp32, weight_offset=bad)[0]
        assert torch.equal(got, want)
        want, got = _run_backward(x, fp32), _run_backward(x, fp32, weight_offset=bad)
        assert all(torch.equal(got[k], want[k]) for k in want)


def test_scalars_of_absent_parts_beside_a_norm_after_the_block():
    """The next block's norm is absent, the offset is that of the weight that is there."""
    x = _inputs(21, 264, True, "row", False, True)
    rows = {k: torch.empty_like(v) for k, v in _dev({"d_branch": x["b"], "d_gate": x["gate"], "dw_post": x["w_post"]}).items()}
    d = _dev(x)
    B.alst_block_norm_backward(None, branch=d["b"], w_post=d["w_post"], gate=d["gate"], d_residual_out=d["du"], weight_offset=1.0, **rows,
                               workspace=B.alloc_block_norm_workspace(21, 264), flags=B.ALST_FLAG_RESIDUAL_FP32)
    want = _run_backward(x, True, weight_offset=1.0)
    assert all(torch.equal(rows[k], want[k]) for k in rows)
