"""Block norms: values that are not finite reach the results whose definition contains them, and no others."""
import pytest
import torch

from tests.test_gpu_block_norm import _check_forward, _inputs, _run_backward, _run_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,H", [(37, 200), (9, 1600), (5, 8200)])
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("gate", ["row", "element"])
@pytest.mark.parametrize("pre", [False, True])
def test_a_branch_under_a_gate_alone_is_not_in_its_own_gradient(N, H, fp32, gate, pre):
    """Without a norm after the block d_branch = scale sigmoid(z) dr; the branch is in d_gate alone."""
    x = _inputs(N, H, False, gate, pre, fp32)
    want = _run_backward(x, fp32, branch_scale=0.5)
    for bad in (float("inf"), -float("inf"), float("nan")):
        spoiled = dict(x, b=x["b"].clone())
        spoiled["b"][1, 3] = spoiled["b"][N - 1, H - 1] = bad
        got = _run_backward(spoiled, fp32, branch_scale=0.5)
        same = torch.ones(x["gate"].shape, dtype=torch.bool)
        for i, h in ((1, 3), (N - 1, H - 1)):
            same[(i, h) if gate == "element" else i] = False
        for k in want:
            if k == "d_gate":
                assert torch.equal(got[k][same], want[k][same]) and not torch.isfinite(got[k][~same]).any()
            else:
                assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("fp32", [False, True])
def test_rows_whose_squares_fp32_cannot_add_up(fp32):
    """4096 * 2.8e17^2 = 3.2e38 is below fp32's largest number 3.4e38 by more than the sum's roundings, 4096 * 3e17^2 = 3.7e38 and
    (2e19)^2 = 4e38 are above it: such a row is normalised to zeros."""
    N, H = 6, 4096
    x = _inputs(N, H, True, "none", True, fp32)
    x["r"][1], x["b"][1] = 2.8e17, 0
    _check_forward(x, *_run_forward(x, fp32))
    x["r"][2], x["b"][2] = 3e17, 0
    x["r"][3], x["b"][3] = 0, 0
    x["r"][3, 77] = -2e19
    x["b"][4] = 3e17
    ro, n = _run_forward(x, fp32)
    assert torch.equal(ro[2:5].cpu(), x["r"][2:5]) and (n[2:4] == 0).all()
    got = _run_backward(x, fp32)
    assert torch.equal(got["d_residual"][2:4].cpu(), x["du"][2:4]) and (got["d_branch"][4] == 0).all()
