"""Block norms: values that are not finite reach the results whose definition contains them, and no others."""
import pytest
import torch

from tests.test_gpu_block_norm import _inputs, _run_backward

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
