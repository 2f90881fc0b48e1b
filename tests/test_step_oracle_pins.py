"""The oracle of the operators around the tiled layers against differences, autograd and small worked examples."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as O


def test_embedding_of_a_worked_example():
    E = np.array([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0]])
    t = np.array([2, -100, 0, 2, 7])
    y = O.embedding_forward(t, E, 2.0, -100)
    assert (y == [[10, 12], [0, 0], [2, 4], [10, 12], [0, 0]]).all()
    dE, mag, rows = O.embedding_backward(t, np.arange(10.0).reshape(5, 2) - 4, 2.0, -100, 3)
    assert (dE == [[0, 2], [0, 0], [-4, 0]]).all() and (rows == [1, 0, 2]).all()
    assert (mag[2] == [2 * (4 + 2), 2 * (3 + 3)]).all()


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", ["none", "row", "element"])
@pytest.mark.parametrize("pre", [False, True])
def test_block_norm_gradients_are_those_of_autograd_and_of_differences(post, gate, pre):
    rng = np.random.default_rng(3)
    N, H = 5, 8
    kw = dict(scale=0.7, eps=1e-3, offset=1.0)
    x = {"r": rng.normal(size=(N, H)), "b": rng.normal(size=(N, H)), "w_post": rng.normal(size=H) if post else None,
         "gate": {"none": None, "row": rng.normal(size=N), "element": rng.normal(size=(N, H))}[gate],
         "w_pre": rng.normal(size=H) if pre else None}
    du, dn = rng.normal(size=(N, H)), rng.normal(size=(N, H))

    def value(v):
        f = O.block_norm_forward(v["r"], v["b"], v["w_post"], v["gate"], v["w_pre"], **kw)
        return (f["residual_out"] * du).sum() + ((f["normed"] * dn).sum() if pre else 0.0)

    f = O.block_norm_forward(x["r"], x["b"], x["w_post"], x["gate"], x["w_pre"], **kw)
    g = O.block_norm_backward(f["residual_out"], x["b"], x["w_post"], x["gate"], x["w_pre"], dn if pre else None, du, **kw)
    t = {k: torch.tensor(v, requires_grad=True) for k, v in x.items() if v is not None}
    rms = lambda a, w: a * torch.rsqrt((a * a).mean(1, keepdim=True) + 1e-3) * (w + 1)  # noqa: E731
    p = rms(t["b"], t["w_post"]) if post else t["b"]
    if gate != "none":
        p = p * torch.sigmoid(t["gate"] if gate == "element" else t["gate"][:, None])
    out = t["r"] + 0.7 * p
    loss = (out * torch.tensor(du)).sum() + ((rms(out, t["w_pre"]) * torch.tensor(dn)).sum() if pre else 0.0)
    assert abs(float(loss) - value(x)) < 1e-12
    loss.backward()
    names = {"r": "d_residual", "b": "d_branch", "gate": "d_gate", "w_post": "dw_post", "w_pre": "dw_pre"}
    for k, v in t.items():
        np.testing.assert_allclose(g[names[k]], v.grad.numpy(), rtol=1e-10, atol=1e-12)
        for _ in range(3):
            at = tuple(int(rng.integers(n)) for n in x[k].shape)
            ends = []
            for sign in (1, -1):
                moved = {q: (w.copy() if w is not None else None) for q, w in x.items()}
                moved[k][at] += sign * 1e-6
                ends.append(value(moved))
            assert abs((ends[0] - ends[1]) / 2e-6 - g[names[k]][at]) < 1e-6


def test_clip_of_a_worked_example():
    S, norm, out = O.grad_norm_clip([np.array([3.0]), np.array([[4.0]])], 2.5)
    assert S == 25 and norm == 5 and out[0][0] == 1.5 and out[1][0, 0] == 2
    assert O.grad_norm_clip([np.array([3.0])], 4.0)[2][0][0] == 3
    assert O.grad_norm_clip([np.array([np.inf, 1.0])], 4.0)[2][0][1] == 1
