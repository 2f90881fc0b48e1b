"""Host-only: how the binding of the operators around the tiled layers takes lists of gradients."""
import pytest
import torch

from paper_2506_13996_amd import binding as B


class _Device(torch.Tensor):
    """A host tensor that says it is a device tensor, for calls that end before the library."""
    @property
    def is_cuda(self):
        return True


def _device(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(_Device)


def test_gradients_may_come_from_an_iterator():
    grads = [_device(4), _device(6, 2, dtype=torch.float32)]
    want = B.GradTensors(grads)
    for given in (iter(grads), (g for g in grads), dict(enumerate(grads)).values()):
        h = B.GradTensors(given)
        assert h.grads == grads and h.outs == grads
        assert [(a.grad, a.out, a.n, a.fp32) for a in h.array] == [(a.grad, a.out, a.n, a.fp32) for a in want.array]
    outs = [_device(4), _device(6, 2, dtype=torch.float32)]
    h = B.GradTensors(iter(grads), iter(outs))
    assert h.grads == grads and h.outs == outs
    # nothing shared between the two lists of a handle
    assert B.GradTensors(grads).outs is not grads
    with pytest.raises(TypeError, match="2 gradients and 1 outs"):
        B.GradTensors(iter(grads), iter(outs[:1]))


def test_calls_take_an_iterator_of_gradients():
    """They get as far as the check of their other tensors' place."""
    for call in (lambda g: B.alst_grad_norm(g, sumsq_out=torch.zeros(1, dtype=torch.float64), workspace=torch.zeros(64, dtype=torch.uint8)),
                 lambda g: B.alst_grad_clip(g, torch.zeros(1, dtype=torch.float64), 1.0),
                 lambda g: B.alst_grad_norm_clip(g, 1.0, workspace=torch.zeros(64, dtype=torch.uint8))):
        with pytest.raises(TypeError, match="must be a device tensor, got device cpu"):
            call(g for g in [_device(4), _device(3)])
