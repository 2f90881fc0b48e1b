"""Results of 96 MB and more are written past the caches: the same bits as those of short calls, and right."""
import numpy as np
import pytest
import torch

from paper_2506_13996_amd import binding as B
from tests import step_util as U

pytestmark = pytest.mark.gpu
LIMIT = 96 << 20


def _halves(N):
    return slice(0, N // 2), slice(N // 2, N)


def test_lookup():
    for N, H in ((50001, 1024), (25000, 2048 + 8), (200000, 264)):
        V = 3000
        assert N * H * 2 >= LIMIT > (N - N // 2) * H * 2
        g = torch.Generator().manual_seed(H)
        E = U.bf16((V, H), g).cuda()
        t = torch.randint(-1, V, (N,), generator=g, dtype=torch.int32).cuda()       # (-1: ignored)
        whole, parts = U.Guarded((N, H), torch.bfloat16), torch.empty((N, H), dtype=torch.bfloat16, device="cuda")
        B.alst_embedding_forward(t, E, 3.0, -1, y=whole.t)
        for s in _halves(N):
            B.alst_embedding_forward(t[s], E, 3.0, -1, y=parts[s])
        want = (E[t.clamp(min=0).long()].float() * 3 * (t >= 0)[:, None]).bfloat16()
        assert torch.equal(whole.t, want) and torch.equal(parts, want) and whole.intact()


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("N,V,H", [(3000, 50001, 1024), (30000, 25001, 2056)])
def test_table_gradient(N, V, H, fp32):
    assert V * H * 2 >= LIMIT
    rng = np.random.default_rng(N)
    t = rng.integers(0, V, N).astype(np.int32)
    t[rng.random(N) < 0.2] = 77
    dy = U.bf16((N, H), torch.Generator().manual_seed(N)).cuda()
    dE = U.Guarded((V, H), torch.float32 if fp32 else torch.bfloat16)
    index = torch.from_numpy(t).cuda()
    B.alst_embedding_backward(index, dy, dE=dE.t, workspace=B.alloc_embedding_workspace(N, H, V), flags=B.ALST_FLAG_DW_FP32 if fp32 else 0)
    names, where = torch.unique(index.long(), return_inverse=True)
    zero = lambda: torch.zeros((len(names), H), dtype=torch.float64)  # noqa: E731
    want = zero().index_add_(0, where.cpu(), dy.double().cpu())
    mag = zero().index_add_(0, where.cpu(), dy.double().abs().cpu())
    rows = np.bincount(where.cpu().numpy())[:, None]
    U.check("dE", dE.t[names], want.numpy(), mag.numpy(), rows + 2.0)
    rest = torch.ones(V, dtype=torch.bool, device="cuda")
    rest[names] = False
    assert not dE.t[rest].any() and dE.intact()


@pytest.mark.parametrize("H", [256, 1600, 4096, 8200])
@pytest.mark.parametrize("fp32,gate", [(False, "row"), (True, "element")])
def test_block_norms(H, fp32, gate):
    N = LIMIT // (2 * H) + 3
    g = torch.Generator(device="cuda").manual_seed(H)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    rows = torch.float32 if fp32 else torch.bfloat16
    x = {"residual": r(N, H).to(rows), "branch": r(N, H), "gate": r(N) if gate == "row" else r(N, H), "d_normed": r(N, H), "d_residual_out": r(N, H).to(rows)}
    w = dict(w_post=r(H), w_pre=r(H))
    flags = B.ALST_FLAG_RESIDUAL_FP32 if fp32 else 0

    def call(s):
        n = len(x["branch"][s])
        new = lambda dtype=torch.bfloat16: U.Guarded((n, H), dtype)  # noqa: E731
        ro, no, dr, db, dg = new(rows), new(), new(rows), new(), U.Guarded(tuple(x["gate"][s].shape), torch.bfloat16)
        part = dict(branch=x["branch"][s], gate=x["gate"][s], **w)
        B.alst_block_norm_forward(x["residual"][s], **part, residual_out=ro.t, normed=no.t, flags=flags)
        dw = [torch.empty(H, dtype=torch.float32, device="cuda") for _ in range(2)]
        B.alst_block_norm_backward(ro.t, **part, d_normed=x["d_normed"][s], d_residual_out=x["d_residual_out"][s], d_residual=dr.t, d_branch=db.t,
                                   d_gate=dg.t, dw_post=dw[0], dw_pre=dw[1], workspace=B.alloc_block_norm_workspace(n, H),
                                   flags=flags | B.ALST_FLAG_DW_FP32)
        torch.cuda.synchronize()
        assert all(o.intact() for o in (ro, no, dr, db, dg))
        return [o.t for o in (ro, no, dr, db, dg)], dw

    whole, dw = call(slice(0, N))
    halves = [call(s) for s in _halves(N)]
    for k, t in enumerate(whole):
        assert torch.equal(t, torch.cat([h[0][k] for h in halves]))
    for k, t in enumerate(dw):          # other orders of the rows' sum: half a step of fp32 at the sum of magnitudes for each row of a workgroup
        both = halves[0][1][k].double() + halves[1][1][k].double()
        assert (t.double() - both).abs().max() <= (N / 256 + 200) * U.FP32 * 40 * N ** 0.5 * both.abs().max().clamp(min=1)


def test_clipping():
    n = LIMIT // 2 + 12345
    g = torch.Generator(device="cuda").manual_seed(1)
    grads = [torch.randn(n, generator=g, device="cuda").to(torch.bfloat16), torch.randn(777, generator=g, device="cuda")]
    sumsq = torch.full((1,), 4.0 * n, dtype=torch.float64, device="cuda")
    outs = [U.Guarded((n,), torch.bfloat16), U.Guarded((777,), torch.float32)]
    B.alst_grad_clip(B.GradTensors(grads, [o.t for o in outs]), sumsq, 100.0)
    parts = [torch.empty_like(t) for t in grads]
    for s in _halves(n):
        B.alst_grad_clip(B.GradTensors([grads[0][s]], [parts[0][s]]), sumsq, 100.0)
    B.alst_grad_clip(B.GradTensors(grads[1:], parts[1:]), sumsq, 100.0)
    torch.cuda.synchronize()
    assert all(torch.equal(o.t, p) and o.intact() for o, p in zip(outs, parts))
    want = grads[0].double() * (100.0 / (4.0 * n) ** 0.5)
    assert ((outs[0].t.double() - want).abs() <= want.abs() * (U.half_step(torch.bfloat16) + 2 * U.FP32)).all()
    B.alst_grad_clip(grads, sumsq, 100.0)          # in place
    assert all(torch.equal(a, b) for a, b in zip(grads, parts))
