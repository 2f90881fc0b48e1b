"""Kernels of the embedding and the block norms that only some sizes, types and gates reach, against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2506_13996_amd import binding as B
from tests import step_util as U
from tests.test_gpu_block_norm import BACKWARD, FORWARD, _check_backward, _check_forward, _inputs, _run_backward, _run_forward
from tests.test_gpu_embedding import _backward, _tokens

pytestmark = pytest.mark.gpu
LIMIT = 96 << 20            # bytes from which on results are written past the caches


@pytest.mark.parametrize("N,H", [(5, 8200), (3, 12288), (2, 16384), (700, 8712)])
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("post", [False, True])
def test_a_gate_for_each_element_of_long_rows(N, H, fp32, post):
    x = _inputs(N, H, post, "element", True, fp32)
    _check_forward(x, *_run_forward(x, fp32))
    _check_backward(x, _run_backward(x, fp32, B.ALST_FLAG_DW_FP32))


@pytest.mark.parametrize("N,H", [(33001, 64), (65539, 8), (33003, 512)])
@pytest.mark.parametrize("gate", ["none", "element"])
def test_forward_of_more_short_rows_than_workgroups_take_at_once(N, H, gate):
    x = _inputs(N, H, True, gate, True, False)
    _check_forward(x, *_run_forward(x, False))


def _additions(rows, run):
    """fp32 additions one behind the other in a token's sum: the rows of a range and those that follow it into the next, the partial sums
    of a wavefront (an eighth of the ranges), eight wavefronts; the scale and the old value."""
    return np.minimum(rows, 2 * run + rows / (8 * run) + 9) + 2.0


# run: rows of a range, 128 where that leaves 4096 wavefronts of 512 columns
@pytest.mark.parametrize("N,H,V,run", [(16385, 256, 3000, 8), (4097, 520, 513, 8), (530001, 8, 700, 128)])
@pytest.mark.parametrize("law", ["zipf", "two", "same"])
@pytest.mark.parametrize("fp32_rows,fp32_sums,accumulate", [(False, True, True), (True, True, True), (False, False, True), (True, True, False),
                                                            (True, False, False)])
def test_table_gradients_sorted_by_many_workgroups(N, H, V, run, law, fp32_rows, fp32_sums, accumulate):
    """Above 4096 rows: rows of fp32, and sums that are added to (no marks of the tokens, no zeros, joins into what is there)."""
    g = torch.Generator().manual_seed(N)
    t = _tokens(law, N, V, 3)
    t[t == 5] = 6                       # a token that does not occur
    dy = torch.randn((N, H), generator=g) if fp32_rows else U.bf16((N, H), g)
    flags = (B.ALST_FLAG_RESIDUAL_FP32 if fp32_rows else 0) | (B.ALST_FLAG_DW_FP32 if fp32_sums else 0)
    start = None
    if accumulate:
        flags |= B.ALST_FLAG_DW_ACCUMULATE
        start = torch.randn((V, H), generator=g).to(torch.float32 if fp32_sums else torch.bfloat16)
        start[5] = float("nan")         # is neither read nor written
    got, status = _backward(t, dy, V, scale=3.0, flags=flags, start=start)
    assert status == B.ALST_OK
    got = U.to64(got)
    old = 0.0
    if accumulate:
        assert np.isnan(got[5]).all()
        got[5] = 0
        start[5] = 0
        old = U.to64(start)
    keep = torch.from_numpy(t >= 0)
    index = torch.from_numpy(t)[keep].long()
    want = 3.0 * torch.zeros((V, H), dtype=torch.float64).index_add_(0, index, dy[keep].double()).numpy() + old
    mag = 3.0 * torch.zeros((V, H), dtype=torch.float64).index_add_(0, index, dy[keep].double().abs()).numpy() + np.abs(old)
    rows = np.bincount(t[t >= 0], minlength=V)[:, None]
    arithmetic = _additions(rows, run) * U.FP32 * mag
    rounding = 0.0 if fp32_sums else U.half_step(torch.bfloat16)
    off = np.abs(got - want)
    bound = rounding * (np.abs(want) + arithmetic) + arithmetic + 2.0 ** -126
    assert (off <= bound).all(), float((off / bound).max())


def _exact(x, w, gate, stored):
    """The definitions in 64 bits on the device, and magnitudes as the oracle has them, a block of rows at a time: yields (slice, {name:
    (value, magnitude)}), then the weights' sums.  stored: the r' that backward goes by."""
    N, H = x["branch"].shape
    sums = {}
    w1, w2 = w["w_post"].double(), w["w_pre"].double()
    for i in range(0, N, max(1, (1 << 24) // H)):
        s = slice(i, i + max(1, (1 << 24) // H))
        d = {k: v[s].double() for k, v in x.items()}
        z = d["gate"] if gate == "element" else d["gate"][:, None]
        mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
        q_of = lambda v: 1.0 / (mean(v * v) + 1e-6).sqrt()  # noqa: E731
        on, off = torch.sigmoid(z), torch.sigmoid(-z)
        q1 = q_of(d["branch"])
        x1 = d["branch"] * q1
        change = on * x1 * w1
        out, mag = d["residual"] + change, d["residual"].abs() + change.abs()
        q = q_of(out)
        res = {"residual_out": (out, mag), "normed": (out * q * w2, mag * q * w2.abs())}
        r = stored[s].double()
        q2 = q_of(r)
        x2, u = r * q2, d["d_normed"] * w2
        dr = d["d_residual_out"] + q2 * (u - x2 * mean(u * x2))
        mag = d["d_residual_out"].abs() + q2 * (u.abs() + x2.abs() * mean((u * x2).abs()))
        dp, mp = on * dr, on * mag
        dz, mz = dp * off * x1 * w1, mp * off * (x1 * w1).abs()
        v, mv = dp * w1, mp * w1.abs()
        res["d_residual"] = (dr, mag)
        res["d_branch"] = (q1 * (v - x1 * mean(v * x1)), q1 * (mv + x1.abs() * mean(mv * x1.abs())))
        res["d_gate"] = (dz, mz) if gate == "element" else (dz.sum(1), mz.sum(1))
        for k, (a, b) in {"dw_pre": (d["d_normed"] * x2, (d["d_normed"] * x2).abs()), "dw_post": (dp * x1, mp * x1.abs())}.items():
            had = sums.get(k, (0.0, 0.0))
            sums[k] = (had[0] + a.sum(0), had[1] + b.sum(0))
        yield s, res
    yield None, sums


@pytest.mark.parametrize("H", [256, 1600, 4096, 8200])
@pytest.mark.parametrize("fp32,gate", [(False, "row"), (True, "element")])
def test_block_norms_of_long_sequences(H, fp32, gate):
    """Rows that are written past the caches, forward of short rows that walks, weights' sums over all rows."""
    N = LIMIT // (2 * H) + 3
    g = torch.Generator(device="cuda").manual_seed(H + 1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    rows = torch.float32 if fp32 else torch.bfloat16
    x = {"residual": r(N, H).to(rows), "branch": r(N, H), "gate": r(N) if gate == "row" else r(N, H), "d_normed": r(N, H),
         "d_residual_out": r(N, H).to(rows)}
    w = dict(w_post=r(H), w_pre=r(H))
    flags = B.ALST_FLAG_RESIDUAL_FP32 if fp32 else 0
    out = {k: U.Guarded((N, H), rows if "residual" in k else torch.bfloat16) for k in ("residual_out", "normed", "d_residual", "d_branch")}
    out["d_gate"] = U.Guarded(tuple(x["gate"].shape), torch.bfloat16)
    out.update({k: U.Guarded((H,), torch.float32) for k in ("dw_post", "dw_pre")})
    t = {k: v.t for k, v in out.items()}
    part = dict(branch=x["branch"], gate=x["gate"], **w)
    B.alst_block_norm_forward(x["residual"], **part, residual_out=t["residual_out"], normed=t["normed"], flags=flags)
    B.alst_block_norm_backward(t["residual_out"], **part, d_normed=x["d_normed"], d_residual_out=x["d_residual_out"],
                               **{k: v for k, v in t.items() if k.startswith("d")}, workspace=B.alloc_block_norm_workspace(N, H),
                               flags=flags | B.ALST_FLAG_DW_FP32)
    torch.cuda.synchronize()
    assert all(o.intact() for o in out.values())
    # a weight's gradient: the rows of one place of 256 workgroups, up to 16 places, 4 workgroups, 4 and 16 of these
    steps = {"residual_out": FORWARD, "normed": FORWARD, "dw_pre": BACKWARD + N / 256 + 1 + 16 + 24, "dw_post": BACKWARD + N / 256 + 1 + 16 + 24}
    for s, want in _exact(x, w, gate, t["residual_out"]):
        for k, (v, mag) in want.items():
            got = t[k] if s is None else t[k][s]
            arithmetic = steps.get(k, BACKWARD) * U.FP32 * mag
            rounding = U.half_step(got.dtype) if got.dtype != torch.float32 else 0.0
            off, bound = (got.double() - v).abs(), rounding * (v.abs() + arithmetic) + arithmetic + 2.0 ** -126
            assert bool((off <= bound).all()), (k, s, float((off / bound).max()))
