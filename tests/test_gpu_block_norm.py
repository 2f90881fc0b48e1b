"""The norms around a block, gate and scaled residual, forward and backward against 64 bits."""
import itertools

import numpy as np
import pytest
import torch

from oracle import step_oracle as O
from paper_2506_13996_amd import binding as B
from tests import step_util as U

pytestmark = pytest.mark.gpu

# fp32 operations on the longest path of an output: products and sums of one element (at most 12 each way), a row's sum of H
# squares (8 to 32 a lane, 6 across lanes, up to 16 wavefronts) halved by the square root; backward goes through two norms.
FORWARD, BACKWARD = 64, 160
# of a weight's gradient besides: the rows of a workgroup (here at most 9) of up to 16 at a time, up to 4 partial sums a thread, 4 and
# 16 of these
WEIGHTS = BACKWARD + 96


def _inputs(N, H, post, gate, pre, fp32, seed=0, offset=0.0):
    g = torch.Generator().manual_seed(seed + N * 31 + H)
    rows = torch.float32 if fp32 else torch.bfloat16
    x = {"r": torch.randn((N, H), generator=g).mul_(2).to(rows), "b": U.bf16((N, H), g, 0.5),
         "w_post": U.bf16((H,), g, 0.2, 1 - offset) if post else None, "w_pre": U.bf16((H,), g, 0.2, 1 - offset) if pre else None,
         "gate": {"none": None, "row": U.bf16((N,), g), "element": U.bf16((N, H), g)}[gate],
         "dn": U.bf16((N, H), g) if pre else None, "du": torch.randn((N, H), generator=g).to(rows)}
    return x


def _dev(x):
    return {k: None if v is None else v.cuda() for k, v in x.items()}


def _n(x):
    return {k: None if v is None else U.to64(v) for k, v in x.items()}


def _run_forward(x, fp32, **kw):
    N, H = x["r"].shape
    rows = torch.float32 if fp32 else torch.bfloat16
    ro = U.Guarded((N, H), rows) if x["b"] is not None else None
    n = U.Guarded((N, H), torch.bfloat16) if x["w_pre"] is not None else None
    d = _dev(x)
    B.alst_block_norm_forward(d["r"], branch=d["b"], w_post=d["w_post"], gate=d["gate"], w_pre=d["w_pre"],
                              residual_out=ro and ro.t, normed=n and n.t, flags=B.ALST_FLAG_RESIDUAL_FP32 if fp32 else 0, **kw)
    torch.cuda.synchronize()
    assert all(o is None or o.intact() for o in (ro, n))
    return ro and ro.t, n and n.t


def _run_backward(x, fp32, flags=0, start=None, **kw):
    N, H = x["r"].shape
    rows, sums = torch.float32 if fp32 else torch.bfloat16, torch.float32 if flags & B.ALST_FLAG_DW_FP32 else torch.bfloat16
    out = {"d_residual": U.Guarded((N, H), rows), "d_branch": U.Guarded((N, H), torch.bfloat16) if x["b"] is not None else None,
           "d_gate": U.Guarded(tuple(x["gate"].shape), torch.bfloat16) if x["gate"] is not None else None,
           "dw_post": U.Guarded((H,), sums) if x["w_post"] is not None else None,
           "dw_pre": U.Guarded((H,), sums) if x["w_pre"] is not None else None}
    if start is not None:
        for k in ("dw_post", "dw_pre"):
            if out[k]:
                out[k].t.copy_(start)
    d = _dev(x)
    ws = U.guarded_workspace(B.alst_block_norm_workspace_bytes(N, H))
    B.alst_block_norm_backward(d["r"], branch=d["b"], w_post=d["w_post"], gate=d["gate"], w_pre=d["w_pre"], d_normed=d["dn"],
                               d_residual_out=d["du"], **{k: v and v.t for k, v in out.items()}, workspace=ws.t,
                               flags=flags | (B.ALST_FLAG_RESIDUAL_FP32 if fp32 else 0), **kw)
    torch.cuda.synchronize()
    assert ws.intact() and all(o is None or o.intact() for o in out.values())
    return {k: v.t for k, v in out.items() if v is not None}


def _check_forward(x, ro, n, scale=1.0, eps=1e-6, offset=0.0):
    x = _n(x)
    want = O.block_norm_forward(x["r"], x["b"], x["w_post"], x["gate"], x["w_pre"], scale, eps, offset)
    for name, got in (("residual_out", ro), ("normed", n)):
        if got is not None:
            U.check(name, got, want[name], want["mag_" + name], FORWARD)


def _check_backward(x, got, scale=1.0, eps=1e-6, offset=0.0, start=None):
    x = _n(x)
    want = O.block_norm_backward(x["r"], x["b"], x["w_post"], x["gate"], x["w_pre"], x["dn"], x["du"], scale, eps, offset,
                                 branch=x["b"] is not None)
    for name, t in got.items():
        old = U.to64(start) if start is not None and name.startswith("dw") else 0.0
        U.check(name, t, want[name] + old, want["mag_" + name] + np.abs(old), WEIGHTS if name.startswith("dw") else BACKWARD)


SHAPES = [(1, 8), (3, 64), (5, 504), (5, 512), (7, 520), (9, 1024), (6, 1032), (4, 1600), (3, 2048), (5, 2056), (3, 4096), (2, 5120),
          (2, 12288), (3, 16384)]


@pytest.mark.parametrize("N,H", SHAPES)
@pytest.mark.parametrize("fp32", [False, True])
def test_every_row_length(N, H, fp32):
    x = _inputs(N, H, True, "none", True, fp32)
    _check_forward(x, *_run_forward(x, fp32))
    _check_backward(x, _run_backward(x, fp32))


@pytest.mark.parametrize("post,gate,pre", list(itertools.product([False, True], ["none", "row", "element"], [False, True])))
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("H", [200, 1600])
def test_every_combination_of_parts(post, gate, pre, fp32, H):
    kw = dict(branch_scale=0.6, eps=1e-5, weight_offset=1.0)
    x = _inputs(37, H, post, gate, pre, fp32, offset=1.0)
    s = float(np.float32(0.6))
    _check_forward(x, *_run_forward(x, fp32, **kw), scale=s, eps=float(np.float32(1e-5)), offset=1.0)
    _check_backward(x, _run_backward(x, fp32, **kw), scale=s, eps=float(np.float32(1e-5)), offset=1.0)


@pytest.mark.parametrize("fp32", [False, True])
def test_the_norm_alone_and_missing_gradients(fp32):
    N, H = 21, 264
    x = _inputs(N, H, False, "none", True, fp32)
    x["b"] = None
    _check_forward(x, *_run_forward(x, fp32))
    _check_backward(x, _run_backward(x, fp32))
    x["du"] = None                                   # nothing comes from behind: zeros
    got = _run_backward(x, fp32)
    x["du"] = torch.zeros((N, H))
    _check_backward(x, got)
    # without w_pre, d_residual is d_residual_out and need not be written; residual_out is not read
    x = _inputs(N, H, True, "row", False, fp32)
    d, rows = _dev(x), {}
    for k, shape, dtype in (("d_branch", (N, H), torch.bfloat16), ("d_gate", (N,), torch.bfloat16), ("dw_post", (H,), torch.bfloat16)):
        rows[k] = torch.empty(shape, dtype=dtype, device="cuda")
    B.alst_block_norm_backward(None, branch=d["b"], w_post=d["w_post"], gate=d["gate"], d_residual_out=d["du"], **rows,
                               workspace=B.alloc_block_norm_workspace(N, H), flags=B.ALST_FLAG_RESIDUAL_FP32 if fp32 else 0)
    _check_backward(x, rows)


@pytest.mark.parametrize("N,H", [(9000, 256), (1030, 4096), (2100, 1096), (600, 8200), (300, 16384)])
def test_more_rows_than_workgroups(N, H):
    x = _inputs(N, H, True, "row", True, False)
    _check_forward(x, *_run_forward(x, False))
    got = _run_backward(x, False, B.ALST_FLAG_DW_FP32)
    _check_backward(x, got)
    again = _run_backward(x, False, B.ALST_FLAG_DW_FP32)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("fp32_sums", [False, True])
def test_accumulated_weight_gradients(fp32_sums):
    N, H = 300, 520
    x = _inputs(N, H, True, "none", True, False)
    g = torch.Generator().manual_seed(5)
    flags = B.ALST_FLAG_DW_ACCUMULATE | (B.ALST_FLAG_DW_FP32 if fp32_sums else 0)
    start = torch.randn(H, generator=g).to(torch.float32 if fp32_sums else torch.bfloat16)
    _check_backward(x, _run_backward(x, False, flags, start), start=start)


@pytest.mark.parametrize("fp32", [False, True])
def test_outputs_over_inputs(fp32):
    """The aliases that the header allows give the bits of separate buffers."""
    N, H = 130, 1600
    flags = B.ALST_FLAG_RESIDUAL_FP32 if fp32 else 0
    x = _inputs(N, H, True, "element", True, fp32)
    ro, n = _run_forward(x, fp32)
    d = _dev(x)
    B.alst_block_norm_forward(d["r"], branch=d["b"], w_post=d["w_post"], gate=d["gate"], w_pre=d["w_pre"], residual_out=d["r"],
                              normed=d["b"], flags=flags)
    assert torch.equal(d["r"], ro) and torch.equal(d["b"], n)
    if not fp32:
        d = _dev(x)
        out = torch.empty_like(d["b"])
        B.alst_block_norm_forward(d["r"], branch=d["b"], w_post=d["w_post"], gate=d["gate"], w_pre=d["w_pre"], residual_out=d["b"],
                                  normed=out)
        assert torch.equal(d["b"], ro) and torch.equal(out, n)
    want = _run_backward(x, fp32)
    for over in ("b", "dn"):
        d = _dev(x)
        dw = [torch.empty(H, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        B.alst_block_norm_backward(d["r"], branch=d["b"], w_post=d["w_post"], gate=d["gate"], w_pre=d["w_pre"], d_normed=d["dn"],
                                   d_residual_out=d["du"], d_residual=d["du"], d_branch=d[over], d_gate=d["gate"], dw_post=dw[0],
                                   dw_pre=dw[1], workspace=B.alloc_block_norm_workspace(N, H), flags=flags)
        got = {"d_residual": d["du"], "d_branch": d[over], "d_gate": d["gate"], "dw_post": dw[0], "dw_pre": dw[1]}
        assert all(torch.equal(got[k], want[k]) for k in want), over


def test_rows_of_zeros_large_and_small_values_and_saturated_gates():
    N, H = 8, 520
    x = _inputs(N, H, True, "element", True, False)
    x["r"][0] = 0; x["b"][0] = 0                              # (a padding token)
    x["b"][1] = 0
    x["r"][2] *= 1e15; x["b"][2] *= 1e15                      # squares of 1e30
    x["r"][3] *= 1e-12; x["b"][3] *= 1e-12                    # eps rules
    x["gate"][4] = 80; x["gate"][5] = -80
    x["gate"][6] = 3e38; x["gate"][7] = -3e38
    ro, n = _run_forward(x, False)
    _check_forward(x, ro, n)
    assert (ro[0] == 0).all() and (n[0] == 0).all()
    got = _run_backward(x, False, B.ALST_FLAG_DW_FP32)
    with np.errstate(over="ignore"):
        _check_backward(x, got)


def test_infinite_gates_close_and_open():
    N, H = 6, 200
    for gate in ("row", "element"):
        x = _inputs(N, H, True, gate, True, True)
        x["gate"][0], x["gate"][1] = float("-inf"), float("inf")
        ro, n = _run_forward(x, True)
        got = _run_backward(x, True)
        assert torch.equal(ro[0].cpu(), x["r"][0]) and (got["d_branch"][0] == 0).all()
        assert (got["d_gate"][:2] == 0).all()
        x["gate"][0], x["gate"][1] = -200, 200          # as far as fp32 tells
        _check_forward(x, ro, n)
        _check_backward(x, got)


def test_a_row_with_nan_or_infinity_stays_by_itself():
    N, H = 40, 1600
    x = _inputs(N, H, True, "none", True, False)
    clean_f, clean_b = _run_forward(x, False), _run_backward(x, False)
    x["r"][3, 7] = float("nan"); x["b"][21, 0] = float("inf")
    ro, n = _run_forward(x, False)
    got = _run_backward(x, False)
    others = [i for i in range(N) if i not in (3, 21)]
    for a, b in zip((ro, n), clean_f):
        assert torch.equal(a[others], b[others])
    for k in ("d_residual", "d_branch"):
        assert torch.equal(got[k][others], clean_b[k][others])
    assert torch.isnan(n[3]).all()


def test_captured_calls_follow_their_inputs_and_streams():
    N, H = 333, 1024
    sets = [_dev(_inputs(N, H, True, "row", True, False, seed)) for seed in range(3)]
    x = {k: v.clone() for k, v in sets[0].items()}
    out = {k: torch.empty_like(x["r"]) for k in ("residual_out", "normed", "d_residual", "d_branch")}
    dg, dw = torch.empty_like(x["gate"]), [torch.empty(H, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ws = B.alloc_block_norm_workspace(N, H)
    parts = dict(branch=x["b"], w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"], branch_scale=0.5)

    def step():
        B.alst_block_norm_forward(x["r"], **parts, residual_out=out["residual_out"], normed=out["normed"])
        B.alst_block_norm_backward(out["residual_out"], **parts, d_normed=x["dn"], d_residual_out=x["du"], d_residual=out["d_residual"],
                                   d_branch=out["d_branch"], d_gate=dg, dw_post=dw[0], dw_pre=dw[1], workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    results = [*out.values(), dg, *dw]
    for s in sets + sets[:1]:
        for k in x:
            x[k].copy_(s[k])
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in results]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, results))
