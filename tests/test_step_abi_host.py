"""Host-only checks of the operators around the tiled layers: declared and exported names, workspace sizes, refusals."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2506_13996_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADERS = ("alst_embedding.h", "alst_block_norm.h", "alst_grads.h")
vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2506_13996_amd.build import build_library
        build_library(verbose=False)
    return B.load_library()


def test_every_declared_symbol_is_exported(lib):
    text = "".join(open(os.path.join(ROOT, "include", h)).read() for h in HEADERS)
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(alst_[a-z_0-9]+)\s*\(", text))
    assert declared == set(B.STEP_EXPORTS)
    for name in declared:
        assert hasattr(lib, name), name


def test_the_headers_are_c(tmp_path):
    src = tmp_path / "all.c"
    src.write_text("".join(f'#include "{h}"\n' for h in HEADERS) + "int main(void) { return 0; }\n")
    r = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert ctypes.sizeof(B.GradTensor) == 32


def test_workspace_sizes(lib):
    size = B.alst_embedding_workspace_bytes
    assert size(0, 64, 10) == size(1, 0, 10) == size(1, 64, 0) == size(2 ** 30 + 1, 64, 10) == size(1, 64, 2 ** 24 + 1) == 0
    assert size(1, 2 ** 20 + 8, 10) == 0
    # the sorted order, a share of the rows and a mark a token
    N, H, V = 131072, 4096, 128256
    assert 16 * N < size(N, H, V) <= 16 * N + N * H // 8 + V + (2 << 20)
    for n in (1, 100, 4096, 4097, 8191, 8192, 16383, 16384, 32767, 32768, N):         # a workspace serves shorter calls
        assert size(n, H, V) <= size(n + 1, H, V) <= size(N + 1, H, V)
    norm = B.alst_block_norm_workspace_bytes
    assert norm(0, 64) == norm(1, 0) == norm(5, 16392) == 0
    assert norm(1, 4096) <= norm(2000, 4096) <= 1024 * 8 * 4096 and norm(1 << 30, 4096) == norm(1 << 20, 4096) > 0
    grads = B.alst_grad_norm_workspace_bytes
    assert grads(0) == grads(-1) == grads(2 ** 20 + 1) == 0
    assert 0 < grads(1) <= grads(300) < 1 << 20


def test_embedding_refusals(lib):
    def fwd(tokens=0x1000, E=0x2000, N=4, H=64, V=10, y=0x3000, status=None, flags=0):
        return lib.alst_embedding_forward(vp(tokens), vp(E), N, H, V, -100, 1.0, vp(y), vp(status), flags, None)
    assert fwd(tokens=None) == fwd(E=None) == fwd(y=None) == B.ALST_ERR_NULL
    assert fwd(N=0) == fwd(H=0) == fwd(V=0) == fwd(V=2 ** 24 + 1) == fwd(N=2 ** 30 + 1) == fwd(H=2 ** 20 + 8) == B.ALST_ERR_SHAPE
    assert fwd(H=60) == fwd(E=0x2008) == fwd(y=0x3002) == fwd(tokens=0x1002) == fwd(status=0x4002) == B.ALST_ERR_ALIGN
    assert fwd(flags=B.ALST_FLAG_DW_FP32) == fwd(flags=64) == B.ALST_ERR_UNSUPPORTED

    def bwd(tokens=0x1000, dy=0x2000, N=4, H=64, V=10, dE=0x3000, ws=0x4000, wsb=1 << 40, flags=0):
        return lib.alst_embedding_backward(vp(tokens), vp(dy), N, H, V, -100, 1.0, vp(dE), vp(ws), wsb, flags, None)
    assert bwd(tokens=None) == bwd(dy=None) == bwd(dE=None) == bwd(ws=None) == B.ALST_ERR_NULL
    assert bwd(N=0) == bwd(V=-1) == B.ALST_ERR_SHAPE
    assert bwd(H=4) == bwd(dy=0x2004) == bwd(dE=0x3008) == bwd(ws=0x4008) == bwd(tokens=0x1002) == B.ALST_ERR_ALIGN
    assert bwd(flags=B.ALST_FLAG_REDUCE_SUM) == bwd(flags=B.ALST_FLAG_FORWARD_ONLY) == B.ALST_ERR_UNSUPPORTED
    assert bwd(wsb=B.alst_embedding_workspace_bytes(4, 64, 10) - 1) == B.ALST_ERR_WORKSPACE


def test_block_norm_refusals(lib):
    def fwd(r=0x1000, b=0x2000, w1=0x3000, z=None, cols=0, w2=0x4000, N=4, H=64, eps=1e-6, ro=0x5000, n=0x6000, flags=0):
        return lib.alst_block_norm_forward(vp(r), vp(b), vp(w1), vp(z), cols, vp(w2), N, H, 1.0, eps, 0.0, vp(ro), vp(n), flags, None)
    assert fwd(r=None) == fwd(ro=None) == fwd(n=None) == fwd(w2=None) == B.ALST_ERR_NULL
    # without a branch: nothing of it, and something to do
    assert fwd(b=None) == fwd(b=None, ro=None) == fwd(b=None, w1=None) == B.ALST_ERR_NULL
    assert fwd(b=None, w1=None, ro=None, z=0x7000, cols=1) == fwd(b=None, w1=None, ro=None, w2=None, n=None) == B.ALST_ERR_NULL
    assert fwd(N=0) == fwd(H=0) == fwd(H=16392) == fwd(N=2 ** 30 + 1) == B.ALST_ERR_SHAPE
    assert fwd(z=0x7000) == fwd(z=0x7000, cols=2) == fwd(cols=64) == fwd(cols=1) == B.ALST_ERR_SHAPE
    assert fwd(H=60) == fwd(r=0x1004) == fwd(w1=0x3002) == fwd(n=0x6008) == fwd(z=0x7001, cols=1) == fwd(z=0x7002, cols=64) == B.ALST_ERR_ALIGN
    for eps in (0.0, -1e-6, 1e-40, float("nan"), float("inf")):
        assert fwd(eps=eps) == B.ALST_ERR_UNSUPPORTED
    assert fwd(flags=B.ALST_FLAG_DW_FP32) == fwd(flags=1 << 9) == B.ALST_ERR_UNSUPPORTED

    def bwd(r=0x1000, b=0x2000, w1=0x3000, z=None, cols=0, w2=0x4000, dn=0x5000, du=0x6000, N=4, H=64, dr=0x7000, db=0x8000, dz=None,
            dw1=0x9000, dw2=0xa000, ws=0xb000, wsb=1 << 40, eps=1e-6, flags=0):
        return lib.alst_block_norm_backward(vp(r), vp(b), vp(w1), vp(z), cols, vp(w2), vp(dn), vp(du), N, H, 1.0, eps, 0.0, vp(dr), vp(db),
                                            vp(dz), vp(dw1), vp(dw2), vp(ws), wsb, flags, None)
    for missing in ("r", "b", "w1", "w2", "dn", "dr", "db", "dw1", "dw2", "ws"):
        assert bwd(**{missing: None}) == B.ALST_ERR_NULL, missing
    assert bwd(z=0xc000, cols=1) == bwd(dz=0xc000) == B.ALST_ERR_NULL
    assert bwd(w2=None, dn=None, dw2=None, du=None) == B.ALST_ERR_NULL                  # nothing upstream
    assert bwd(w2=None, dn=None, dw2=None, b=None, w1=None, dw1=None, db=None) == B.ALST_ERR_NULL       # nothing to compute
    assert bwd(N=0) == bwd(H=16392) == bwd(z=0xc000, dz=0xd000, cols=3) == B.ALST_ERR_SHAPE
    assert bwd(H=36) == bwd(dn=0x5008) == bwd(dw1=0x9004) == bwd(dr=0x7002) == bwd(ws=0xb004) == B.ALST_ERR_ALIGN
    assert bwd(eps=0.0) == bwd(flags=B.ALST_FLAG_TILE_SCRATCH) == B.ALST_ERR_UNSUPPORTED
    assert bwd(wsb=B.alst_block_norm_workspace_bytes(4, 64) - 1) == B.ALST_ERR_WORKSPACE


def test_grads_refusals(lib):
    def ts(grad=0x1000, out=0x2000, n=8, fp32=0, reserved=0):
        return (B.GradTensor * 1)(B.GradTensor(grad, out, n, fp32, reserved))
    norm = lambda t, count=1, S=0x3000, ws=0x4000, wsb=1 << 40, nrm=None: lib.alst_grad_norm(t, count, vp(S), vp(nrm), vp(ws), wsb, None)  # noqa: E731
    clip = lambda t, count=1, S=0x3000, m=1.0, nrm=None: lib.alst_grad_clip(t, count, vp(S), m, vp(nrm), None)  # noqa: E731
    both = lambda t, count=1, m=1.0, S=None, ws=0x4000, wsb=1 << 40, nrm=None: lib.alst_grad_norm_clip(  # noqa: E731
        t, count, m, vp(S), vp(nrm), vp(ws), wsb, None)
    for f in (norm, clip, both):
        assert f(None) == f(ts(grad=None)) == B.ALST_ERR_NULL
        assert f(ts(), 0) == f(ts(), -1) == f(ts(), 2 ** 20 + 1) == f(ts(n=-1)) == f(ts(n=2 ** 40 + 1)) == B.ALST_ERR_SHAPE
        assert f(ts(fp32=2)) == f(ts(fp32=-1)) == f(ts(reserved=1)) == B.ALST_ERR_UNSUPPORTED
        assert f(ts(grad=0x1001)) == f(ts(grad=0x1002, fp32=1)) == f(ts(), nrm=0x5002) == B.ALST_ERR_ALIGN
        many = (B.GradTensor * 40)(*[B.GradTensor(0x1000, 0x2000, 2 ** 40, 1, 0)] * 40)
        assert f(many, 40) == B.ALST_ERR_SHAPE
    assert clip(ts(out=None)) == both(ts(out=None)) == norm(ts(), S=None) == clip(ts(), S=None) == B.ALST_ERR_NULL
    assert norm(ts(), ws=None) == both(ts(), ws=None) == B.ALST_ERR_NULL
    assert clip(ts(out=0x2001)) == norm(ts(), S=0x3004) == both(ts(), S=0x3004) == norm(ts(), ws=0x4008) == B.ALST_ERR_ALIGN
    for m in (0.0, -1.0, float("nan")):
        assert clip(ts(), m=m) == both(ts(), m=m) == B.ALST_ERR_UNSUPPORTED
    short = B.alst_grad_norm_workspace_bytes(1) - 1
    assert norm(ts(), wsb=short) == both(ts(), wsb=short) == B.ALST_ERR_WORKSPACE


def test_the_tiled_operators_refuse_an_fp32_stream(lib):
    f = B.ALST_FLAG_RESIDUAL_FP32
    assert lib.alst_tiled_ce_forward(vp(0x1000), vp(0x2000), vp(0x3000), 16, 64, 32, 8, -100, vp(0x4000), None, None, vp(0x5000), 1 << 40, f,
                                     None) == B.ALST_ERR_UNSUPPORTED
    assert lib.alst_tiled_mlp_forward(vp(0x1000), vp(0x2000), vp(0x3000), vp(0x4000), 16, 64, 64, 8, vp(0x5000), vp(0x6000), 1 << 40, f,
                                      None) == B.ALST_ERR_UNSUPPORTED
    assert lib.alst_tiled_linear_forward(vp(0x1000), vp(0x2000), 16, 64, 64, 8, vp(0x5000), None, 0, f, None) == B.ALST_ERR_UNSUPPORTED


def test_binding_refuses_tensors_the_abi_would_reinterpret():
    N, H, V = 4, 16, 10
    bf = lambda *sh: torch.zeros(sh, dtype=torch.bfloat16)  # noqa: E731
    t, ws = torch.zeros(N, dtype=torch.int32), torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(TypeError, match="tokens: must be torch.int32"):
        B.alst_embedding_forward(t.long(), bf(V, H), y=bf(N, H))
    with pytest.raises(TypeError, match="y: expected shape"):
        B.alst_embedding_forward(t, bf(V, H), y=bf(N, H + 8))
    with pytest.raises(TypeError, match="y: must be torch.float32"):
        B.alst_embedding_forward(t, bf(V, H), y=bf(N, H), flags=B.ALST_FLAG_RESIDUAL_FP32)
    with pytest.raises(TypeError, match="E: must be contiguous"):
        B.alst_embedding_forward(t, bf(H, V).t(), y=bf(N, H))
    with pytest.raises(TypeError, match="E: must be a device tensor|tokens: must be a device tensor"):
        B.alst_embedding_forward(t, bf(V, H), y=bf(N, H))
    with pytest.raises(TypeError, match="dE: must be torch.float32"):
        B.alst_embedding_backward(t, bf(N, H), dE=bf(V, H), workspace=ws, flags=B.ALST_FLAG_DW_FP32)
    with pytest.raises(TypeError, match="dE: expected shape"):
        B.alst_embedding_backward(t, bf(N, H), dE=bf(V, H + 8), workspace=ws)
    with pytest.raises(TypeError, match="dy: expected two dimensions"):
        B.alst_embedding_backward(t, bf(2, N, H), dE=bf(V, H), workspace=ws)
    with pytest.raises(TypeError, match="gate: expected shape"):
        B.alst_block_norm_forward(bf(N, H), branch=bf(N, H), gate=bf(N + 1), residual_out=bf(N, H))
    with pytest.raises(TypeError, match="branch: expected shape"):
        B.alst_block_norm_forward(bf(N, H), branch=bf(N, H + 8), residual_out=bf(N, H))
    with pytest.raises(TypeError, match="residual: must be torch.float32"):
        B.alst_block_norm_forward(bf(N, H), w_pre=bf(H), normed=bf(N, H), flags=B.ALST_FLAG_RESIDUAL_FP32)
    with pytest.raises(TypeError, match="d_gate: a tensor is required"):
        B.alst_block_norm_backward(bf(N, H), branch=bf(N, H), gate=bf(N), d_residual_out=bf(N, H), d_branch=bf(N, H))
    with pytest.raises(TypeError, match="dw_pre: must be torch.float32"):
        B.alst_block_norm_backward(bf(N, H), w_pre=bf(H), d_normed=bf(N, H), d_residual=bf(N, H), dw_pre=bf(H), workspace=ws,
                                   flags=B.ALST_FLAG_DW_FP32)
    with pytest.raises(TypeError, match="gradient 1: must be a bfloat16 or float32"):
        B.GradTensors([bf(3), torch.zeros(3, dtype=torch.float16)])
    with pytest.raises(TypeError, match="gradient 0: must be contiguous"):
        B.GradTensors([bf(4, 6).t()])
    with pytest.raises(TypeError, match="out 0: must be torch.bfloat16"):
        B.GradTensors([bf(4)], [torch.zeros(4)])
    with pytest.raises(TypeError, match="1 gradients and 2 outs"):
        B.GradTensors([bf(4)], [bf(4), bf(4)])
    with pytest.raises(TypeError, match="must be a device tensor"):
        B.GradTensors([bf(4)])


def test_host_logic_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    """The sources rebuilt with the sanitizers on the host pass, driven by tests/step_sanitize_main.cpp (no kernel is launched)."""
    from paper_2506_13996_amd.build import CSRC, hipcc_path
    exe = str(tmp_path / "step_sanitize")
    srcs = [os.path.join(ROOT, "tests", "step_sanitize_main.cpp")]
    srcs += [os.path.join(CSRC, f) for f in ("embedding.hip", "block_norm.hip", "grads.hip")]
    cmd = [hipcc_path(), "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), *srcs, "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    assert run.returncode == 0, (run.stdout[-2000:], run.stderr[-4000:])
    assert "runtime error" not in run.stderr and "AddressSanitizer" not in run.stderr, run.stderr[-4000:]
    assert "0 failures" in run.stdout
