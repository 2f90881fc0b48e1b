"""A training step out of the library's operators: token embedding, two gated MLP blocks with norms before and after them, gates
and scaled residual additions on an fp32 residual stream, the tied LM head with its loss, all gradients, and clipping by the
global norm; against the same step differentiated in 64 bits on the CPU.

Bar: 2e-2 of the largest gradient, that of the library's other parity tests.  Between the parameters and a gradient there are about 20
roundings to bf16 (half a step of 2^-9 of the value each, independent): 20 ** 0.5 * 2^-9 * 0.6 = 5e-3 of a typical value."""
import threading

import numpy as np
import pytest
import torch

from paper_2506_13996_amd import binding as B

pytestmark = pytest.mark.gpu
IGN, TOL, EPS = -100, 2e-2, 1e-5


class Step:
    """Parameters, buffers and the calls, in the order of a step."""

    def __init__(self, N, H, I, V, blocks=2, seed=0, max_norm=0.25):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, std=1.0: (std * torch.randn(s, generator=g)).to(torch.bfloat16)  # noqa: E731
        self.N, self.H, self.I, self.V, self.tile, self.max_norm = N, H, I, V, 256, max_norm
        self.p = {"E": r(V, H, std=0.05), "w_in": r(H, std=0.1), "w_out": r(H, std=0.1)}
        for k in range(blocks):
            self.p.update({f"Wg{k}": r(I, H, std=0.06), f"Wu{k}": r(I, H, std=0.06), f"Wd{k}": r(H, I, std=0.06), f"w_post{k}": r(H, std=0.1)})
            if k + 1 < blocks:
                self.p[f"w_pre{k}"] = r(H, std=0.1)
        self.blocks = blocks
        rng = np.random.default_rng(seed)
        t = rng.integers(0, V, N).astype(np.int32)
        t[rng.random(N) < 0.3] = 7                  # a token that is common
        t[N - N // 10:] = IGN                       # padding at the end
        self.tokens = torch.from_numpy(t)
        self.gates = r(blocks, N)
        # device side
        new = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
        f32 = torch.float32
        self.d = {k: v.cuda() for k, v in self.p.items()}
        self.t, self.z = self.tokens.cuda(), self.gates.cuda()
        self.y = torch.empty_like(self.t)
        self.res = [new(N, H, dtype=f32) for _ in range(blocks + 1)]
        self.normed = [new(N, H) for _ in range(blocks + 1)]
        self.out = [new(N, H) for _ in range(blocks)]
        self.loss = new(1, dtype=f32)
        self.dn, self.dr, self.db = new(N, H), new(N, H, dtype=f32), new(N, H)
        self.dz = new(blocks, N)
        # matrices' gradients in fp32, the norms' in bf16
        self.grad = {k: new(*v.shape, dtype=f32 if v.dim() == 2 else torch.bfloat16) for k, v in self.d.items()}
        self.clipped = {k: torch.empty_like(v) for k, v in self.grad.items()}
        self.handle = B.GradTensors(self.grad.values(), self.clipped.values())
        self.norm = new(1, dtype=f32)
        F = B.ALST_FLAG_DW_FP32
        self.ws = {"mlp": B.alloc_mlp_workspace(N, H, I, self.tile, False), "mlp_b": B.alloc_mlp_workspace(N, H, I, self.tile, True, F),
                   "ce": B.alloc_workspace(N, H, V, self.tile, F), "norm": B.alloc_block_norm_workspace(N, H),
                   "embed": B.alloc_embedding_workspace(N, H, V), "grads": B.alloc_grad_norm_workspace(self.handle)}

    def parts(self, k):
        last = k + 1 == self.blocks
        return dict(branch=self.out[k], w_post=self.d[f"w_post{k}"], gate=self.z[k], w_pre=self.d["w_out" if last else f"w_pre{k}"],
                    branch_scale=0.7, eps=EPS, weight_offset=1.0)

    def run(self):
        d, g, R, F = self.d, self.grad, B.ALST_FLAG_RESIDUAL_FP32, B.ALST_FLAG_DW_FP32
        scale = self.H ** 0.5
        B.alst_shift_labels(self.t, self.y, IGN)
        B.alst_embedding_forward(self.t, d["E"], scale, IGN, y=self.res[0], flags=R)
        B.alst_block_norm_forward(self.res[0], w_pre=d["w_in"], eps=EPS, weight_offset=1.0, normed=self.normed[0], flags=R)
        for k in range(self.blocks):
            B.alst_tiled_mlp_forward(self.normed[k], d[f"Wg{k}"], d[f"Wu{k}"], d[f"Wd{k}"], self.tile, y=self.out[k], workspace=self.ws["mlp"])
            B.alst_block_norm_forward(self.res[k], **self.parts(k), residual_out=self.res[k + 1], normed=self.normed[k + 1], flags=R)
        B.alst_tiled_ce_forward_backward(self.normed[-1], d["E"], self.y, self.tile, IGN, 1.0, loss_out=self.loss, dHidden=self.dn,
                                         dW=g["E"], workspace=self.ws["ce"], flags=F)
        up = None
        for k in reversed(range(self.blocks)):
            last = k + 1 == self.blocks
            B.alst_block_norm_backward(self.res[k + 1], **self.parts(k), d_normed=self.dn, d_residual_out=up, d_residual=self.dr,
                                       d_branch=self.db, d_gate=self.dz[k], dw_post=g[f"w_post{k}"],
                                       dw_pre=g["w_out" if last else f"w_pre{k}"], workspace=self.ws["norm"], flags=R)
            B.alst_tiled_mlp_backward(self.normed[k], d[f"Wg{k}"], d[f"Wu{k}"], d[f"Wd{k}"], self.db, self.tile, dx=self.dn, dWg=g[f"Wg{k}"],
                                      dWu=g[f"Wu{k}"], dWd=g[f"Wd{k}"], workspace=self.ws["mlp_b"], flags=F)
            up = self.dr
        B.alst_block_norm_backward(self.res[0], w_pre=d["w_in"], eps=EPS, weight_offset=1.0, d_normed=self.dn, d_residual_out=self.dr,
                                   d_residual=self.dr, dw_pre=g["w_in"], workspace=self.ws["norm"], flags=R)
        B.alst_embedding_backward(self.t, self.dr, scale, IGN, dE=g["E"], workspace=self.ws["embed"],
                                  flags=R | F | B.ALST_FLAG_DW_ACCUMULATE)
        B.alst_grad_norm_clip(self.handle, self.max_norm, norm_out=self.norm, workspace=self.ws["grads"])

    def results(self):
        return [self.loss, self.norm, self.dz, *self.grad.values(), *self.clipped.values()]


def _reference(s):
    p = {k: v.double().requires_grad_() for k, v in s.p.items()}
    z = s.gates.double().requires_grad_()
    t = s.tokens.long()
    labels = torch.cat([t[1:], torch.tensor([IGN])])
    norm = lambda x, w: x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * (w + 1)  # noqa: E731
    r = torch.where((t >= 0)[:, None], p["E"][t.clamp(min=0)] * s.H ** 0.5, 0.0)
    n = norm(r, p["w_in"])
    for k in range(s.blocks):
        g, u = n @ p[f"Wg{k}"].T, n @ p[f"Wu{k}"].T
        out = (torch.nn.functional.silu(g) * u) @ p[f"Wd{k}"].T
        r = r + 0.7 * torch.sigmoid(z[k])[:, None] * norm(out, p[f"w_post{k}"])
        n = norm(r, p["w_out" if k + 1 == s.blocks else f"w_pre{k}"])
    loss = torch.nn.functional.cross_entropy(n @ p["E"].T, labels, ignore_index=IGN)
    loss.backward()
    return float(loss.detach()), {k: v.grad for k, v in p.items()}, z.grad


@pytest.mark.parametrize("N,H,I,V", [(700, 128, 200, 1000), (1, 64, 64, 50), (300, 72, 136, 9000)])
def test_a_step_against_64_bits(N, H, I, V):
    s = Step(N, H, I, V, seed=N)
    if N == 1:
        s.t.fill_(3)
        s.tokens.fill_(3)
    s.run()
    loss, grads, dz = _reference(s)
    if N == 1:                                     # one token has no label: no loss, no gradients
        assert float(s.loss) == 0 and float(s.norm) == 0
        assert all(not v.any() for v in s.grad.values()) and not s.dz.any()
        return
    assert abs(float(s.loss) - loss) <= 1e-2 * loss
    total = float(sum((v ** 2).sum() for v in grads.values())) ** 0.5
    for k, v in s.grad.items():
        off = (v.double().cpu() - grads[k]).abs().max()
        assert off <= TOL * grads[k].abs().max(), (k, float(off), float(grads[k].abs().max()))
    assert (s.dz.double().cpu() - dz).abs().max() <= TOL * dz.abs().max()
    assert abs(float(s.norm) - total) <= TOL * total and total > s.max_norm
    for k, v in s.clipped.items():
        want = grads[k] * (s.max_norm / total)
        assert (v.double().cpu() - want).abs().max() <= 2 * TOL * want.abs().max(), k


def test_a_captured_step_follows_its_tokens():
    s = Step(600, 128, 192, 700, seed=5)
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for seed in range(3):
        s.t.copy_(Step(600, 8, 8, 700, seed=seed).tokens)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in s.results()]
        s.run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, s.results()))


def test_two_threads_with_streams_and_workspaces_of_their_own():
    steps = [Step(600, 128, 192, 700, seed=5), Step(350, 264, 96, 3000, seed=6)]
    want = []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in s.results()])
        for t in s.results():
            t.zero_()
    torch.cuda.synchronize()
    failed = []

    def work(s):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(3):
                    s.run()
                torch.cuda.current_stream().synchronize()
        except Exception as e:      # (a thread's exception would be lost)
            failed.append(e)

    threads = [threading.Thread(target=work, args=(s,)) for s in steps]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for s, w in zip(steps, want):
        assert all(torch.equal(a, b) for a, b in zip(s.results(), w))
