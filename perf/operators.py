"""The operators around the tiled layers of a training step, as they are measured: which calls, at which sizes, on which data.

  op "embed"   alst_embedding_forward (entry "forward"), alst_embedding_backward (entry "backward"; "accum": two
               micro-batches whose fp32 gradient is accumulated)
  op "norm"    alst_block_norm_forward / alst_block_norm_backward: the norm after a block, its gate, the scaled residual
               addition and the norm before the next block
  op "grads"   the global gradient norm and clipping: alst_grad_norm_clip (entry "fused"), or alst_grad_norm and then
               alst_grad_clip (entry "split": what data-parallel ranks call, with an all-reduce of the sum between)

The clipped gradients go to tensors of their own, so that a pass can be repeated on the same gradients.

listed() holds the cases, draw() gives more of the same ranges.  With `own` false, run() computes the plain form: elementary
operations in 32 bits, each output rounded once.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

IGNORE = -100
EPS = 1e-6


def _embed(name, N, H, V, entry, law, pad, fp32):
    """fp32: of the rows (y, dy) for "forward" and "backward", which are then those of an fp32 residual stream."""
    return {"name": name, "op": "embed", "entry": entry, "N": N, "H": H, "V": V, "law": law, "pad": pad, "fp32": fp32}


def _norm(name, N, H, entry, post, gate, fp32, offset, scale):
    return {"name": name, "op": "norm", "entry": entry, "N": N, "H": H, "post": post, "gate": gate, "fp32": fp32,
            "offset": offset, "scale": scale}


def _grads(name, entry, layers, H, I, V, fp32, flat, clipped):
    return {"name": name, "op": "grads", "entry": entry, "layers": layers, "H": H, "I": I, "V": V, "fp32": fp32, "flat": flat,
            "clipped": clipped}


def listed():
    return [
        # the smallest lookup: the tiny workload's tokens
        _embed("embed_tiny", 512, 256, 4096, "forward", "uniform", 0.0, False),
        # the first operation of a 128K training sequence
        _embed("embed_llama8b_128k", 131072, 4096, 128256, "forward", "zipf", 0.0, False),
        # a short batch on a small model: odd vocabulary and row count, padded documents
        _embed("embed_grad_3001_v50257", 3001, 1600, 50257, "backward", "zipf", 0.1, False),
        # the table's gradient of a 128K sequence, its rows as token frequencies in text have them: the commonest
        # token is an eighth of all
        _embed("embed_grad_llama8b_128k", 131072, 4096, 128256, "backward", "zipf", 0.0, False),
        # gradient accumulation over two micro-batches of packed documents, fp32 sums
        _embed("embed_grad_qwen32b_2x16k_accum", 32768, 5120, 152064, "accum", "zipf", 0.05, False),
        # the smallest norm call
        _norm("norm_tiny", 512, 256, "forward", True, "none", False, 0.0, 1.0),
        # between two blocks of a layer at 32K, norms before and after each block
        _norm("norm_llama8b_32k", 32768, 4096, "forward", True, "none", False, 0.0, 1.0),
        # backward of a ragged sequence with an fp32 residual stream and one gate a token, weights kept as 1 + w
        _norm("norm_grad_llama8b_6000", 6001, 4096, "backward", True, "token", True, 1.0, 0.5),
        # backward with a gate for each element, no norm after the block
        _norm("norm_grad_qwen32b_32k", 32768, 5120, "backward", False, "dense", False, 0.0, 0.7),
        # the largest: backward over the 256000 rows that one MLP call takes
        _norm("norm_grad_llama8b_256k", 256000, 4096, "backward", True, "none", False, 0.0, 1.0),
        # the gradients of the tiny workloads
        _grads("grads_tiny", "fused", 1, 256, 768, 4096, False, False, True),
        # five layers' MLP and norm gradients in bf16, the LM head's in fp32
        _grads("grads_llama8b_5_layers", "split", 5, 4096, 14336, 128256, True, False, True),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _extent(rng, lo, hi):
    """A hidden or intermediate size: usually a multiple of 64, now and then only of 8."""
    step = 8 if rng.random() < 0.3 else 64
    return max(step, int(_log_uniform(rng, lo, hi)) // step * step)


def draw(rng):
    largest = work(_norm("", 256000, 4096, "backward", True, "none", False, 0.0, 1.0))["bytes"]
    while True:
        op = rng.choice(["embed", "norm", "grads"])
        if op == "embed":
            V = int(_log_uniform(rng, 300, 200000))
            case = _embed("", int(_log_uniform(rng, 64, 300000)), _extent(rng, 64, 8192), V // 64 * 64 if rng.random() < 0.5 else V,
                          rng.choice(["forward", "backward", "backward", "accum"]), rng.choice(["zipf", "zipf", "uniform"]),
                          rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.4), 3)]), rng.random() < 0.3)
            if case["entry"] == "accum":
                case["fp32"] = False
        elif op == "norm":
            case = _norm("", int(_log_uniform(rng, 64, 300000)), _extent(rng, 64, 12288), rng.choice(["forward", "backward"]),
                         rng.random() < 0.6, rng.choice(["none", "none", "token", "dense"]), rng.random() < 0.4,
                         rng.choice([0.0, 1.0]), rng.choice([1.0, round(rng.uniform(0.1, 1.5), 3)]))
        else:
            case = _grads("", rng.choice(["fused", "split"]), rng.randint(1, 6), _extent(rng, 64, 6144), _extent(rng, 128, 16384),
                          int(_log_uniform(rng, 300, 160000)), rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.75)
        if work(case)["bytes"] <= largest:
            del case["name"]
            return case


# ---- what a user's program has in hand ----

def _token_law(case):
    V = case["V"]
    if case["law"] == "zipf":           # weights k^-1.1, id = rank - 1
        w = np.arange(1, V + 1, dtype=np.float64) ** -1.1
        return w / w.sum()
    return np.full(V, 1.0 / V)


def _tokens(case, N, g, seed, device):
    V = case["V"]
    if case["law"] == "zipf":
        cdf = torch.cumsum(torch.arange(1, V + 1, dtype=torch.float64, device=device) ** -1.1, 0)
        u = torch.rand(N, dtype=torch.float64, device=device, generator=g) * cdf[-1]
        t = torch.searchsorted(cdf, u).clamp_(max=V - 1).to(torch.int32)
    else:
        t = torch.randint(0, V, (N,), dtype=torch.int32, device=device, generator=g)
    if case["pad"]:                     # documents of 64..4096 tokens, the tail of each is padding
        rng, mask, pos = np.random.default_rng(seed), np.zeros(N, dtype=bool), 0
        while pos < N:
            end = min(N, pos + int(math.exp(rng.uniform(math.log(64), math.log(4096)))))
            mask[end - int(case["pad"] * (end - pos)):end] = True
            pos = end
        t[torch.from_numpy(mask).to(device)] = IGNORE
    return t


def _batches(case):
    N = case["N"]
    return [N - N // 2, N // 2] if case["entry"] == "accum" else [N]


def _gradient_sizes(case):
    """(elements, fp32) of each gradient: per layer the three of the MLP, two norm weights and a gate's bias of odd size; the LM
    head's comes last."""
    H, I = case["H"], case["I"]
    layer = [(I * H, False), (I * H, False), (H * I, False), (H, False), (H, case["fp32"]), (H // 3 * 2 + 1, False)]
    return layer * case["layers"] + [(case["V"] * H, case["fp32"])]


def _normal(shape, std, g, dtype=torch.bfloat16):
    t = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)
    return t if std == 1.0 else t.mul_(std)


def _stream(shape, g, dtype):
    """Rows of a residual stream: a few channels are many times as large as the others."""
    t = _normal(shape, 1.0, g, dtype)
    t[:, ::97] *= 20
    return t


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": dict(case)}
    rows = torch.float32 if case["fp32"] else torch.bfloat16
    if case["op"] == "embed":
        H, V = case["H"], case["V"]
        if case["entry"] == "forward":
            s["E"], s["scale"] = _normal((V, H), 0.02, g), math.sqrt(H)
            s["tokens"] = _tokens(case, case["N"], g, seed, "cuda")
        else:
            s["scale"] = math.sqrt(H)
            s["calls"] = [{"tokens": _tokens(case, n, g, seed + 1000 * k, "cuda"), "dy": _normal((n, H), 0.01, g, rows)}
                          for k, n in enumerate(_batches(case))]
        return s
    if case["op"] == "norm":
        N, H = case["N"], case["H"]
        s["residual"], s["branch"] = _stream((N, H), g, rows), _normal((N, H), 0.5, g)
        weight = lambda: _normal((H,), 0.1, g) if case["offset"] else (1 + _normal((H,), 0.1, g, torch.float32)).to(torch.bfloat16)  # noqa: E731
        s["w_pre"], s["w_post"] = weight(), weight() if case["post"] else None
        s["gate"] = {"none": None, "token": (N,), "dense": (N, H)}[case["gate"]]
        if s["gate"]:
            s["gate"] = _normal(s["gate"], 1.0, g)
        if case["entry"] == "backward":
            s["d_normed"], s["d_residual_out"] = _normal((N, H), 0.01, g), _normal((N, H), 0.01, g, rows)
        return s
    sizes = _gradient_sizes(case)
    std = [0.01 * (1 + k % 4) for k in range(len(sizes))]
    if case["flat"]:                    # views one behind the other in a flat buffer of each type
        of = {f: torch.empty(sum(n for n, q in sizes if q == f), dtype=torch.float32 if f else torch.bfloat16, device="cuda")
              for f in {q for _, q in sizes}}
        at, s["grads"] = {f: 0 for f in of}, []
        for (n, f), d in zip(sizes, std):
            s["grads"].append(of[f][at[f]:at[f] + n].normal_(generator=g).mul_(d))
            at[f] += n
    else:
        s["grads"] = [_normal((n,), d, g, torch.float32 if f else torch.bfloat16) for (n, f), d in zip(sizes, std)]
    expected = math.sqrt(sum(n * d * d for (n, _), d in zip(sizes, std)))
    s["max_norm"] = 0.3 * expected if case["clipped"] else 3.0 * expected
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:     # what a program keeps beside its tensors: the results' buffers, a workspace, the list of its gradients
        _buffers(s)
    return s


def _buffers(s):
    from paper_2506_13996_amd import binding as B
    case = s["case"]
    rows = torch.float32 if case["fp32"] else torch.bfloat16
    new = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if case["op"] == "embed":
        N, H, V = case["N"], case["H"], case["V"]
        if case["entry"] == "forward":
            s["y"] = new(N, H, dtype=rows)
        else:
            s["dE"] = new(V, H, dtype=torch.float32 if case["entry"] == "accum" else torch.bfloat16)
            s["workspace"] = B.alloc_embedding_workspace(max(_batches(case)), H, V)
    elif case["op"] == "norm":
        N, H = case["N"], case["H"]
        if case["entry"] == "forward":
            s["residual_out"], s["normed"] = new(N, H, dtype=rows), new(N, H)
        else:
            s["d_residual"], s["d_branch"], s["dw_pre"] = new(N, H, dtype=rows), new(N, H), new(H, dtype=torch.float32)
            s["dw_post"] = new(H, dtype=torch.float32) if case["post"] else None
            s["d_gate"] = None if s["gate"] is None else torch.empty_like(s["gate"])
            s["workspace"] = B.alloc_block_norm_workspace(N, H)
    else:
        if case["flat"]:
            at, s["outs"] = {}, []
            for t in s["grads"]:
                if t.dtype not in at:
                    at[t.dtype] = torch.empty(t.untyped_storage().nbytes() // t.element_size(), dtype=t.dtype, device="cuda")
                o = t.storage_offset()
                s["outs"].append(at[t.dtype][o:o + t.numel()])
        else:
            s["outs"] = [torch.empty_like(t) for t in s["grads"]]
        s["handle"] = B.GradTensors(s["grads"], s["outs"])
        s["norm"], s["sumsq"] = new(1, dtype=torch.float32), new(1, dtype=torch.float64)
        s["workspace"] = B.alloc_grad_norm_workspace(s["handle"])


# ---- the plain forms ----

def _plain_embed(s):
    case, scale = s["case"], s["scale"]
    rows = torch.float32 if case["fp32"] else torch.bfloat16
    if case["entry"] == "forward":
        t = s["tokens"]
        keep = t != IGNORE
        y = s["E"][torch.where(keep, t, 0).long()].float() * scale
        return [(y * keep[:, None]).to(rows)]
    dE = torch.zeros(case["V"], case["H"], dtype=torch.float32, device="cuda")
    for c in s["calls"]:
        keep = c["tokens"] != IGNORE
        dE.index_add_(0, c["tokens"][keep].long(), c["dy"][keep].float())
    dE *= scale
    return [dE if case["entry"] == "accum" else dE.to(torch.bfloat16)]


def _rms(x):
    return torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)


def _gate(s):
    z = s["gate"].float()
    return torch.sigmoid(z[:, None] if z.dim() == 1 else z)


def _plain_norm(s):
    case = s["case"]
    rows, scale, offset = torch.float32 if case["fp32"] else torch.bfloat16, case["scale"], case["offset"]
    w2 = s["w_pre"].float() + offset
    b = s["branch"].float()
    w1 = s["w_post"].float() + offset if case["post"] else None
    if case["entry"] == "forward":
        p = b * _rms(b) * w1 if case["post"] else b
        if s["gate"] is not None:
            p = p * _gate(s)
        r = s["residual"].float() + scale * p
        return [r.to(rows), (r * _rms(r) * w2).to(torch.bfloat16)]
    r, dn = s["residual"].float(), s["d_normed"].float()        # (backward: the rows that forward wrote)
    q2 = _rms(r)
    x2 = r * q2
    u = dn * w2
    dw2 = (dn * x2).sum(0)
    dr = s["d_residual_out"].float() + q2 * (u - x2 * (u * x2).mean(1, keepdim=True))
    out = {"d_residual": dr.to(rows), "dw_pre": dw2}
    del u, x2
    dp = scale * dr
    q1 = _rms(b) if case["post"] else None
    x1 = b * q1 if case["post"] else b
    if s["gate"] is not None:
        g = _gate(s)
        dz = dp * (x1 * w1 if case["post"] else x1) * g * (1 - g)
        out["d_gate"] = (dz if case["gate"] == "dense" else dz.sum(1)).to(torch.bfloat16)
        dp = dp * g
    if case["post"]:
        out["dw_post"] = (dp * x1).sum(0)
        u = dp * w1
        dp = q1 * (u - x1 * (u * x1).mean(1, keepdim=True))
    out["d_branch"] = dp.to(torch.bfloat16)
    return out


def _plain_grads(s):
    sumsq = torch.stack([g.double().square().sum() for g in s["grads"]]).sum()      # (a long sum: in 64 bits)
    norm = sumsq.sqrt()
    c = torch.clamp(s["max_norm"] / norm, max=1.0).float()
    return {"norm": norm.float().reshape(1), "sumsq": sumsq.reshape(1), "outs": [(g.float() * c).to(g.dtype) for g in s["grads"]]}


# ---- the calls ----

def _own_embed(s):
    from paper_2506_13996_amd import binding as B
    case, scale = s["case"], s["scale"]
    flags = B.ALST_FLAG_RESIDUAL_FP32 if case["fp32"] else 0
    if case["entry"] == "forward":
        B.alst_embedding_forward(s["tokens"], s["E"], scale, IGNORE, y=s["y"], flags=flags)
        return [s["y"]]
    for k, c in enumerate(s["calls"]):
        if case["entry"] == "accum":
            flags = B.ALST_FLAG_DW_FP32 | (B.ALST_FLAG_DW_ACCUMULATE if k else 0)
        B.alst_embedding_backward(c["tokens"], c["dy"], scale, IGNORE, dE=s["dE"], workspace=s["workspace"], flags=flags)
    return [s["dE"]]


def _own_norm(s):
    from paper_2506_13996_amd import binding as B
    case = s["case"]
    flags = B.ALST_FLAG_RESIDUAL_FP32 if case["fp32"] else 0
    parts = dict(branch=s["branch"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"], branch_scale=case["scale"], eps=EPS,
                 weight_offset=case["offset"])
    if case["entry"] == "forward":
        B.alst_block_norm_forward(s["residual"], **parts, residual_out=s["residual_out"], normed=s["normed"], flags=flags)
        return [s["residual_out"], s["normed"]]
    B.alst_block_norm_backward(s["residual"], **parts, d_normed=s["d_normed"], d_residual_out=s["d_residual_out"],
                               d_residual=s["d_residual"], d_branch=s["d_branch"], d_gate=s["d_gate"], dw_post=s["dw_post"],
                               dw_pre=s["dw_pre"], workspace=s["workspace"], flags=flags | B.ALST_FLAG_DW_FP32)
    return {k: s[k] for k in ("d_residual", "dw_pre", "d_gate", "dw_post", "d_branch") if s[k] is not None}


def _own_grads(s):
    from paper_2506_13996_amd import binding as B
    if s["case"]["entry"] == "fused":
        B.alst_grad_norm_clip(s["handle"], s["max_norm"], norm_out=s["norm"], sumsq_out=s["sumsq"], workspace=s["workspace"])
    else:
        B.alst_grad_norm(s["handle"], sumsq_out=s["sumsq"], norm_out=s["norm"], workspace=s["workspace"])
        B.alst_grad_clip(s["handle"], s["sumsq"], s["max_norm"])
    return {"norm": s["norm"], "sumsq": s["sumsq"], "outs": s["outs"]}


def run(s):
    op = s["case"]["op"]
    if own:
        return {"embed": _own_embed, "norm": _own_norm, "grads": _own_grads}[op](s)
    return {"embed": _plain_embed, "norm": _plain_norm, "grads": _plain_grads}[op](s)


# ---- the definitions, in 64 bits ----

def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "embed":
        V, H, scale = case["V"], case["H"], s["scale"]
        if case["entry"] == "forward":
            y = torch.zeros(case["N"], H, dtype=torch.float64, device="cuda")
            at = torch.nonzero(s["tokens"] != IGNORE).flatten()
            y[at] = scale * torch.index_select(s["E"].double(), 0, s["tokens"][at].long())
            return [y]
        t = torch.cat([c["tokens"] for c in s["calls"]]).long()
        dy = torch.cat([c["dy"] for c in s["calls"]])
        at = torch.nonzero(t != IGNORE).flatten()
        order = at[torch.argsort(t[at], stable=True)]
        counts = torch.bincount(t[at], minlength=V)
        dE = torch.empty(V, H, dtype=torch.float64, device="cuda")
        for h in range(0, H, 512):      # (a sum of each token's run of sorted rows)
            run_sums = torch.segment_reduce(dy[order, h:h + 512].double(), "sum", lengths=counts, axis=0, initial=0.0)
            dE[:, h:h + 512] = scale * run_sums
        return [dE]
    if case["op"] == "norm":
        return _exact_norm(case, s)
    total = math.fsum(float((g.double() ** 2).sum()) for g in s["grads"])
    c = min(1.0, s["max_norm"] / math.sqrt(total))
    one = lambda v: torch.tensor([v], dtype=torch.float64)  # noqa: E731
    return {"norm": one(math.sqrt(total)), "sumsq": one(total), "outs": [g.double() * c for g in s["grads"]]}


def _exact_norm(case, s):
    """Forward from the definition, gradients by differentiating it, a block of rows at a time."""
    N, H, keys = case["N"], case["H"], [k for k in ("w_pre", "w_post") if s[k] is not None]
    W = {k: s[k].double().requires_grad_() for k in keys}
    norm = lambda x, w: x / torch.sqrt(torch.mean(x ** 2, dim=1, keepdim=True) + EPS) * (w + case["offset"])  # noqa: E731
    step = max(1, (1 << 27) // H)
    parts = []
    for i in range(0, N, step):
        rows = slice(i, i + step)
        branch = s["branch"][rows].double().requires_grad_()
        gate = None if s["gate"] is None else s["gate"][rows].double().requires_grad_()
        change = norm(branch, W["w_post"]) if case["post"] else branch
        if gate is not None:
            change = change / (1 + torch.exp(-(gate if gate.dim() == 2 else gate.unsqueeze(1))))
        change = case["scale"] * change
        if case["entry"] == "forward":
            r = s["residual"][rows].double() + change
            parts.append([r.detach(), norm(r, W["w_pre"]).detach()])
            continue
        # the stream's value is given; r' = (r' - change) + change has its gradients
        before = (s["residual"][rows].double() - change.detach()).requires_grad_()
        r = before + change
        out = (norm(r, W["w_pre"]) * s["d_normed"][rows].double()).sum() + (r * s["d_residual_out"][rows].double()).sum()
        out.backward()
        parts.append([before.grad, branch.grad] + ([] if gate is None else [gate.grad]))
    whole = [torch.cat(p) for p in zip(*parts)]
    if case["entry"] == "forward":
        return whole
    names = ["d_residual", "d_branch"] + ([] if s["gate"] is None else ["d_gate"])
    return {**dict(zip(names, whole)), **{"d" + k: W[k].grad for k in keys}}


def work(case):
    """Each input once, each output once.  Of the table, the rows that the batch names (their expected number)."""
    if case["op"] == "embed":
        H, V, p = case["H"], case["V"], _token_law(case)
        keep, rows = 1.0 - case["pad"], 4 if case["fp32"] else 2
        if case["entry"] == "forward":
            N = case["N"]
            named = float((1 - (1 - p) ** (keep * N)).sum())
            return {"bytes": 4 * N + 2 * named * H + rows * N * H, "flops": keep * N * H}
        out, total = 4 if case["entry"] == "accum" else 2, 0.0
        for k, n in enumerate(_batches(case)):
            named = float((1 - (1 - p) ** (keep * n)).sum())
            total += 4 * n + rows * keep * n * H + (out * V * H if k == 0 else 2 * out * named * H)
        return {"bytes": total, "flops": (keep * case["N"] + V) * H}
    if case["op"] == "norm":
        N, H, rows = case["N"], case["H"], 4 if case["fp32"] else 2
        gate = {"none": 0, "token": 2 * N, "dense": 2 * N * H}[case["gate"]]
        weights = 2 * H * (2 if case["post"] else 1)
        if case["entry"] == "forward":
            return {"bytes": (2 * rows + 4) * N * H + gate + weights, "flops": (12 if case["post"] else 7) * N * H}
        # (without a norm or a gate after the block, its gradient needs nothing of the block's output)
        branch = 2 * N * H if case["post"] or case["gate"] != "none" else 0
        return {"bytes": (3 * rows + 4) * N * H + branch + 2 * gate + 3 * weights, "flops": (30 if case["post"] else 15) * N * H}
    sizes = _gradient_sizes(case)
    total = sum(n * (4 if f else 2) for n, f in sizes)
    # norm: all once; outputs: all once more, from what is read again, as no cache of this card holds a model's gradients
    return {"bytes": 3 * total, "flops": 3 * sum(n for n, _ in sizes)}
