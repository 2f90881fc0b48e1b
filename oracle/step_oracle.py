"""The operators around the tiled layers in 64 bits (numpy), with the magnitudes that rounding errors are relative to.

Definitions: token embedding and its table's gradient, the norms around a block with gate and scaled residual, the global
gradient norm and clipping, as include/alst_embedding.h, alst_block_norm.h and alst_grads.h state them.
"""
from __future__ import annotations

import numpy as np


def embedding_forward(tokens, E, scale, ignore_index):
    V = E.shape[0]
    keep = (tokens >= 0) & (tokens < V) & (tokens != ignore_index)
    y = np.zeros((len(tokens), E.shape[1]))
    y[keep] = scale * E[tokens[keep]]
    return y


def embedding_backward(tokens, dy, scale, ignore_index, V):
    """(dE, sum of |scale dy| over a token's rows, rows of each token)."""
    keep = (tokens >= 0) & (tokens < V) & (tokens != ignore_index)
    dE, mag = np.zeros((V, dy.shape[1])), np.zeros((V, dy.shape[1]))
    np.add.at(dE, tokens[keep], scale * dy[keep])
    np.add.at(mag, tokens[keep], np.abs(scale * dy[keep]))
    return dE, mag, np.bincount(tokens[keep], minlength=V)


def sigmoid(z):
    t = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, t) / (1.0 + t)


def _q(x, eps):
    return 1.0 / np.sqrt(np.mean(x * x, axis=1, keepdims=True) + eps)


def _gate(gate, sign=1.0):
    return 1.0 if gate is None else sigmoid(sign * (gate if gate.ndim == 2 else gate[:, None]))


def block_norm_forward(r, b=None, w_post=None, gate=None, w_pre=None, scale=1.0, eps=1e-6, offset=0.0):
    """{"residual_out", "normed"} and their magnitudes under "mag_..."."""
    out, mag = r, np.abs(r)
    if b is not None:
        p = b if w_post is None else b * _q(b, eps) * (w_post + offset)
        change = scale * _gate(gate) * p
        out, mag = r + change, mag + np.abs(change)
    res = {"residual_out": out, "mag_residual_out": mag}
    if w_pre is not None:
        q = _q(out, eps)
        res["normed"], res["mag_normed"] = out * q * (w_pre + offset), mag * q * np.abs(w_pre + offset)
    return res


def block_norm_backward(r, b=None, w_post=None, gate=None, w_pre=None, d_normed=None, d_residual_out=None, scale=1.0,
                        eps=1e-6, offset=0.0, branch=True):
    """Gradients from r = r' as stored, by the formulas; "mag_..." as above."""
    mean = lambda v: np.mean(v, axis=1, keepdims=True)  # noqa: E731
    up = np.zeros_like(d_normed) if d_residual_out is None else d_residual_out
    dr, mag = up.copy(), np.abs(up)
    res = {}
    if w_pre is not None:
        q = _q(r, eps)
        x, u = r * q, d_normed * (w_pre + offset)
        dr = dr + q * (u - x * mean(u * x))
        mag = mag + q * (np.abs(u) + np.abs(x) * mean(np.abs(u * x)))
        res["dw_pre"], res["mag_dw_pre"] = (d_normed * x).sum(0), np.abs(d_normed * x).sum(0)
    res["d_residual"], res["mag_d_residual"] = dr, mag
    if not branch:
        return res
    g = _gate(gate)
    dp, mp = scale * g * dr, np.abs(scale) * g * mag
    w = 1.0 if w_post is None else w_post + offset
    q = 1.0 if w_post is None else _q(b, eps)
    if gate is not None:
        rest = _gate(gate, -1.0)         # 1 - sigmoid
        dz, mz = dp * rest * q * w * b, mp * rest * np.abs(q * w * b)
        res["d_gate"], res["mag_d_gate"] = (dz, mz) if gate.ndim == 2 else (dz.sum(1), mz.sum(1))
    if w_post is not None:
        x, u, mu = b * q, dp * w, mp * np.abs(w)
        res["dw_post"], res["mag_dw_post"] = (dp * x).sum(0), (mp * np.abs(x)).sum(0)
        dp, mp = q * (u - x * mean(u * x)), q * (mu + np.abs(x) * mean(mu * np.abs(x)))
    res["d_branch"], res["mag_d_branch"] = dp, mp
    return res


def grad_norm_clip(grads, max_norm):
    """(sum of squares, norm, clipped gradients)."""
    total = float(sum(np.sum(np.square(g, dtype=np.float64)) for g in grads))
    norm = np.sqrt(total)
    c = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return total, norm, [g * c for g in grads]
