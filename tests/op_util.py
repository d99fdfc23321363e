"""Contexts and 64-bit reference forms for the operators on the caller's tensors (distillation loss,
sampling, q/k norms): written from the definitions in include/alr.h, one row at a time."""
from __future__ import annotations

import math

import numpy as np

from paper_2609_38795_amd import binding, workloads as W

EPS = 1e-6
BASE = 10000.0


def engine(dtype="f32", q_heads=1, k_heads=1, hd=64, max_pos=8, sections=(0, 0, 0), stream=None):
    """A context without layers: head shape, dtype and rotation are what the operators read."""
    import torch

    shape = W.ModelShape(0, 64, q_heads, k_heads, hd, 64, 64, EPS, BASE, dtype, (),
                         mrope_sections=sections)
    z = np.zeros((64, 64), np.uint16 if dtype == "bf16" else np.float32)
    w = {"tok_embed": z, "lm_head": z, "final_norm": z[0], "layers": []}
    return binding.Engine(shape, w, max_pos, binding.make_limits(1, 1, 1, 1),
                          device=torch.device("cuda:0"), stream=stream)


def distill_ref(z, ids, logp, tail, w, scale, up=1.0):
    """(loss, W, row losses, gradients) in float64; z [n, V] float64 (exact values of the inputs)."""
    n, V = z.shape
    rows, grads = np.zeros(n), np.zeros_like(z)
    Wsum = float(np.sum(w.astype(np.float64)))
    for r in range(n):
        if w[r] == 0:
            continue
        m = z[r].max()
        e = np.exp(z[r] - m)
        q = e / e.sum()
        outside = np.ones(V, bool)
        pis = []
        for j in range(ids.shape[1]):
            if 0 <= ids[r, j] < V:
                outside[ids[r, j]] = False
                pis.append((int(ids[r, j]), math.exp(float(logp[r, j]))))
        P = sum(p for _, p in pis) + float(tail[r])
        logq = z[r] - m - math.log(e.sum())
        loss = -sum(p * logq[i] for i, p in pis if p > 0)
        t = z[r][outside]
        tm = t.max() if t.size else -np.inf
        cond = np.zeros(V)
        if tm > -np.inf:
            et = np.exp(t - tm)
            cond[outside] = et / et.sum()
            lt = tm - m + math.log(et.sum()) - math.log(e.sum())
        else:
            lt = -np.inf
        if tail[r] > 0:
            loss -= float(tail[r]) * lt
        g = P * q - float(tail[r]) * cond
        for i, p in pis:
            g[i] -= p
        rows[r] = loss
        grads[r] = g * (up * scale * float(w[r]) / Wsum if Wsum != 0 else 0.0)
    loss = scale * float(np.dot(w.astype(np.float64), rows)) / Wsum if Wsum != 0 else 0.0
    return loss, Wsum, rows, grads


def sample_ref(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-prob) of one row by a full sort, in float64."""
    z = np.where(np.isnan(z), -np.inf, z.astype(np.float64))
    u = min(max(float(np.float32(u)), 0.0), 1 - 2.0 ** -24)
    V = z.size
    m = z.max()
    if m == -np.inf:
        return -1, -np.inf
    if not temperature > 0 or m == np.inf:
        return int(np.argmax(z)), 0.0
    order = np.lexsort((np.arange(V), -z))
    order = order[z[order] > -np.inf]  # weight 0: never drawn
    with np.errstate(over="ignore"):
        w = np.exp((z[order] - m) / float(np.float32(temperature)))
    n = len(order)
    if 0 < top_k < V:
        n = min(n, top_k)
    if top_p < 1:
        before = np.concatenate(([0.0], np.cumsum(w[:n])[:-1]))
        k = before < float(np.float32(top_p)) * np.sum(w[:n])
        k[0] = True
        n = int(k.sum())
    if min_p > 0:
        n = min(n, max(1, int((w >= min(float(np.float32(min_p)), 1.0)).sum())))
    by_id = np.argsort(order[:n])
    ids, w = order[:n][by_id], w[:n][by_id]
    c = np.cumsum(w)
    j = min(int(np.searchsorted(c, u * c[-1], side="right")), n - 1)
    with np.errstate(divide="ignore"):
        return int(ids[j]), float(np.log(w[j] / c[-1]))


def angles(pos, hd, sections):
    """cos, sin [n, half] of positions [n, 3] in float64."""
    half = hd // 2
    axis = np.zeros(half, int) if sum(sections) == 0 else np.repeat(np.arange(3), sections)
    a = pos[:, axis].astype(np.float64) * BASE ** (-2.0 * np.arange(half) / hd)
    return np.cos(a), np.sin(a)


def qk_ref(x, g, pos, sections):
    """Forward of x [n, heads, hd] in float64."""
    hd = x.shape[2]
    half = hd // 2
    c, s = (t[:, None, :] for t in angles(pos, hd, sections))
    y = x / np.sqrt(np.mean(x * x, axis=2, keepdims=True) + EPS) * g
    lo, hi = y[..., :half], y[..., half:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], 2)


def qk_back_ref(x, g, pos, sections, dy):
    """(dx, dg, sum of |terms of dg|) in float64."""
    hd = x.shape[2]
    half = hd // 2
    c, s = (t[:, None, :] for t in angles(pos, hd, sections))
    lo, hi = dy[..., :half], dy[..., half:]
    d = np.concatenate([lo * c + hi * s, hi * c - lo * s], 2)
    r = 1 / np.sqrt(np.mean(x * x, axis=2, keepdims=True) + EPS)
    xh = x * r
    dx = r * (g * d - xh * np.mean(g * d * xh, axis=2, keepdims=True))
    return dx, np.sum(d * xh, (0, 1)), np.sum(np.abs(d * xh), (0, 1))
