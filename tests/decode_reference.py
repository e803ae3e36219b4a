"""Plain forms in 64 bits of the decode step's operators (numpy, one row at a
time), and the tolerances that the kernels are held to.

Tolerances, from the types' roundings (u = 2^-8 bf16, 2^-11 f16: half a unit
in the last place, relative; f32: 2^-24):
* norm and rotation: 32-bit arithmetic of at most D + 20 roundings on values
  whose sizes are bounded by the row's (|a| + |b| per rotated pair), then one
  rounding: u |y| + (D + 20) 2^-24 (|a| + |b|);
* their weight gradients: sums of n = tokens * heads terms in 32 bits in a
  fixed tree: 2^-24 (D + 40 + sqrt(n)) sum |terms|;
* attention: weights p rounded to the type before the second product, u sum p |v|,
  one output rounding, u |o|, and 32-bit sums and exponentials: 2e-6 (sum p |v|)
  times the number of score roundings that an exponent of up to 30 amplifies (8);
  lse: D 2^-24 times the largest sum |q k| scale, plus 4e-6;
* sampled tokens: equal, unless the two best ratios agree within 1e-5 or a
  token's membership turns on a mass within 1e-5 of top_p, where either side's
  token is right; logp: 2e-5 absolute.
"""
from __future__ import annotations

import numpy as np

UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def torch_dtype(name):
    import torch

    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


def f64(t):
    return t.detach().double().cpu().numpy()


def pairs(D, R, interleaved):
    """(first, second) component of each rotated pair."""
    h = R // 2
    return (np.arange(0, R, 2), np.arange(1, R, 2)) if interleaved else (np.arange(h), h + np.arange(h))


def norm_rope(x, w, eps, cos, sin, interleaved):
    """x [N, H, D]; cos, sin [N, R/2] (of each token) or None.  Returns y and
    the size |a| + |b| that bounds each component's rounding errors."""
    u = x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    y, size = u.copy(), np.abs(u)
    if cos is not None:
        i, j = pairs(x.shape[-1], 2 * cos.shape[-1], interleaved)
        c, s = cos[:, None], sin[:, None]
        y[..., i], y[..., j] = u[..., i] * c - u[..., j] * s, u[..., i] * s + u[..., j] * c
        size[..., i] = size[..., j] = np.abs(u[..., i]) + np.abs(u[..., j])
    return y, size


def norm_rope_backward(dy, x, w, eps, cos, sin, interleaved):
    """dx, dw (None without weight), the size of dx's terms and of dw's."""
    du, size = norm_rope(dy, None, eps, cos, None if sin is None else -sin, interleaved)
    if w is None:
        return du, None, size, None
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n, g = x * r, du * w
    dx = r * (g - n * (g * n).mean(-1, keepdims=True))
    size = r * (size * np.abs(w) + np.abs(n) * (size * np.abs(w) * np.abs(n)).mean(-1, keepdims=True))
    return dx, (du * n).sum((0, 1)), size, np.abs(du * n).sum((0, 1))


def attention(q, K, V, seen, scale):
    """q [D], K, V [L, D] of the slots, seen bool [L]: out, lse, sum p |v|."""
    if not seen.any():
        return np.zeros(V.shape[1]), -np.inf, np.zeros(V.shape[1])
    s = K[seen] @ q * scale
    p = np.exp(s - s.max())
    l = p.sum()  # noqa: E741
    return p @ V[seen] / l, s.max() + np.log(l), p @ np.abs(V[seen]) / l


def sample(x, noise, T, top_k, top_p, min_p, p_slack=0.0):
    """One row: (acceptable tokens, the token, its log-probability); (.., -1, nan) where there is none."""
    V = len(x)
    if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any() or not (T >= 0) or T == np.inf \
            or np.isnan(top_p) or np.isnan(min_p):
        return {-1}, -1, np.nan
    order = np.lexsort((np.arange(V), -x))
    if T == 0:
        return {int(order[0])}, int(order[0]), 0.0
    with np.errstate(over="ignore"):
        d = (x - x.max()) / T
    kept = [i for i in order if x[i] > -np.inf]
    if 0 < top_k < V:
        kept = kept[:top_k]
    w = np.exp(d)
    if top_p < 1:
        mass = np.cumsum(w[kept])
        n = int((mass - w[kept] < (top_p + p_slack) * mass[-1]).sum())
        kept = kept[:max(1, n)]
    kept = np.array([i for i in kept if w[i] >= min(min_p, 1)])
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        ratio = w[kept] / noise[kept]
    ratio = np.where(np.isnan(ratio), -1.0, ratio)
    if not (ratio > 0).any():
        return {-1}, -1, np.nan
    best = ratio.max()
    token = int(kept[ratio == best].min())
    near = {int(i) for i in kept[ratio >= best * (1 - 1e-5)]} if np.isfinite(best) else {token}
    return near, token, d[token] - np.log(w[kept].sum())


def acceptable(x, noise, T, top_k, top_p, min_p):
    """All tokens that one of top_p - 1e-5, top_p, top_p + 1e-5 makes right."""
    got = set()
    for slack in (-1e-5, 0.0, 1e-5) if top_p < 1 else (0.0,):
        got |= sample(x, noise, T, top_k, top_p, min_p, slack)[0]
    return got
