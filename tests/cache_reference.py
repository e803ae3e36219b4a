"""Plain forms in 64 bits (numpy, one row at a time) of the operators around a
rollout's cache and its logits, and the tolerances that the kernels are held to.

* attention weights: a score is a sum of D exact products in 32 bits, each step
  off by a unit in the last place at most (2^-23): D 2^-23 scale sum |q k|; the
  difference to lse, its product with log2 e and the exponential's argument are
  rounded once each: 2^-23 |s - lse| more, and 2^-22 for the exponential itself.
  All are relative errors of a weight.  Sums of R weights, in 32 bits in any
  order: R 2^-24 of their sum; the decayed mass and the last sum: 2^-23 of each.
  Weights below 2^-126 may be zeros.
* eviction: slots, lengths, masses and rows are equal, bit for bit.
* controls: a quotient or product, a product and two differences, a sum, each
  rounded in 32 bits (2^-24 of the sizes of their terms; five of them), then one
  rounding to the type, u |y|.
"""
from __future__ import annotations

import numpy as np


def mass(old, q, lse, K, ctx, sees, scale, decay):
    """One sequence and kv head: old [>= L] masses, q [n, G, D], lse [n, G], K [L, D] of its slots, sees [n, L] bool.
    Returns the masses of the L slots and their tolerances."""
    n, G, D = q.shape
    L = len(K)
    w, tol = np.zeros(L), np.zeros(L)
    for i in range(n):
        for g in range(G):
            if lse[i, g] == -np.inf:
                continue
            j = np.flatnonzero(sees[i])
            s = K[j] @ q[i, g] * scale
            e = np.exp(s - lse[i, g])
            off = D * 2.0 ** -23 * scale * (np.abs(K[j]) @ np.abs(q[i, g])) + 2.0 ** -23 * np.abs(s - lse[i, g]) + 2.0 ** -22
            w[j] += e
            tol[j] += e * np.expm1(off) + 2.0 ** -126
    tol += n * G * 2.0 ** -24 * w
    got = w.copy()
    if decay:
        got[:ctx] += decay * old[:ctx]
        tol[:ctx] += 2.0 ** -23 * (np.abs(decay * old[:ctx]) + w[:ctx])
    return got, tol


def remaining(m, n, budget, sink, recent):
    """The slots of a sequence of n that remain, in order; m [>= n] masses."""
    k = min(n, budget)
    a = min(k, sink)
    z = min(k - a, recent)
    between = np.arange(a, n - z)
    with np.errstate(invalid="ignore"):
        value = np.where(np.isnan(m[between]), -np.inf, m[between].astype(np.float64))
    nan = np.isnan(m[between])
    order = np.lexsort((between, nan, -value))  # falling, NaN after -inf, then the lower slot
    return np.sort(np.concatenate([np.arange(a), between[order[:k - a - z]], np.arange(n - z, n)]))


def controls(x, history, prompt, rep, freq, pres, biases, allowed):
    """One row: x [V] in 64 bits, biases a list of (token, value), allowed [V] bool or None.  Returns y and the sizes that
    its roundings are of."""
    V, y = len(x), x.copy()
    history = np.asarray(history, np.int64)
    for t in {int(t) for t in history if 0 <= t < V}:
        y[t] = y[t] / rep if y[t] > 0 else y[t] * rep
    size = np.abs(y)
    made = history[prompt:]
    tokens, times = np.unique(made[(made >= 0) & (made < V)], return_counts=True)
    y[tokens] -= freq * times + pres
    size[tokens] += np.abs(freq) * times + np.abs(pres)
    last = {int(t): v for t, v in biases if 0 <= t < V}
    for t, v in last.items():
        y[t] += v
        size[t] += abs(v)
    if allowed is not None:
        y[~allowed] = -np.inf
        size[~allowed] = 0
    return y, size
