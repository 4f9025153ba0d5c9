"""Plain 64-bit forms of drawing, distillation and embedding rows, with the
error bounds that the GPU tests hold the kernels to.

A float32 rounding is off by at most U32 = 2^-24 of the value, a bfloat16 one
by at most U16 = 2^-8 of it."""

from __future__ import annotations

import numpy as np

U32, U16 = 2.0 ** -24, 2.0 ** -8


def weights(x, T):
    """exp((x - max) / T) of a row, 0 for NaN and -inf; None if nothing is left."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    best = x.max()
    if best == -np.inf:
        return None
    if best == np.inf:
        return (x == np.inf).astype(np.float64)
    return np.exp((x - best) / T)


def kept(x, T=1.0, k=0, p=1.0, m=0.0):
    """(weights of the entities that the settings keep, the smallest distance
    of a running weight from the border of top-p, relative to the total)."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    w = None if not (np.isfinite(T) and T >= 0 and k >= 0 and p > 0 and 0 <= m <= 1) else weights(x, T or 1.0)
    if w is None:
        return None, 1.0
    order = np.lexsort((np.arange(x.size), -x))       # score descending, index ascending
    if T == 0:
        order, k, p = order[:1], 0, 1.0
    if 0 < k < order.size:
        order = order[:k]
    margin = 1.0
    if p < 1.0:
        run = np.cumsum(w[order])
        n = int((run < p * run[-1]).sum()) + 1
        margin = np.abs(run - p * run[-1]).min() / run[-1]
        order = order[:n]
    out = np.zeros_like(w)
    out[order] = w[order]
    if T == 0:
        out[order] = 1.0
    out[out < m] = 0.0
    return out, margin


def check_draws(idx, logp, x, u, what, **settings):
    """Draws idx [S] of a row against the definition. A draw whose u lies
    within 1e-12 of the border between two entities may be either one's."""
    w, margin = kept(x, **settings)
    if w is None:
        assert (idx == -1).all(), f"{what}: {idx}"
        assert logp is None or np.isnan(logp).all(), what
        return
    assert margin > 1e-12 or settings.get("p", 1.0) >= 1.0 or margin == 0.0, f"{what}: choose other inputs"
    run = np.cumsum(w)
    z = run[-1]
    last = int(np.nonzero(w)[0][-1])
    t = np.where(u >= 0, np.minimum(u.astype(np.float64), 1.0), 0.0) * z
    ref = np.minimum(np.searchsorted(run, t, side="right"), last)
    for s in np.nonzero(ref != idx)[0]:
        i = int(idx[s])
        assert 0 <= i < x.size and w[i] > 0, f"{what} draw {s}: {i} is not kept (expected {ref[s]})"
        assert run[i] - w[i] - 1e-12 * z <= t[s] <= run[i] + 1e-12 * z, f"{what} draw {s}: {i}, expected {ref[s]}"
    if logp is not None:
        want = np.log(w[idx] / z)
        # doubles, rounded to float32 once
        bad = np.abs(logp - want) > U32 * np.abs(want) + 1e-12
        assert not bad.any(), f"{what}: log-probabilities {logp[bad]} against {want[bad]}"


def distill(z, idx, t, tau, w):
    """(loss [B], gradient [B x N], bound of the loss, bound of the gradient).

    The bounds: an exponential's argument is off by U32 |z - max| / tau (the
    difference's rounding) and by up to 4 U32 (its reduction and the
    hardware's exponential); a float32 sum of N positive terms in threads of
    at most N / 64 terms each by U32 N / 64 + 8 U32; the rest is doubles; the
    gradient is rounded to float32 twice (its factor and the product)."""
    B, N = z.shape
    loss, grad = np.zeros(B), np.zeros((B, N))
    lb, gb = np.zeros(B), np.zeros((B, N))
    for b in range(B):
        on = (idx[b] >= 0) & (idx[b] < N) & ~(t[b] == -np.inf)
        if not on.any():
            continue
        x, a, tt = z[b].astype(np.float64), idx[b][on], t[b][on].astype(np.float64)
        if np.isnan(tt).any() or np.isnan(x).any() or x.max() in (np.inf, -np.inf):
            loss[b] = np.nan
            grad[b] = np.nan if w[b] != 0 else 0.0
            continue
        p = (tt == np.inf).astype(np.float64) if tt.max() == np.inf else np.exp((tt - tt.max()) / tau)
        p /= p.sum()
        d = (x - x.max()) / tau
        e = np.exp(d)
        q = e / e.sum()
        with np.errstate(divide="ignore"):
            logq = d - np.log(e.sum())
        s = p > 0
        loss[b] = tau * tau * (p[s] * (np.log(p[s]) - logq[a[s]])).sum()
        if loss[b] >= 2.0 ** 128 * (1 - 2.0 ** -25):      # what rounds to float32's infinity
            loss[b] = np.inf
        g = q.copy()
        np.add.at(g, a, -p)
        finite = np.where(e > 0, np.abs(np.where(e > 0, d, 0.0)), 0.0)
        each = U32 * (finite + 4.0)
        total = (q * each).sum() + U32 * (N / 64 + 8.0)
        lb[b] = tau * tau * total + (2 * U32 * abs(loss[b]) if np.isfinite(loss[b]) else 0.0) + 1e-12
        grad[b] = w[b] * tau * g
        gb[b] = abs(w[b]) * tau * (q * (each + total + 4 * U32) + 2 * U32 * np.abs(g) + 1e-15) + 1e-37
        if w[b] == 0:
            grad[b] = 0.0
    return loss, grad, lb, gb


def embed_grad(g, ids, V, scale, base=None):
    """(gradient [V x d], bound): a float32 sum of the n tokens of an id is off
    by at most n U32 times the sum of their magnitudes, then a product and, with
    a base, an addition."""
    g = np.asarray(g, np.float64)
    out, mag = np.zeros((V, g.shape[1])), np.zeros((V, g.shape[1]))
    on = (ids >= 0) & (ids < V)
    np.add.at(out, ids[on], g[on])
    np.add.at(mag, ids[on], np.abs(g[on]))
    n = np.bincount(ids[on], minlength=V)[:, None]
    bound = U32 * (n + 2) * mag * abs(scale)
    out = out * scale
    if base is not None:
        out = out + base
        bound = bound + U32 * (np.abs(out) + bound)
    return out, bound
