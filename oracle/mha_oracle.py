"""Definitions in 64 bits of the attention branch's operators: rotary positions with several axes, attention over
sequences and windows of frames with its row sums, and its gradients.  numpy, one row or one sequence at a time, written
from the formulas; nothing here is shared with the kernels.

``forward`` and ``backward`` also give, beside each result, the sizes of the terms that it is a sum of: what an error of
a share u in the factors of those terms can come to is u times them, so tests state tolerances by arithmetic."""

from __future__ import annotations

import numpy as np


def rope(x, heads, axes, positions, theta=10000.0, halves=False, first_rows=0, backward=False):
    """x [rows, heads * d]; positions [rows, axes]; theta one or one for each axis."""
    x = np.asarray(x, np.float64)
    rows = x.shape[0]
    out = x.reshape(rows, heads, -1).copy()
    thetas = [theta] * len(axes) if np.isscalar(theta) else list(theta)
    turned, p = sum(axes), 0
    for a, n in enumerate(axes):
        for j in range(n // 2):
            angle = np.asarray(positions, np.float64)[first_rows:, a] * float(np.float32(thetas[a])) ** (-2.0 * j / n)
            c, s = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1 if backward else 1)
            i, k = (p, p + turned // 2) if halves else (2 * p, 2 * p + 1)
            u, v = out[first_rows:, :, i].copy(), out[first_rows:, :, k].copy()
            out[first_rows:, :, i], out[first_rows:, :, k] = u * c - v * s, u * s + v * c
            p += 1
    return out.reshape(rows, -1)


def grid_positions(rows, grid, origin=None, first_rows=0):
    """Positions of rows from first_rows on over a repeated grid, the last axis fastest."""
    out = np.zeros((rows, len(grid)))
    n = np.arange(rows - first_rows)
    for a in reversed(range(len(grid))):
        out[first_rows:, a] = n % grid[a] + (0 if origin is None else origin[a])
        n = n // grid[a]
    return out


def visible(nq, nk, frame=0, before=-1, after=-1, q_first=0):
    """[nq, nk] truth values."""
    if frame == 0:
        return np.ones((nq, nk), bool)
    at = (np.arange(nq) + (nk - nq if q_first < 0 else q_first)) // frame
    frames = np.arange(nk) // frame
    ok = np.ones((nq, nk), bool)
    if before >= 0:
        ok &= frames[None] >= at[:, None] - before
    if after >= 0:
        ok &= frames[None] <= at[:, None] + after
    return ok


def _each(q, k, heads, kv_heads, q_bounds, k_bounds, window):
    d = q.shape[1] // heads
    for (qa, qe), (ka, ke) in zip(q_bounds, k_bounds):
        ok = visible(qe - qa, ke - ka, **window)
        for h in range(heads):
            g = h * kv_heads // heads
            yield slice(qa, qe), slice(ka, ke), h, slice(h * d, (h + 1) * d), slice(g * d, (g + 1) * d), ok


def _weights(q, k, scale, ok):
    s = np.where(ok, scale * (q @ k.T), -np.inf)
    if s.shape[1] == 0:
        return np.zeros(s.shape), np.full(len(s), -np.inf)
    top = s.max(1, keepdims=True)
    e = np.exp(s - np.where(np.isfinite(top), top, 0))
    e = np.where(ok, e, 0)
    total = e.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (np.where(np.isfinite(top), top, 0) + np.log(total))[:, 0]
    return e / np.where(total > 0, total, 1), lse


def forward(q, k, v, heads, kv_heads, q_bounds, k_bounds, scale, **window):
    """dict of out, lse (rows of no sequence: NaN), and size_out = sum p |v|, size_lse = the largest sum |q k| scale."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    out, size = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, size_lse = np.full((heads, len(q)), np.nan), np.full((heads, len(q)), np.nan)
    for rows, keys, h, mine, its, ok in _each(q, k, heads, kv_heads, q_bounds, k_bounds, window):
        p, lse[h, rows] = _weights(q[rows, mine], k[keys, its], scale, ok)
        out[rows, mine] = p @ v[keys, its]
        size[rows, mine] = p @ np.abs(v[keys, its])
        terms = np.where(ok, np.abs(q[rows, mine]) @ np.abs(k[keys, its]).T, 0) * abs(scale)
        size_lse[h, rows] = terms.max(1) if terms.shape[1] else 0
    return dict(out=out, lse=lse, size_out=size, size_lse=size_lse)


def backward(dout, q, k, v, heads, kv_heads, q_bounds, k_bounds, scale, **window):
    """dict of dq, dk, dv (rows of no sequence: NaN), and for each the sizes of its terms: size_dv = sum P |dout|,
    size_dq = scale sum |dS| |k|, size_dk = scale sum |dS| |q|, and flat_dq, flat_dk, the same with
    P sum(|dout| |out|) in the place of |dS|: what an error in the row's sum of dout out is multiplied by, and raw_dq,
    raw_dk with P sum(|dout| |v|): what one in dout v^T is."""
    dout, q, k, v = (np.asarray(t, np.float64) for t in (dout, q, k, v))
    r = {n: np.full(t.shape, np.nan) for n, t in (("dq", q), ("dk", k), ("dv", v))}
    r.update({f"{n}_d{x}": np.full(t.shape, np.nan) for n in ("size", "flat", "raw") for x, t in (("q", q), ("k", k))})
    r["size_dv"] = np.full(v.shape, np.nan)
    for (qa, qe), (ka, ke) in zip(q_bounds, k_bounds):
        for n in r:
            r[n][(slice(qa, qe) if n.endswith("q") else slice(ka, ke))] = 0
    for rows, keys, h, mine, its, ok in _each(q, k, heads, kv_heads, q_bounds, k_bounds, window):
        p, _ = _weights(q[rows, mine], k[keys, its], scale, ok)
        g, kk, qq, vv = dout[rows, mine], k[keys, its], q[rows, mine], v[keys, its]
        dp = g @ vv.T
        ds = p * (dp - (p * dp).sum(1, keepdims=True))
        flat = p * (np.abs(g) * np.abs(p @ vv)).sum(1, keepdims=True)
        r["dv"][keys, its] += p.T @ g
        r["size_dv"][keys, its] += p.T @ np.abs(g)
        r["dq"][rows, mine] += scale * ds @ kk
        r["dk"][keys, its] += scale * ds.T @ qq
        raw = p * (np.abs(g) @ np.abs(vv).T)
        for n, t in (("size", np.abs(ds)), ("flat", flat), ("raw", raw)):
            r[n + "_dq"][rows, mine] += abs(scale) * t @ np.abs(kk)
            r[n + "_dk"][keys, its] += abs(scale) * t.T @ np.abs(qq)
    return r
