"""Norm sites and 4-bit modulation projections in 64 bits on the CPU (numpy),
written from their formulas and sharing nothing with the GPU path.  The paper
has no counterpart; the definitions are those of include/acid.h.

A site: r = res_scale x + branch_scale g (N_post(y) post_w),
u = N_pre(r) pre_w (1 + scale) + shift, with the vectors of the row's group.
"""

from __future__ import annotations

import numpy as np

F = np.float64


def row_groups(rows: int, first_rows: int = 0, group_rows: int = 0) -> np.ndarray:
    """Modulation group of each row: the first rows are one (if there are any), then each group_rows rows."""
    out = np.zeros(rows, dtype=np.int64)
    size = group_rows if group_rows > 0 else max(rows - first_rows, 1)
    for i in range(first_rows, rows):
        out[i] = (1 if first_rows > 0 else 0) + (i - first_rows) // size
    return out


def norm(v: np.ndarray, kind: str, eps: float) -> np.ndarray:
    v = np.asarray(v, F)
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(-1, keepdims=True)
    return v / np.sqrt((v * v).mean(-1, keepdims=True) + eps)


def norm_backward(v: np.ndarray, kind: str, eps: float, grad: np.ndarray) -> np.ndarray:
    """Gradient of norm's input: with n = N(v) and s the root, (grad - n mean(grad n)) / s, for LayerNorm less its mean."""
    if kind == "none":
        return np.asarray(grad, F)
    v = np.asarray(v, F)
    c = v - v.mean(-1, keepdims=True) if kind == "layer" else v
    s = np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    n = c / s
    out = grad - n * (grad * n).mean(-1, keepdims=True)
    if kind == "layer":
        out = out - grad.mean(-1, keepdims=True)
    return out / s


def _vectors(a, rows, d):
    at = row_groups(rows, a.get("first_rows", 0), a.get("group_rows", 0))

    def of(name, none):
        t = a.get(name)
        return np.full((rows, d), none, F) if t is None else np.asarray(t, F).reshape(-1, d)[at]

    gate = of("gate", 1.0)
    slope = np.ones_like(gate)
    if a.get("gate_tanh") and a.get("gate") is not None:
        gate = np.tanh(gate)
        slope = 1 - gate * gate
    ones = np.ones(d)
    w = [ones if a.get(n) is None else np.asarray(a[n], F) for n in ("post_w", "pre_w")]
    return at, gate, slope, 1 + of("scale", 0.0), of("shift", 0.0), w[0], w[1]


def norm_site(x, y, **a):
    """(r, u) of a site; keywords as acid_norm_site_forward's."""
    x = np.asarray(x, F)
    rows, d = x.shape
    _, gate, _, scale, shift, post_w, pre_w = _vectors(a, rows, d)
    eps = a.get("eps", 1e-6)
    r = a.get("res_scale", 1.0) * x
    if y is not None:
        r = r + a.get("branch_scale", 1.0) * gate * norm(y, a.get("post_norm", "rms"), eps) * post_w
    return r, norm(r, a.get("pre_norm", "layer"), eps) * pre_w * scale + shift


def norm_site_grad(du, r, y, dr=None, **a) -> dict:
    """Gradients of norm_site with the statistics of the given r and y."""
    like = np.asarray(r if r is not None else dr, F)
    rows, d = like.shape
    at, gate, slope, scale, _, post_w, pre_w = _vectors(a, rows, d)
    groups = int(at.max()) + 1 if rows else 0
    eps, pre, post = a.get("eps", 1e-6), a.get("pre_norm", "layer"), a.get("post_norm", "rms")
    branch = a.get("branch_scale", 1.0)

    def by_group(v):
        out = np.zeros((groups, d), F)
        np.add.at(out, at, v)
        return out

    out, total = {}, np.zeros((rows, d), F) if dr is None else np.asarray(dr, F)
    if du is not None:
        du = np.asarray(du, F)
        n = norm(r, pre, eps)
        out["dshift"], out["dscale"] = by_group(du), by_group(du * n * pre_w)
        out["dpre_w"] = (du * n * scale).sum(0)
        total = total + norm_backward(r, pre, eps, du * scale * pre_w)
    out["dx"] = a.get("res_scale", 1.0) * total
    if y is not None:
        p = norm(y, post, eps)
        out["dgate"] = by_group(total * branch * p * post_w * slope)
        out["dpost_w"] = (total * branch * gate * p).sum(0)
        out["dy"] = norm_backward(y, post, eps, total * branch * gate * post_w)
    return out


# ------------------------------------------------------------ 4-bit weights
def q4_pack(codes: np.ndarray) -> np.ndarray:
    """Codes [n, k] (0 .. 15) -> uint8 [n, 64 ceil(k / 128)], column by column as the layout is described."""
    n, k = codes.shape
    out = np.zeros((n, 64 * -(-k // 128)), dtype=np.uint8)
    for c in range(k):
        slab, in_slab = divmod(c, 128)
        i, t, j = in_slab // 32, in_slab % 32 // 8, in_slab % 8
        byte = 64 * slab + 4 * (4 * t + i) + j // 2
        out[:, byte] |= (codes[:, c].astype(np.uint8) & 15) << (4 * (j % 2))
    return out


def q4_unpack(packed: np.ndarray, k: int) -> np.ndarray:
    codes = np.zeros((packed.shape[0], k), dtype=np.int64)
    for c in range(k):
        slab, in_slab = divmod(c, 128)
        i, t, j = in_slab // 32, in_slab % 32 // 8, in_slab % 8
        codes[:, c] = packed[:, 64 * slab + 4 * (4 * t + i) + j // 2] >> (4 * (j % 2)) & 15
    return codes


def q4_values(codes, scales, zeros, group: int) -> np.ndarray:
    k = codes.shape[1]
    s = np.repeat(np.asarray(scales, F), group, 1)[:, :k]
    z = 8 if zeros is None else np.repeat(np.asarray(zeros, F), group, 1)[:, :k]
    return s * (codes - z)


def q4_quantize(w: np.ndarray, group: int, zeros: bool, round_scale=None):
    """(codes, scales, zeros or None) of w [n, k]; quotients in 32 bits, as the definition says; round_scale
    rounds the scales to their stored type."""
    w = np.asarray(w, np.float32)
    n, k = w.shape
    per_row = -(-k // group)
    codes = np.zeros((n, k), np.int64)
    scales, zs = np.zeros((n, per_row), np.float32), np.zeros((n, per_row), np.uint8)
    for b in range(per_row):
        v = w[:, b * group:min(k, (b + 1) * group)]
        lo, hi = np.minimum(v.min(1), 0), np.maximum(v.max(1), 0)
        s = (hi - lo) / np.float32(15) if zeros else np.maximum(hi, -lo) / np.float32(7)
        s = s if round_scale is None else round_scale(s)
        div = np.where(s == 0, np.float32(1), s)
        z = np.clip(np.rint(-lo / div), 0, 15) if zeros else np.full(n, 8, np.float32)
        codes[:, b * group:b * group + v.shape[1]] = np.clip(np.rint(v / div[:, None]) + z[:, None], 0, 15)
        scales[:, b], zs[:, b] = s, z
    return codes, scales, zs if zeros else None


def _act(x, silu):
    x = np.asarray(x, F)
    return x / (1 + np.exp(-x)) if silu else x


def q4_linear(x, w, bias=None, silu=False):
    """a(x) W^T + bias with the weight's values w [n, k]."""
    return _act(x, silu) @ np.asarray(w, F).T + (0 if bias is None else np.asarray(bias, F))


def q4_linear_grad(g, w, x=None, silu=False):
    """(dx, dbias)."""
    dx = np.asarray(g, F) @ np.asarray(w, F)
    if silu:
        x = np.asarray(x, F)
        e = 1 / (1 + np.exp(-x))
        dx = dx * e * (1 + x * (1 - e))
    return dx, np.asarray(g, F).sum(0)
