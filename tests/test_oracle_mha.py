"""Pins of the attention branch's 64-bit definitions: gradients against differences, the rotation against complex
numbers, windows against a loop over rows and keys."""

import numpy as np
import pytest

from oracle import mha_oracle as O

WINDOWS = [dict(), dict(frame=3, before=1, after=0), dict(frame=1, after=0), dict(frame=4, before=0, after=1, q_first=6),
           dict(frame=2, before=-1, after=0, q_first=-1)]


@pytest.mark.parametrize("w", WINDOWS)
def test_windows_row_by_row(w):
    nq, nk = 9, 14
    got = O.visible(nq, nk, **w)
    for i in range(nq):
        for j in range(nk):
            want = True
            if w.get("frame"):
                first = w.get("q_first", 0)
                at = (i + (nk - nq if first < 0 else first)) // w["frame"]
                if w.get("before", -1) >= 0 and j // w["frame"] < at - w["before"]:
                    want = False
                if w.get("after", -1) >= 0 and j // w["frame"] > at + w["after"]:
                    want = False
            assert got[i, j] == want


@pytest.mark.parametrize("w", WINDOWS)
def test_gradients_are_differences(w):
    rng = np.random.default_rng(5)
    heads, kv, d = 4, 2, 3
    qb, kb = [(0, 5), (7, 11)], [(1, 7), (7, 10)]
    q, g = rng.normal(size=(12, heads * d)), rng.normal(size=(12, heads * d))
    k, v = rng.normal(size=(11, kv * d)), rng.normal(size=(11, kv * d))
    used = np.zeros(12, bool)
    for a, e in qb:
        used[a:e] = True

    def loss(q, k, v):
        o = O.forward(q, k, v, heads, kv, qb, kb, 0.6, **w)["out"]
        return (np.where(used[:, None], o, 0) * g).sum()

    got = O.backward(g, q, k, v, heads, kv, qb, kb, 0.6, **w)
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        for _ in range(12):
            i = tuple(rng.integers(0, n) for n in t.shape)
            if np.isnan(got[name][i]):  # a row of no sequence
                continue
            old, h = t[i], 1e-6
            t[i] = old + h
            up = loss(q, k, v)
            t[i] = old - h
            down = loss(q, k, v)
            t[i] = old
            # central differences: h^2 of the third derivative and 2^-52 |loss| / h
            assert abs((up - down) / (2 * h) - got[name][i]) < 1e-7


def test_forward_is_a_softmax():
    rng = np.random.default_rng(0)
    q, k, v = (rng.normal(size=(6, 8)) for _ in range(3))
    r = O.forward(q, k, v, 2, 2, [(0, 6)], [(0, 6)], 0.5)
    for h in range(2):
        c = slice(4 * h, 4 * h + 4)
        e = np.exp(0.5 * q[:, c] @ k[:, c].T)
        assert np.allclose(r["out"][:, c], e @ v[:, c] / e.sum(1, keepdims=True), atol=1e-14)
        assert np.allclose(r["lse"][h], np.log(e.sum(1)), atol=1e-14)


def test_a_row_that_sees_nothing():
    rng = np.random.default_rng(0)
    q, k, v = (rng.normal(size=(6, 4)) for _ in range(3))
    w = dict(frame=2, before=0, after=0, q_first=4)
    r = O.forward(q, k, v, 1, 1, [(0, 6)], [(0, 6)], 0.5, **w)
    assert np.isinf(r["lse"][0, 2:]).all() and (r["out"][2:] == 0).all() and np.isfinite(r["lse"][0, :2]).all()
    b = O.backward(q, q, k, v, 1, 1, [(0, 6)], [(0, 6)], 0.5, **w)
    assert (b["dq"][2:] == 0).all() and (b["dk"][:4] == 0).all() and (b["dv"][:4] == 0).all()


@pytest.mark.parametrize("halves", [False, True])
def test_rotation(halves):
    rng = np.random.default_rng(3)
    axes, heads, d, rows = (4, 2, 6), 3, 16, 7
    x, pos = rng.normal(size=(rows, heads * d)), rng.uniform(0, 50, size=(rows, 3))
    y = O.rope(x, heads, axes, pos, halves=halves, first_rows=2)
    back = O.rope(y, heads, axes, pos, halves=halves, first_rows=2, backward=True)
    assert np.allclose(back, x, atol=1e-13) and (y[:2] == x[:2]).all()
    xs, ys = x.reshape(rows, heads, d), y.reshape(rows, heads, d)
    assert (xs[:, :, 12:] == ys[:, :, 12:]).all()
    p = 0
    for a, n in enumerate(axes):
        for j in range(n // 2):
            i, k = (p, p + 6) if halves else (2 * p, 2 * p + 1)
            turn = np.exp(1j * pos[2:, a] * 10000.0 ** (-2 * j / n))[:, None]
            z = (xs[2:, :, i] + 1j * xs[2:, :, k]) * turn
            assert np.allclose(ys[2:, :, i], z.real, atol=1e-13) and np.allclose(ys[2:, :, k], z.imag, atol=1e-13)
            p += 1


def test_grid_positions():
    p = O.grid_positions(2 + 2 * 12 + 3, (2, 2, 3), origin=(5, 0, 0), first_rows=2)
    assert (p[2] == (5, 0, 0)).all() and (p[3] == (5, 0, 1)).all() and (p[5] == (5, 1, 0)).all()
    assert (p[2 + 11] == (6, 1, 2)).all() and (p[2 + 12] == (5, 0, 0)).all()
