"""Attention with row sums and its gradient against the definitions in 64 bits: types, heads that share keys, sequences
that are packed, padded or empty, windows of frames, rows that see nothing, lengths around the tiles' edges.

Tolerances.  u is half a step of the type (bf16 2^-8, fp32 2^-24), w = 2^-24.  A score is a sum of head_dim products in
fp32: off by (head_dim + 4) w times the sum of its terms' sizes; so is the row sum's logarithm, and both meet in the
exponent, so a probability is off by the share ep = 2 (head_dim + 8) w S + |lse| w + 2^-20, S the largest of those sums
(2^-20: the exponential's own error and those of its argument's scaling).  In bf16 a probability and a score's gradient
enter the next product rounded, each off by u of itself.  A sum of n terms in fp32 adds n w of its terms' sizes, and the
result's own rounding u of itself.  dout out is formed from the rounded out: off by (u + (head_dim + 4) w) sum |dout out|."""

import numpy as np
import pytest

from oracle import mha_oracle as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"
W = 2.0 ** -24


@pytest.fixture(autouse=True)
def fp32_by_default():
    """Whatever default another module of the run has set."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.fixture(scope="module")
def acid():
    import __graft_entry__ as g

    g.build()
    from paper_2607_12358_gb300 import acid as a

    return a


def bounds(lengths, room):
    out, at = [], 0
    for n in lengths:
        out.append((at, at + n))
        at += room or n
    return out, at


def rounded(t, dtype):
    return torch.from_numpy(np.ascontiguousarray(t)).to(dtype).double().numpy()


class Case:
    """Operands on the GPU (column blocks of one matrix where they can be) and, rounded as they are there, on the CPU."""

    def __init__(self, dtype, heads, kv, d, q, k, room=0, scale=None, seed=0, spread=1.2, behind=0, **window):
        self.dtype, self.heads, self.kv, self.d, self.window = dtype, heads, kv, d, window
        self.scale = d ** -0.5 if scale is None else scale
        self.qb, nq = bounds(q, 0)
        self.kb, nk = bounds(k, room)
        nq, nk = nq + behind, nk + behind
        self.bounded = len(q) > 1 or room or behind
        rng = np.random.default_rng(seed)
        self.u = 2.0 ** -8 if dtype == torch.bfloat16 else W
        self.nq, self.nk = nq, nk

        def rows(n, width, spread, used):
            t = rng.normal(size=(n, width)) * spread
            keep = np.zeros(n, bool)
            for a, e in used:
                keep[a:e] = True
            t[~keep] = np.nan  # rows of no sequence may hold anything
            return rounded(t, dtype)

        self.q, self.k = rows(nq, heads * d, spread, self.qb), rows(nk, kv * d, spread, self.kb)
        self.v, self.g = rows(nk, kv * d, 1, self.kb), rows(nq, heads * d, 1, self.qb)

    def gpu(self, t, extra=8):
        """Columns of a wider matrix, so that row strides are not the widths."""
        wide = torch.full((t.shape[0], t.shape[1] + 2 * extra), float("nan"), dtype=self.dtype, device=DEV)
        view = wide[:, extra:extra + t.shape[1]]
        view.copy_(torch.from_numpy(t))
        return view

    def how(self, acid):
        h = dict(scale=self.scale)
        if self.bounded:
            h["q_bounds"] = torch.tensor(self.qb, dtype=torch.int32, device=DEV)
            h["k_bounds"] = torch.tensor(self.kb, dtype=torch.int32, device=DEV)
        names = dict(frame="frame_rows", before="frames_before", after="frames_after", q_first="q_first")
        h.update({names[n]: x for n, x in self.window.items()})
        return h

    def error_of_weights(self, f):
        s = np.nanmax(f["size_lse"], initial=0)
        finite = f["lse"][np.isfinite(f["lse"])]
        return 2 * (self.d + 8) * W * s + W * np.abs(finite).max(initial=0) + 2.0 ** -20


SENTINEL = 7.0


def check(name, got, want, tol):
    got = got.double().cpu().numpy()
    out = np.isnan(want)
    assert (got[out] == SENTINEL).all(), f"{name}: rows of no sequence were written"
    same = np.isinf(want) & (got == want)
    with np.errstate(invalid="ignore"):
        bad = ~out & ~same & ~(np.abs(got - want) <= tol)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{name}{i}: {got[i]} for {want[i]}, off by {abs(got[i] - want[i]):.3g}, allowed {tol[i]:.3g};"
                             f" {bad.sum()} of {bad.size}")


def forward(acid, c):
    f = O.forward(c.q, c.k, c.v, c.heads, c.kv, c.qb, c.kb, c.scale, **c.window)
    out = torch.full((c.nq, c.heads * c.d), SENTINEL, dtype=c.dtype, device=DEV)
    lse = torch.full((c.heads, c.nq), SENTINEL, device=DEV)
    acid.acid_mha_forward(c.gpu(c.q), c.gpu(c.k), c.gpu(c.v), c.heads, out=out, lse=lse, **c.how(acid))
    acid.check_device_error()
    ep, n = c.error_of_weights(f), max([e - a for a, e in c.kb])
    round_p = c.u if c.dtype == torch.bfloat16 else 0
    check("out", out, f["out"], 1.01 * ((round_p + 2 * ep + (n + 4) * W) * f["size_out"] + c.u * np.abs(f["out"])) + 1e-30)
    check("lse", lse, f["lse"], np.broadcast_to(ep + (n + 4) * W + 4 * W * np.abs(f["lse"]), f["lse"].shape))
    return f


def backward(acid, c, want=("q", "k", "v")):
    f = O.forward(c.q, c.k, c.v, c.heads, c.kv, c.qb, c.kb, c.scale, **c.window)
    b = O.backward(c.g, c.q, c.k, c.v, c.heads, c.kv, c.qb, c.kb, c.scale, **c.window)
    lse = torch.from_numpy(f["lse"]).float().to(DEV)
    out = {n: torch.full((rows, h * c.d), SENTINEL, dtype=c.dtype, device=DEV)
           for n, rows, h in (("q", c.nq, c.heads), ("k", c.nk, c.kv), ("v", c.nk, c.kv))}
    given = {"d" + n: out[n] for n in want}
    got = acid.acid_mha_backward(c.gpu(c.g), c.gpu(c.q), c.gpu(c.k), c.gpu(c.v), c.gpu(rounded(f["out"], c.dtype)), lse,
                                 c.heads, want=(), **given, **c.how(acid))
    acid.check_device_error()
    assert [t is not None for t in got] == [n in want for n in "qkv"]
    ep, dw = c.error_of_weights(f), (c.d + 4) * W
    round_p = c.u if c.dtype == torch.bfloat16 else 0
    nq, nk = max([e - a for a, e in c.qb]) * (c.heads // c.kv), max([e - a for a, e in c.kb])
    if "v" in want:
        check("dv", out["v"], b["dv"], 1.01 * ((round_p + ep + (nq + 4) * W) * b["size_dv"] + c.u * np.abs(b["dv"])) + 1e-30)
    for n, terms in (("q", nk), ("k", nq)):
        if n in want:
            tol = ((round_p + 2 * ep + (terms + 8) * W) * b["size_d" + n] + (c.u + dw) * b["flat_d" + n]
                   + dw * b["raw_d" + n] + c.u * np.abs(b["d" + n]))
            check("d" + n, out[n], b["d" + n], 1.01 * tol + 1e-30)


B, F = torch.bfloat16, torch.float32
CASES = {
    # name: arguments of Case
    "one row, one key": ((B, 2, 2, 64, [1], [1]), {}),
    "one row, one key, 128": ((B, 1, 1, 128, [1], [1]), {}),
    "one row, many keys": ((B, 3, 3, 128, [1], [1000]), {}),
    "many rows, one key": ((B, 2, 2, 64, [300], [1]), {}),
    "two rows": ((B, 2, 2, 64, [2], [300]), {}),
    "four rows, shared": ((B, 6, 2, 128, [4], [700]), {}),
    "five rows": ((B, 2, 2, 128, [5], [700]), {}),
    "one row, five heads on one": ((B, 5, 1, 64, [1], [513]), {}),
    "one row each": ((B, 4, 2, 128, [1, 1, 0, 1, 1, 1], [300, 1, 50, 0, 64, 1000]), {}),
    "a few rows each, padded": ((B, 4, 1, 64, [3, 1, 4, 0], [60, 64, 1, 13]), dict(room=64)),
    "a few rows, behind": ((B, 2, 2, 64, [3], [100]), dict(behind=1)),
    "a few rows, window": ((B, 2, 2, 128, [4], [400]), dict(frame=2, before=40, after=0, q_first=-1)),
    "a few rows that see nothing": ((B, 2, 1, 64, [4], [60]), dict(frame=1, before=0, after=0, q_first=58)),
    "one row, no scale": ((B, 2, 2, 64, [1], [200]), dict(scale=0.0)),
    "127": ((B, 1, 1, 128, [127], [127]), {}),
    "128": ((B, 1, 1, 128, [128], [128]), {}),
    "129": ((B, 2, 2, 64, [129], [129]), {}),
    "257 by 383": ((B, 2, 2, 128, [257], [383]), {}),
    "640 by 200, 64": ((B, 2, 2, 64, [640], [200]), {}),
    "520 by 1300": ((B, 2, 1, 128, [520], [1300]), {}),
    "shared heads": ((B, 6, 2, 64, [200], [150]), {}),
    "one key head": ((B, 5, 1, 128, [130], [260]), {}),
    "packed": ((B, 2, 2, 64, [5, 128, 1, 300], [7, 64, 130, 256]), {}),
    "packed, empty among them": ((B, 2, 1, 128, [0, 100, 40, 0, 33], [10, 0, 129, 0, 64]), {}),
    "padded": ((B, 2, 2, 128, [140, 60, 200], [77, 128, 3]), dict(room=128)),
    "rows behind the last": ((B, 2, 2, 64, [100, 29], [100, 29]), dict(behind=150)),
    "causal": ((B, 2, 2, 128, [300], [300]), dict(frame=1, after=0)),
    "causal, few rows at the end": ((B, 2, 2, 64, [3], [700]), dict(frame=1, after=0, q_first=-1)),
    "frames": ((B, 2, 2, 64, [400], [400]), dict(frame=50, after=0)),
    "window": ((B, 4, 2, 128, [520], [520]), dict(frame=20, before=2, after=1)),
    "own frame alone": ((B, 1, 1, 64, [390], [390]), dict(frame=39, before=0, after=0)),
    "rows that see nothing": ((B, 2, 2, 128, [300], [200]), dict(frame=10, before=3, after=0)),
    "all see nothing": ((B, 2, 2, 64, [40], [50]), dict(frame=10, before=1, after=0, q_first=500)),
    "before the keys": ((B, 2, 2, 64, [200], [60]), dict(frame=16, before=-1, after=0, q_first=-1)),
    "packed frames": ((B, 2, 1, 64, [150, 40, 260], [150, 80, 260]), dict(frame=32, before=1, after=0, q_first=-1)),
    "no keys": ((B, 1, 1, 64, [10], [0]), dict(behind=1)),
    "peaked": ((B, 2, 2, 128, [200], [300]), dict(spread=4.0)),
    "flat": ((B, 2, 2, 64, [200], [300]), dict(scale=0.0)),
    "negative scale": ((B, 1, 1, 64, [100], [200]), dict(scale=-0.2)),
    "fp32 32": ((F, 2, 2, 32, [70], [45]), {}),
    "fp32 64": ((F, 4, 4, 64, [100], [100]), {}),
    "fp32 96, shared": ((F, 4, 2, 96, [33], [129]), {}),
    "fp32 128": ((F, 2, 2, 128, [130], [257]), {}),
    "fp32 one of many": ((F, 4, 2, 96, [1], [900]), {}),
    "fp32 one of many, 32": ((F, 3, 1, 32, [3], [300]), {}),
    "fp32 one of many, 128": ((F, 8, 2, 128, [2], [300]), dict(frame=1, after=0, q_first=-1)),
    "fp32 one each": ((F, 2, 2, 64, [1, 1, 1], [200, 3, 77]), dict(room=256)),
    "fp32 one": ((F, 1, 1, 32, [1], [1]), {}),
    "fp32 packed": ((F, 2, 1, 64, [5, 0, 40, 17], [17, 9, 33, 1]), {}),
    "fp32 padded": ((F, 2, 2, 64, [30, 50], [7, 48]), dict(room=64)),
    "fp32 behind": ((F, 2, 2, 32, [30], [50]), dict(behind=20)),
    "fp32 frames": ((F, 2, 2, 64, [100], [100]), dict(frame=7, before=2, after=0)),
    "fp32 few at the end": ((F, 2, 2, 64, [2], [300]), dict(frame=1, after=0, q_first=-1)),
    "fp32 nothing seen": ((F, 2, 2, 64, [60], [40]), dict(frame=10, before=0, after=0)),
    "fp32 peaked": ((F, 2, 2, 64, [100], [100]), dict(spread=6.0)),
}


@pytest.mark.parametrize("name", CASES)
def test_forward(acid, name):
    args, how = CASES[name]
    forward(acid, Case(*args, **how))


@pytest.mark.parametrize("name", CASES)
def test_backward(acid, name):
    args, how = CASES[name]
    backward(acid, Case(*args, seed=1, **how))


@pytest.mark.parametrize("want", [("q",), ("k",), ("v",), ("q", "v"), ("k", "v")])
@pytest.mark.parametrize("dtype", [B, F])
def test_some_gradients(acid, want, dtype):
    backward(acid, Case(dtype, 2, 1, 64, [150], [140], seed=2), want=want)


@pytest.mark.parametrize("dtype", [B, F])
def test_gradients_along_the_forward_pass(acid, dtype):
    """The kernels' own out and lse, and the three gradients against a difference of the forward pass in 64 bits: the
    change of sum(out g) along random directions."""
    c = Case(dtype, 4, 2, 64, [200], [180], seed=3, frame=30, before=2, after=0)
    q, k, v, g = c.gpu(c.q), c.gpu(c.k), c.gpu(c.v), c.gpu(c.g)
    out, lse = acid.acid_mha_forward(q, k, v, c.heads, **c.how(acid))
    grads = acid.acid_mha_backward(g, q, k, v, out, lse, c.heads, **c.how(acid))
    rng, h = np.random.default_rng(0), 1e-5
    for i, t in enumerate((c.q, c.k, c.v)):
        step = rng.normal(size=t.shape)
        loss = []
        for sign in (1, -1):
            ops = [c.q, c.k, c.v]
            ops[i] = t + sign * h * step
            loss.append((O.forward(*ops, c.heads, c.kv, c.qb, c.kb, c.scale, **c.window)["out"] * c.g).sum())
        along = (grads[i].double().cpu().numpy() * step).sum()
        # errors of the gradient's elements are independent of the direction: u of the norm, a few times over
        size = np.linalg.norm(grads[i].double().cpu().numpy())
        assert abs((loss[0] - loss[1]) / (2 * h) - along) <= 8 * c.u * size + 1e-6 * size


@pytest.mark.parametrize("dtype", [B, F])
def test_same_bits_again(acid, dtype):
    c = Case(dtype, 4, 2, 64, [300, 41], [290, 200], seed=4)
    q, k, v, g = c.gpu(c.q), c.gpu(c.k), c.gpu(c.v), c.gpu(c.g)

    def once():
        out, lse = acid.acid_mha_forward(q, k, v, c.heads, **c.how(acid))
        return (out, lse) + acid.acid_mha_backward(g, q, k, v, out, lse, c.heads, **c.how(acid))

    first = [t.view(torch.uint8).clone() for t in once()]
    for _ in range(3):
        for a, b in zip(first, once()):
            assert torch.equal(a, b.view(torch.uint8))


def test_no_rows(acid):
    q, k = torch.empty(0, 128, dtype=B, device=DEV), torch.ones(50, 128, dtype=B, device=DEV)
    out, lse = acid.acid_mha_forward(q, k, k, 2)
    assert out.shape == (0, 128) and lse.shape == (2, 0)
    dq, dk, dv = acid.acid_mha_backward(q, q, k, k, out, lse, 2)
    torch.cuda.synchronize()
    assert dq.shape == (0, 128) and not dk.any() and not dv.any()
    out, lse = acid.acid_mha_forward(k, q, q, 2)
    assert not out.any() and torch.isneginf(lse).all()
    dq, dk, dv = acid.acid_mha_backward(k, k, q, q, out, lse, 2)
    assert not dq.any() and dk.shape == (0, 128)


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("room, behind", [(0, 0), (64, 0), (64, 37), (0, 5)])
def test_allocated_results_are_zero_in_padding(acid, dtype, room, behind):
    """Results that the call allocates: zeros in the rows of no sequence; given ones are left as they are there."""
    c = Case(dtype, 4, 2, 64, [30, 0, 64, 1], [64, 5, 0, 33], room=room, behind=behind, seed=5)
    q, k, v, g = (c.gpu(np.nan_to_num(t)) for t in (c.q, c.k, c.v, c.g))
    used = {}
    for n, rows, bs in (("q", c.nq, c.qb), ("k", c.nk, c.kb)):
        used[n] = torch.zeros(rows, dtype=torch.bool, device=DEV)
        for a, e in bs:
            used[n][a:e] = True
    torch.cuda.empty_cache()
    junk = [torch.full((1 << 18,), float("nan"), device=DEV) for _ in range(4)]
    torch.cuda.synchronize()
    del junk  # (what the results are allocated from)
    out, lse = acid.acid_mha_forward(q, k, v, c.heads, **c.how(acid))
    assert not out[~used["q"]].any() and not lse[:, ~used["q"]].any()
    assert not torch.isnan(out).any() and not torch.isnan(lse).any()
    grads = acid.acid_mha_backward(g, q, k, v, out, lse, c.heads, **c.how(acid))
    for n, t in zip("qkk", grads):
        assert not t[~used[n]].any() and not torch.isnan(t).any()
    given = torch.full_like(out, SENTINEL)
    _, lse2 = acid.acid_mha_forward(q, k, v, c.heads, out=given, **c.how(acid))
    assert (given[~used["q"]] == SENTINEL).all() and torch.equal(given[used["q"]], out[used["q"]])
    assert torch.equal(lse2, lse)
