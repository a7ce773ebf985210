"""Pins of the 64-bit norm-site and 4-bit-weight definitions (CPU): against
torch's own norms and autograd, against differences, and against cases worked
by hand."""

import numpy as np
import pytest

import oracle.adaln_oracle as O

torch = pytest.importorskip("torch")

KINDS = ("none", "rms", "layer")


def _args(rng, rows, d, groups, **more):
    v = lambda: rng.normal(size=(groups, d))  # noqa: E731
    return dict(gate=v(), scale=0.3 * v(), shift=v(), post_w=1 + 0.1 * rng.normal(size=d),
                pre_w=1 + 0.1 * rng.normal(size=d), eps=1e-5, res_scale=0.7, branch_scale=1.3, **more)


def test_groups():
    assert O.row_groups(7).tolist() == [0] * 7
    assert O.row_groups(7, 2).tolist() == [0, 0, 1, 1, 1, 1, 1]
    assert O.row_groups(7, 2, 2).tolist() == [0, 0, 1, 1, 2, 2, 3]
    assert O.row_groups(3, 3, 2).tolist() == [0, 0, 0]
    assert O.row_groups(3, 0, 1).tolist() == [0, 1, 2]


def test_norms_are_torchs():
    x = torch.randn(5, 24, dtype=torch.float64)
    ln = torch.nn.functional.layer_norm(x, (24,), eps=1e-5).numpy()
    rms = torch.nn.functional.rms_norm(x, (24,), eps=1e-5).numpy()
    np.testing.assert_allclose(O.norm(x.numpy(), "layer", 1e-5), ln, atol=1e-12)
    np.testing.assert_allclose(O.norm(x.numpy(), "rms", 1e-5), rms, atol=1e-12)


def test_site_by_hand():
    x, y = np.array([[1.0, 2.0]]), np.array([[3.0, 4.0]])
    r, u = O.norm_site(x, y, gate=np.array([2.0, -1.0]), scale=np.array([1.0, 0.0]), shift=np.array([0.0, 5.0]),
                       post_norm="rms", pre_norm="layer", eps=0.0, res_scale=2.0, branch_scale=0.5)
    rms = np.sqrt(12.5)
    want = np.array([2 + 0.5 * 2 * 3 / rms, 4 - 0.5 * 4 / rms])
    np.testing.assert_allclose(r[0], want)
    sign = np.sign(want[0] - want[1])  # two values normed are 1 and -1
    np.testing.assert_allclose(u[0], [2 * sign, -sign + 5])


@pytest.mark.parametrize("pre", KINDS)
@pytest.mark.parametrize("post", KINDS)
@pytest.mark.parametrize("tanh", [False, True])
def test_gradient_is_the_derivative(post, pre, tanh):
    """Against central differences of a random projection of (r, u), and against autograd through the same formula."""
    rng = np.random.default_rng(3)
    rows, d = 7, 8
    how = dict(post_norm=post, pre_norm=pre, gate_tanh=tanh, first_rows=2, group_rows=2)
    a = _args(rng, rows, d, 4)
    x, y, du, dr = (rng.normal(size=(rows, d)) for _ in range(4))

    def value(**kw):
        b = {**a, "x": x, "y": y, **kw}
        r, u = O.norm_site(b.pop("x"), b.pop("y"), **b, **how)
        return (r * dr).sum() + (u * du).sum()

    g = O.norm_site_grad(du, O.norm_site(x, y, **a, **how)[0], y, dr, **a, **how)
    base = {**a, "x": x, "y": y}
    h = 1e-5
    for name in ("x", "y", "gate", "scale", "shift", "post_w", "pre_w"):
        for _ in range(6):
            way = rng.normal(size=base[name].shape)
            slope = (value(**{name: base[name] + h * way}) - value(**{name: base[name] - h * way})) / (2 * h)
            want = (g["d" + name] * way).sum()
            assert abs(slope - want) <= 1e-6 * (1 + abs(want)), name


def test_packing_layout():
    codes = np.arange(128)[None] % 16
    p = O.q4_pack(codes)[0].view("<u4")
    # word 4 t + i holds columns 32 i + 8 t .., lowest bits first
    assert p[4 * 1 + 2] == sum((int(codes[0, 64 + 8 + j]) << (4 * j)) for j in range(8))
    rng = np.random.default_rng(0)
    for k in (1, 7, 128, 129, 300):
        c = rng.integers(0, 16, (3, k))
        assert (O.q4_unpack(O.q4_pack(c), k) == c).all()


def test_quantiser():
    w = np.array([[7.0, -7.0, 3.4, 3.5, 2.5, 0.0]])
    codes, s, z = O.q4_quantize(w, 32, False)
    assert s[0, 0] == 1 and z is None and (codes[0] - 8).tolist() == [7, -7, 3, 4, 2, 0]  # ties to even
    codes, s, z = O.q4_quantize(np.array([[0.0, 15.0, 5.0]]), 32, True)
    assert s[0, 0] == 1 and z[0, 0] == 0 and codes[0].tolist() == [0, 15, 5]
    codes, s, z = O.q4_quantize(np.array([[-3.0, -15.0]]), 32, True)
    assert s[0, 0] == 1 and z[0, 0] == 15 and codes[0].tolist() == [12, 0]
    codes, s, z = O.q4_quantize(np.zeros((1, 4)), 32, False)
    assert s[0, 0] == 0 and (O.q4_values(codes, s, None, 32) == 0).all()
    rng = np.random.default_rng(1)
    w = rng.normal(size=(9, 100)).astype(np.float32)
    for zeros in (False, True):
        codes, s, z = O.q4_quantize(w, 32, zeros)
        err = np.abs(O.q4_values(codes, s, z, 32) - w)
        # half a step; with a zero point rounded by itself the ends may clip by another half
        assert (err <= np.repeat(s, 32, 1)[:, :100] * (1.0 if zeros else 0.5) * 1.0001).all()


def test_linear_gradient_is_the_derivative():
    rng = np.random.default_rng(2)
    x, w, b, g = rng.normal(size=(3, 20)), rng.normal(size=(11, 20)), rng.normal(size=11), rng.normal(size=(3, 11))
    for silu in (False, True):
        dx, db = O.q4_linear_grad(g, w, x, silu)
        way, wb, h = rng.normal(size=x.shape), rng.normal(size=11), 1e-6
        up = (O.q4_linear(x + h * way, w, b + h * wb, silu) * g).sum()
        dn = (O.q4_linear(x - h * way, w, b - h * wb, silu) * g).sum()
        assert abs((up - dn) / (2 * h) - ((dx * way).sum() + (db * wb).sum())) <= 1e-6
    np.testing.assert_allclose(O.q4_linear(np.array([[np.log(3.0)]]), np.array([[2.0]]), silu=True)[0, 0],
                               1.5 * np.log(3.0))
