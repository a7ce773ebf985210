"""Norm sites where single values decide.  Tolerances are those of test_gpu_norm_site.py."""

import numpy as np
import pytest

import oracle.adaln_oracle as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_norm_site import DEV, SUM_TOL, TOL, TYPES, acid, both, close, f64, fp32_by_default, make  # noqa: E402, F401


def test_vectors_with_strides_of_their_own(acid):
    """One row stride serves gate, scale and shift: a vector that is repeated by a stride of 0 beside others is refused,
    whichever it is, and so are three of them."""
    t, vec = make(12, 256, "mixed", seed=1, groups=3)
    one = torch.zeros(1, 256, device=DEV).expand(3, 256)
    for name in ("gate", "scale", "shift"):
        with pytest.raises(ValueError, match="one row stride"):
            acid.acid_norm_site_forward(t["x"], t["y"], group_rows=4, **{k: vec[k] for k in ("gate", "scale", "shift")} | {name: one})
    for names in (("gate",), ("gate", "scale", "shift")):
        with pytest.raises(acid.A.AcidError):
            acid.acid_norm_site_forward(t["x"], t["y"], group_rows=4, **{k: one for k in names})


@pytest.mark.parametrize("first", [0, 1, 40])
def test_groups_longer_than_the_rows(acid, first):
    """A group of any length holds the rows that there are."""
    t, vec = make(41, 520, "mixed", seed=2, groups=acid.norm_site_groups(41, first, 0))
    how = dict(first_rows=first)
    r, u, g = both(acid, t, vec, how)
    for group in (41, 1 << 62, (1 << 63) - 1):
        assert acid.norm_site_groups(41, first, group) == vec["gate"].shape[0]
        r2, u2, g2 = both(acid, t, vec, dict(how, group_rows=group))
        assert torch.equal(r, r2) and torch.equal(u, u2) and all(torch.equal(g[k], g2[k]) for k in g)


@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("branch", [True, False])
def test_no_epsilon_without_du(acid, pre, branch):
    """Where u was not formed its norm has no part in the gradients, with an epsilon of 0 too."""
    for types in TYPES:
        t, vec = make(33, 520, types, seed=5)
        how = dict(pre_norm=pre, post_norm="rms", eps=0.0, res_scale=0.9)
        some = {k: vec[k] for k in (("gate", "post_w") if branch else ())}
        y = t["y"] if branch else None
        g = acid.acid_norm_site_backward(None, None, y, dr=t["dr"], **some, **how)
        ref = O.norm_site_grad(None, None, f64(y), f64(t["dr"]), **{k: f64(v) for k, v in some.items()}, **how)
        assert set(g) == ({"dx", "dy", "dgate", "dpost_w"} if branch else {"dx"})
        for k, v in g.items():
            close(v.reshape(ref[k].shape), ref[k], TOL[v.dtype] if k in ("dx", "dy") else SUM_TOL, (types, k))


@pytest.mark.parametrize("rows,group", [(1, 0), (5, 1), (700, 0), (700, 100)])
def test_slope_of_gates_far_out(acid, rows, group):
    """dgate of tanh gates from -10 to 10, column by column: the terms have one sign, so that a column's sum is as good as
    they are (2e-6), and the slope adds an exponential (2^-22) and four roundings (2^-24 each)."""
    d, groups = 520, acid.norm_site_groups(rows, 0, group)
    t, _ = make(rows, d, "fp32", seed=rows, vectors=False, weights=False)
    y, dr = t["y"].abs() + 0.1, t["dr"].abs() + 0.01
    gate = torch.linspace(-10, 10, d, device=DEV).repeat(groups, 1)
    how = dict(gate_tanh=True, group_rows=group, pre_norm="none")
    g = acid.acid_norm_site_backward(None, None, y, dr=dr, gate=gate, **how)
    want = O.norm_site_grad(None, None, f64(y), f64(dr), gate=f64(gate), **how)["dgate"]
    assert (np.abs(f64(g["dgate"]) - want) <= (SUM_TOL if rows > 5 else 3e-6) * want).all()
