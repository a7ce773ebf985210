"""Norm sites and their gradients on the GPU against the 64-bit definitions.

Tolerances (2-norm of the difference over that of the result).  Per element
fp32 makes at most 20 roundings of 2^-24 and two reciprocal roots of 2^-22,
2e-6 in all; a rounding to bf16 (8 significant bits) is at most 2^-8 of an element.  A
sum over R <= 700 rows of either sign gathers sqrt(R) 2^-24 of its terms' size:
2e-6, and the terms bring theirs."""

import numpy as np
import pytest

import oracle.adaln_oracle as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"
TOL = {torch.float32: 2e-6, torch.bfloat16: 2.0 ** -8 + 2e-6}
SUM_TOL = 6e-6
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "mixed": (torch.float32, torch.bfloat16),
         "fp32": (torch.float32, torch.float32), "wide": (torch.bfloat16, torch.float32)}


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


def close(got, want, tol, what=""):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    off = np.linalg.norm(got - want)
    assert off <= tol * np.linalg.norm(want) + 1e-30, (what, off / max(np.linalg.norm(want), 1e-30))


def make(rows, d, types, seed=0, groups=1, vectors=True, weights=True):
    stream, branch = TYPES[types]
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s, dt=torch.float32, std=1.0, mean=0.0: (mean + std * torch.randn(*s, device=DEV, generator=gen)).to(dt)  # noqa: E731
    t = dict(x=n(rows, d, dt=stream, mean=0.2), y=n(rows, d, dt=branch, std=0.5), du=n(rows, d, dt=branch, std=0.01),
             dr=n(rows, d, dt=stream, std=0.01))
    if d > 8:
        t["x"][:, 3] *= 20  # a channel far above the others
    vec = {}
    if vectors:
        mod = n(groups, 3 * d, std=0.4)
        vec.update(shift=mod[:, :d], scale=mod[:, d:2 * d], gate=mod[:, 2 * d:])
    if weights:
        vec.update(post_w=n(d, mean=1.0, std=0.1), pre_w=n(d, mean=1.0, std=0.1))
    return t, vec


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def both(acid, t, vec, how, tols=(1, 1), what=""):
    """Forward and backward of one site against the oracle."""
    nv = {k: f64(v) for k, v in vec.items()}
    r, u = acid.acid_norm_site_forward(t["x"], t["y"], **vec, **how)
    rr, ru = O.norm_site(f64(t["x"]), f64(t["y"]), **nv, **how)
    close(r, rr, TOL[r.dtype] * tols[0], (what, "r"))
    close(u, ru, TOL[u.dtype] * tols[0], (what, "u"))
    g = acid.acid_norm_site_backward(t["du"], r, t["y"], dr=t["dr"], **vec, **how)
    ref = O.norm_site_grad(f64(t["du"]), f64(r), f64(t["y"]), f64(t["dr"]), **nv, **how)
    want = {"dx", "dy"} | {"d" + k for k in vec}
    assert set(g) == want
    for k in sorted(want):
        tol = TOL[g[k].dtype] if k in ("dx", "dy") else SUM_TOL
        close(g[k].reshape(ref[k].shape), ref[k], tol * tols[1], (what, k))
    return r, u, g


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,d", [(1, 8), (2, 1536), (37, 264), (300, 256), (129, 1000), (45, 1920), (19, 3072), (5, 4096)])
def test_sizes_and_types(acid, rows, d, types):
    t, vec = make(rows, d, types, seed=d)
    both(acid, t, vec, dict(post_norm="rms", pre_norm="layer", eps=1e-6, res_scale=0.9, branch_scale=1.1))


@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("tanh", [False, True])
def test_norm_kinds(acid, post, pre, tanh):
    t, vec = make(67, 1544, "mixed", seed=7)
    both(acid, t, vec, dict(post_norm=post, pre_norm=pre, gate_tanh=tanh, eps=1e-5))


@pytest.mark.parametrize("rows,first,group", [(700, 0, 0), (700, 226, 0), (700, 700, 5), (700, 0, 100), (700, 3, 1),
                                              (700, 699, 4), (700, 50, 33), (1, 0, 7), (1, 1, 0), (311, 0, 310),
                                              (311, 1, 1000)])
def test_groups_of_rows(acid, rows, first, group):
    groups = acid.norm_site_groups(rows, first, group)
    assert groups == O.row_groups(rows, first, group).max() + 1
    for types in ("mixed", "bf16"):
        t, vec = make(rows, 520, types, seed=rows + first, groups=groups)
        how = dict(first_rows=first, group_rows=group, gate_tanh=True, post_norm="layer", pre_norm="rms")
        both(acid, t, vec, how, what=(rows, first, group))


def test_optional_parts(acid):
    """Each vector alone, no branch, no u, no r, gradients from du or dr alone."""
    t, vec = make(33, 512, "mixed", seed=5)
    for name in ("gate", "scale", "shift", "post_w", "pre_w"):
        one = {name: vec[name]}
        r, u = acid.acid_norm_site_forward(t["x"], t["y"], **one)
        rr, ru = O.norm_site(f64(t["x"]), f64(t["y"]), **{name: f64(vec[name])})
        close(r, rr, TOL[r.dtype], name)
        close(u, ru, TOL[u.dtype], name)
        g = acid.acid_norm_site_backward(t["du"], r, t["y"], **one)
        ref = O.norm_site_grad(f64(t["du"]), f64(r), f64(t["y"]), **{name: f64(vec[name])})
        assert "d" + name in g
        for k, v in g.items():
            close(v.reshape(ref[k].shape), ref[k], TOL[v.dtype] if k in ("dx", "dy") else SUM_TOL, (name, k))
    nv = {k: f64(v) for k, v in vec.items()}
    rr, ru = O.norm_site(f64(t["x"]), f64(t["y"]), **nv)
    r, u = acid.acid_norm_site_forward(t["x"], t["y"], want_u=False, **vec)
    assert u is None
    close(r, rr, TOL[r.dtype])
    r2, u = acid.acid_norm_site_forward(t["x"], t["y"], want_r=False, **vec)
    assert r2 is None
    close(u, ru, TOL[u.dtype])
    # no branch: the norm in front of the first one
    for types in TYPES:
        t2, v2 = make(33, 512, types, seed=6)
        some = {k: v2[k] for k in ("scale", "shift", "pre_w")}
        ns = {k: f64(v) for k, v in some.items()}
        r0, u0 = acid.acid_norm_site_forward(t2["x"], None, res_scale=0.5, branch_dtype=TYPES[types][1], **some)
        rr, ru = O.norm_site(f64(t2["x"]), None, res_scale=0.5, **ns)
        close(r0, rr, TOL[r0.dtype])
        close(u0, ru, TOL[u0.dtype])
        g = acid.acid_norm_site_backward(t2["du"], r0, None, dr=t2["dr"], res_scale=0.5, **some)
        ref = O.norm_site_grad(f64(t2["du"]), f64(r0), None, f64(t2["dr"]), res_scale=0.5, **ns)
        assert set(g) == {"dx", "dscale", "dshift", "dpre_w"}
        for k, v in g.items():
            close(v.reshape(ref[k].shape), ref[k], TOL[v.dtype] if k == "dx" else SUM_TOL, k)
    # the last site of a stack: u was not formed
    g = acid.acid_norm_site_backward(None, None, t["y"], dr=t["dr"], **vec)
    ref = O.norm_site_grad(None, None, f64(t["y"]), f64(t["dr"]), **nv)
    assert set(g) == {"dx", "dy", "dgate", "dpost_w"}
    for k, v in g.items():
        close(v.reshape(ref[k].shape), ref[k], TOL[v.dtype] if k in ("dx", "dy") else SUM_TOL, k)


@pytest.mark.parametrize("post,pre", [("layer", "layer"), ("rms", "rms")])
def test_odd_rows(acid, post, pre):
    """Rows of zeros and of one value, rows far from zero, tiny rows; a row with an infinity or a NaN spoils itself alone."""
    t, vec = make(40, 768, "fp32", seed=9)
    t["x"][0], t["y"][0] = 0.0, 0.0
    t["x"][1], t["y"][1] = 2.5, -1.5
    t["x"][2] += 1000.0
    t["y"][3] += 300.0
    t["x"][4] *= 1e-12
    t["y"][4] *= 1e-12
    how = dict(post_norm=post, pre_norm=pre, eps=1e-6)
    nv = {k: f64(v) for k, v in vec.items()}
    r, u = acid.acid_norm_site_forward(t["x"], t["y"], **vec, **how)
    rr, ru = O.norm_site(f64(t["x"]), f64(t["y"]), **nv, **how)
    # a row at 1000 with unit deviation loses 1000 x 2^-24 of it before any norm
    lossy = np.zeros(40, bool)
    lossy[[2, 3]] = True
    for got, want in ((r, rr), (u, ru)):
        close(got[~torch.from_numpy(lossy).to(DEV)], want[~lossy], 2e-6)
        close(got[torch.from_numpy(lossy).to(DEV)], want[lossy], 2e-4)
    assert (u[0] == vec["shift"][0]).all() or post != "layer"
    clean = acid.acid_norm_site_backward(t["du"], r, t["y"], dr=t["dr"], **vec, **how)
    bad = {k: v.clone() for k, v in t.items()}
    bad["x"][7, 5], bad["x"][8, 0], bad["y"][9, 3], bad["y"][10, 767] = float("inf"), float("nan"), float("nan"), -float("inf")
    r2, u2 = acid.acid_norm_site_forward(bad["x"], bad["y"], **vec, **how)
    keep = torch.ones(40, dtype=torch.bool, device=DEV)
    keep[7:11] = False
    assert torch.equal(r2[keep], r[keep]) and torch.equal(u2[keep], u[keep])
    assert not torch.isfinite(u2[7:11]).all(1).any()
    g = acid.acid_norm_site_backward(t["du"], r2, bad["y"], dr=t["dr"], **vec, **how)
    for k in ("dx", "dy"):
        assert torch.equal(g[k][keep], clean[k][keep]) and not torch.isfinite(g["dx"][7:11]).all(1).any()


def test_strides_places_and_streams(acid):
    """Columns of wider buffers, results over their inputs, a stream of the caller's own, and the same bits again."""
    rows, d = 211, 1536
    how = dict(post_norm="rms", pre_norm="layer", first_rows=17, group_rows=50)
    groups = acid.norm_site_groups(rows, 17, 50)
    t, vec = make(rows, d, "mixed", seed=11, groups=groups)
    r, u, g = both(acid, t, vec, how)
    wide = {k: torch.full((rows, 2 * d + 64), 7.0, device=DEV, dtype=v.dtype) for k, v in t.items()}
    view = {k: v[:, 8:8 + d] for k, v in wide.items()}
    for k, v in t.items():
        view[k].copy_(v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r2, u2 = acid.acid_norm_site_forward(view["x"], view["y"], **vec, **how)
        g2 = acid.acid_norm_site_backward(view["du"], r2, view["y"], dr=view["dr"], **vec, **how)
    side.synchronize()
    assert torch.equal(r, r2) and torch.equal(u, u2)
    for k in g:
        assert torch.equal(g[k], g2[k]), k
    # in place
    y0 = view["y"].clone()
    g3 = acid.acid_norm_site_backward(view["du"], r, view["y"], dr=view["dr"], dx=view["dr"], dy=view["du"], **vec, **how)
    assert torch.equal(view["dr"], g["dx"]) and torch.equal(view["du"], g["dy"]) and torch.equal(g3["dgate"], g["dgate"])
    assert torch.equal(view["y"], y0)
    acid.acid_norm_site_forward(view["x"], view["y"], r=view["x"], u=view["y"], **vec, **how)
    assert torch.equal(view["x"], r) and torch.equal(view["y"], u)
    for v in wide.values():  # nothing beside the columns was touched
        assert (v[:, :8] == 7).all() and (v[:, 8 + d:] == 7).all()


def test_empty(acid):
    t, vec = make(0, 256, "mixed")
    n = acid.launch_count()
    r, u = acid.acid_norm_site_forward(t["x"], t["y"], post_w=vec["post_w"])
    assert r.shape == (0, 256) and u.shape == (0, 256) and acid.launch_count() == n
    g = acid.acid_norm_site_backward(t["du"], r, t["y"], post_w=vec["post_w"], pre_w=vec["pre_w"])
    assert (g["dpost_w"] == 0).all() and (g["dpre_w"] == 0).all()


def test_offsets_past_32_bits(acid):
    """Rows around element 2^31 of a tall matrix, against the same rows by themselves."""
    d, rows = 4096, (1 << 31) // 4096 + 5
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty(rows, d, device=DEV, dtype=torch.bfloat16).normal_(0, 1, generator=gen)
    y = torch.empty(rows, d, device=DEV, dtype=torch.bfloat16).normal_(0, 1, generator=gen)
    r, u = acid.acid_norm_site_forward(x, y)
    g = acid.acid_norm_site_backward(u, r, y, vectors=False)
    for at in (slice(0, 3), slice(rows - 9, rows)):
        r1, u1 = acid.acid_norm_site_forward(x[at], y[at])
        assert torch.equal(r[at], r1) and torch.equal(u[at], u1)
        g1 = acid.acid_norm_site_backward(u[at], r[at], y[at], vectors=False)
        assert torch.equal(g["dx"][at], g1["dx"]) and torch.equal(g["dy"][at], g1["dy"])


def test_binding_refusals(acid):
    t, vec = make(6, 256, "mixed")
    f, b = acid.acid_norm_site_forward, acid.acid_norm_site_backward
    for bad in (dict(gate=vec["gate"][:, :128]), dict(gate=torch.zeros(2, 256, device=DEV)),
                dict(scale=vec["scale"].double()), dict(post_w=torch.zeros(257, device=DEV)),
                dict(first_rows=7), dict(group_rows=-1), dict(r=torch.zeros(6, 256, device=DEV, dtype=torch.bfloat16)),
                dict(u=torch.zeros(5, 256, device=DEV, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            f(t["x"], t["y"], **bad)
    with pytest.raises(ValueError):
        f(t["x"], t["y"].cpu())
    with pytest.raises(ValueError):
        b(t["du"], t["x"][:5], t["y"])
    with pytest.raises(acid.A.AcidError):
        f(t["x"][:, :250], t["y"][:, :250])  # 250 columns
    with pytest.raises(acid.A.AcidError):
        f(t["x"], t["y"], want_r=False, want_u=False)
    with pytest.raises(acid.A.AcidError):
        b(t["du"], t["x"], t["y"], workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
