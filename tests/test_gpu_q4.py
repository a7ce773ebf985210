"""4-bit modulation projections on the GPU against the 64-bit definitions.

Codes, scales and zero points are compared bit by bit.  Tolerance of fp32
products (2-norm of the difference over that of the result): an fp32 input
enters to within 2^-22 of its row's largest value, at most 5 times the row's
root mean square here (1.2e-6); codes times inputs are exact; sums of 128 columns
take at most 16 additions of either rounding (2^-23 each: 2e-6), those of the
groups at most 32 more of 2^-24 (2e-6)."""

import numpy as np
import pytest

import oracle.adaln_oracle as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"
TOL = {torch.float32: 5e-6, torch.bfloat16: 2.0 ** -8 + 5e-6}
BF, F32 = torch.bfloat16, torch.float32


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


def weight(acid, n, k, group, zeros, scale_dtype=BF, seed=0):
    """A Q4Weight of random codes, and its values."""
    rng = np.random.default_rng(seed)
    per_row = -(-k // group)
    codes = rng.integers(0, 16, (n, k))
    packed = torch.from_numpy(O.q4_pack(codes)).to(DEV)
    packed[:, 64 * (k // 128):] |= torch.from_numpy(O.q4_pack(np.where(np.arange(-(-k // 128) * 128) < k, 0, 15)[None]))[
        :, 64 * (k // 128):].to(DEV)  # unused codes are not zero
    scales = torch.from_numpy(rng.uniform(0.003, 0.009, (n, per_row)).astype(np.float32)).to(DEV, scale_dtype)
    z = torch.from_numpy(rng.integers(0, 16, (n, per_row)).astype(np.uint8)).to(DEV) if zeros else None
    w = O.q4_values(codes, scales.double().cpu().numpy(), None if z is None else z.cpu().numpy(), group)
    return acid.Q4Weight(packed, scales, z, n, k, group), w


def randn(*shape, dtype=F32, seed=0, std=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (std * torch.randn(*shape, device=DEV, generator=gen)).to(dtype)


def f64(t):
    return t.double().cpu().numpy()


def check_both(acid, m, n, k, group, zeros, scale_dtype, xdt, odt, silu, bias=True):
    what = (m, n, k, group, zeros, scale_dtype, xdt, odt, silu)
    q, w = weight(acid, n, k, group, zeros, scale_dtype, seed=n + k)
    x, b = randn(m, k, dtype=xdt, seed=m), randn(n, std=0.02, seed=n) if bias else None
    out = acid.acid_q4_linear_forward(x, q, b, silu=silu, out_dtype=odt)
    assert out.dtype == odt
    close(out, O.q4_linear(f64(x), w, None if b is None else f64(b), silu), TOL[odt], what)
    g = randn(m, n, dtype=odt, seed=k, std=0.01)
    dx, db = acid.acid_q4_linear_backward(g, q, x, silu=silu)
    rdx, rdb = O.q4_linear_grad(f64(g), w, f64(x), silu)
    assert dx.dtype == xdt and db.dtype == F32
    close(dx, rdx, TOL[xdt], ("dx", what))
    close(db, rdb, 5e-6, ("dbias", what))


@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 8, 9, 16, 17, 33, 64, 65, 130])
@pytest.mark.parametrize("group,zeros", [(128, False), (64, True), (32, True)])
def test_rows(acid, m, group, zeros):
    check_both(acid, m, 300, 1000, group, zeros, BF, F32, F32, True)


@pytest.mark.parametrize("n", [1, 7, 8, 31, 64, 129, 1536, 9217])
@pytest.mark.parametrize("k", [1, 31, 127, 128, 129, 256, 1536])
def test_sizes(acid, n, k):
    check_both(acid, 1 if n > 1000 else 3, n, k, 128, False, F32, F32, F32, True)
    check_both(acid, 2, n, k, 32, True, BF, BF, F32, False, bias=False)


@pytest.mark.parametrize("xdt", [F32, BF])
@pytest.mark.parametrize("odt", [F32, BF])
@pytest.mark.parametrize("scale_dtype", [F32, BF])
@pytest.mark.parametrize("silu", [False, True])
def test_types(acid, xdt, odt, scale_dtype, silu):
    for m in (1, 6, 20):
        check_both(acid, m, 520, 384, 64, True, scale_dtype, xdt, odt, silu)


def test_wide(acid):
    """The largest k, and more rows of the weight than any grid keeps resident."""
    check_both(acid, 1, 40, 65536, 128, True, F32, F32, F32, False)
    check_both(acid, 3, 70001, 256, 32, False, BF, F32, F32, True)


def test_offsets_past_32_bits(acid):
    """Products, their gradients and values past element 2^31, against the definition in 64 bits at both ends."""
    n, k, m = 1 << 20, 64, 2050
    gen = torch.Generator(device=DEV).manual_seed(5)
    scales = torch.empty(n, 2, device=DEV).uniform_(0.003, 0.009, generator=gen)
    q = acid.Q4Weight(torch.randint(0, 256, (n, 64), device=DEV, generator=gen, dtype=torch.uint8), scales, None, n, k, 32)
    w = acid.acid_q4_dequantize(q).double()
    x = randn(m, k, seed=6)
    out = acid.acid_q4_linear_forward(x, q, out_dtype=BF)
    for rows in (slice(0, 3), slice(m - 5, m)):
        for cols in (slice(0, 300), slice(n - 300, n)):
            close(out[rows, cols], f64(x[rows].double() @ w[cols].T), TOL[BF], (rows, cols))
    dx, db = acid.acid_q4_linear_backward(out, q)
    at = torch.tensor([0, 1, m // 2, m - 2, m - 1], device=DEV)
    close(dx[at], f64(out[at].double() @ w), TOL[F32], "dx")
    cols = slice(n - 300, n)
    close(db[cols], f64(out[:, cols].double().sum(0)), 5e-6, "dbias")
    n, k = (1 << 16) + 3, 65536  # 2^32 codes and more
    packed = torch.randint(0, 256, (n, k // 2), device=DEV, generator=gen, dtype=torch.uint8)
    scales = torch.empty(n, k // 128, device=DEV, dtype=BF).uniform_(0.003, 0.009, generator=gen)
    q = acid.Q4Weight(packed, scales, None, n, k, 128)
    tail = acid.Q4Weight(packed[-5:], scales[-5:], None, 5, k, 128)
    v = acid.acid_q4_dequantize(q, dtype=BF)
    assert torch.equal(v[-5:], acid.acid_q4_dequantize(tail, dtype=BF))
    x = randn(1, k, seed=7)
    y = acid.acid_q4_linear_forward(x, q)
    close(y[:, -5:], f64(x.double() @ acid.acid_q4_dequantize(tail).double().T), TOL[F32], "long rows")


def test_values_of_x(acid):
    """Rows of zeros, of very large and very small values; an infinity or a NaN stays in its row."""
    q, w = weight(acid, 200, 512, 64, False, seed=4)
    for scale in (1e30, 1e-30, 3e4):
        x = randn(3, 512, seed=1) * scale
        close(acid.acid_q4_linear_forward(x, q), O.q4_linear(f64(x), w), TOL[F32], scale)
        g = randn(3, 200, seed=2) * scale
        close(acid.acid_q4_linear_backward(g, q, want_dbias=False)[0], O.q4_linear_grad(f64(g), w)[0], TOL[F32], scale)
    x = randn(5, 512, seed=3)
    x[1] = 0.0
    x[2, 1:] = 0.0  # one value
    x[3, ::2] *= 1e-6
    out = acid.acid_q4_linear_forward(x, q)
    close(out, O.q4_linear(f64(x), w), TOL[F32])
    assert (out[1] == 0).all()
    close(out[2:3], O.q4_linear(f64(x[2:3]), w), TOL[F32])
    big = randn(4, 512, seed=5)
    ref = acid.acid_q4_linear_forward(big, q)
    big[1, 7], big[2, 9] = float("inf"), float("nan")
    out = acid.acid_q4_linear_forward(big, q)
    assert torch.equal(out[[0, 3]], ref[[0, 3]]) and not torch.isfinite(out[1:3]).any()
    col = np.abs(w[:, 7]) > 0
    assert torch.isinf(out[1][torch.from_numpy(col).to(DEV)]).all()
    # SiLU far out: 0 on the left, the value itself on the right
    far = torch.zeros(2, 512, device=DEV)
    far[0], far[1] = -200.0, 200.0
    out = acid.acid_q4_linear_forward(far, q, silu=True)
    assert (out[0] == 0).all()
    close(out[1:], O.q4_linear(f64(far[1:]), w), TOL[F32])
    dx, _ = acid.acid_q4_linear_backward(randn(2, 200, seed=6), q, far, silu=True)
    assert torch.isfinite(dx).all() and (dx[0] == 0).all()


@pytest.mark.parametrize("group,zeros,scale_dtype", [(128, False, BF), (128, True, F32), (64, True, BF), (64, False, F32),
                                                     (32, True, BF), (32, False, BF)])
@pytest.mark.parametrize("n,k", [(1, 1), (5, 40), (33, 129), (100, 512), (3000, 384), (70001, 256), (40, 16384)])
def test_one_row(acid, group, zeros, scale_dtype, n, k):
    check_both(acid, 1, n, k, group, zeros, scale_dtype, F32, F32, True)
    check_both(acid, 1, n, k, group, zeros, scale_dtype, BF, BF, False, bias=False)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_values_of_one_row(acid, group):
    """Codes, zero points and inputs at the ends of their ranges; sizes of a(x); what is not finite."""
    n, k = 64, 400
    rng = np.random.default_rng(group)
    per_row = -(-k // group)
    codes, z = rng.choice([0, 15], (n, k)), rng.choice([0, 15], (n, per_row))
    codes[0], z[0], codes[1], z[1] = 0, 15, 15, 0  # the largest sums of either sign
    scales = np.full((n, per_row), 0.0078125)
    q = acid.Q4Weight(torch.from_numpy(O.q4_pack(codes)).to(DEV), torch.from_numpy(scales).to(DEV, F32),
                      torch.from_numpy(z.astype(np.uint8)).to(DEV), n, k, group)
    w = O.q4_values(codes, scales, z, group)
    for size in (1.0, 1e30, 1e-30):
        for x in (np.full(k, 1.9999999), np.full(k, -2.0), np.full(k, 2.0), rng.choice([-1.0, 1.9999999], k)):
            t = torch.from_numpy((x * size).astype(np.float32))[None].to(DEV)
            got, want = acid.acid_q4_linear_forward(t, q), O.q4_linear(f64(t), w)
            # 2^-23 of the largest value a column, and fp32 sums of the terms
            assert (np.abs(f64(got) - want) <= 5e-6 * np.abs(f64(t)) @ np.abs(w).T).all()
    x = randn(1, k, seed=8)
    x[0, 200:] = 0.0
    x[0, :128] *= 1e-9  # another 128 columns
    close(acid.acid_q4_linear_forward(x, q), O.q4_linear(f64(x), w), TOL[F32])
    assert (acid.acid_q4_linear_forward(torch.zeros(1, k, device=DEV), q) == 0).all()
    for values in ({5: float("inf")}, {5: float("nan")}, {5: float("inf"), 300: -float("inf")}):
        y = x.clone()
        for c, v in values.items():
            y[0, c] = v
        with np.errstate(invalid="ignore"):
            want = O.q4_linear(f64(y), w)
        np.testing.assert_array_equal(f64(acid.acid_q4_linear_forward(y, q)), want)


@pytest.mark.parametrize("group,zeros", [(128, False), (64, True), (32, True)])
def test_gradient_of_one_row(acid, group, zeros):
    """Sizes of g from row to row of the weight, and what is not finite, where a product with 0 is not a number."""
    q, w = weight(acid, 700, 300, group, zeros, seed=9)
    for size in (1e30, 1e-30):
        g = randn(1, 700, seed=2) * size
        close(acid.acid_q4_linear_backward(g, q)[0], O.q4_linear_grad(f64(g), w)[0], TOL[F32], size)
    g = randn(1, 700, seed=3)
    g[0, 100:] *= 1e-6
    close(acid.acid_q4_linear_backward(g, q)[0], O.q4_linear_grad(f64(g), w)[0], TOL[F32])
    for at, value in ((3, float("inf")), (699, -float("inf")), (64, float("nan"))):
        h = g.clone()
        h[0, at] = value
        with np.errstate(invalid="ignore"):
            want = O.q4_linear_grad(f64(h), w)[0]
        np.testing.assert_array_equal(f64(acid.acid_q4_linear_backward(h, q)[0]), want)
    assert (acid.acid_q4_linear_backward(torch.zeros(1, 700, device=DEV), q)[0] == 0).all()


def test_strides_streams_and_bits(acid):
    n, k, m = 1000, 1536, 7
    q, w = weight(acid, n, k, 128, True, seed=8)
    x, b, g = randn(m, k, seed=1), randn(n, seed=2), randn(m, n, seed=3)
    out = acid.acid_q4_linear_forward(x, q, b, silu=True)
    dx, db = acid.acid_q4_linear_backward(g, q, x, silu=True)
    wide = {name: torch.full((m, c + 11), 7.0, device=DEV) for name, c in (("x", k), ("out", n), ("g", n), ("dx", k))}
    view = {name: t[:, 3:-8] for name, t in wide.items()}
    view["x"].copy_(x)
    view["g"].copy_(g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        acid.acid_q4_linear_forward(view["x"], q, b, silu=True, out=view["out"])
        _, db2 = acid.acid_q4_linear_backward(view["g"], q, view["x"], silu=True, dx=view["dx"])
    side.synchronize()
    assert torch.equal(view["out"], out) and torch.equal(view["dx"], dx) and torch.equal(db, db2)
    for t in wide.values():
        assert (t[:, :3] == 7).all() and (t[:, -8:] == 7).all()
    assert acid.acid_q4_linear_backward(g, q, x, silu=True, want_dbias=False)[1] is None
    only, db3 = acid.acid_q4_linear_backward(g, q, want_dx=False)
    assert only is None and torch.equal(db3, db)


@pytest.mark.parametrize("wdt", [BF, F32])
@pytest.mark.parametrize("scale_dtype", [BF, F32])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_quantiser(acid, wdt, scale_dtype, group, zeros):
    for n, k in ((1, 1), (5, 130), (67, 1000), (130, 1536)):
        w = randn(n, k + 3, dtype=wdt, seed=n, std=0.02)[:, 1:k + 1]
        if n > 3:
            w[1] = 0.0
            w[2] = w[2].abs()
            w[3, :min(k, group)] = 0.0
        q = acid.acid_q4_quantize(w, group, zeros=zeros, scale_dtype=scale_dtype)
        rnd = lambda s: torch.from_numpy(s).to(scale_dtype).float().numpy()  # noqa: E731
        codes, scales, zs = O.q4_quantize(w.float().cpu().numpy(), group, zeros, rnd)
        assert (O.q4_unpack(q.packed.cpu().numpy(), k) == codes).all()
        assert (q.scales.float().cpu().numpy() == scales).all()
        assert zs is None or (q.zeros.cpu().numpy() == zs).all()
        want = O.q4_values(codes, scales, zs, group).astype(np.float32)
        got = acid.acid_q4_dequantize(q)
        assert (got.cpu().numpy() == want).all()
        half = acid.acid_q4_dequantize(q, BF)
        assert torch.equal(half, got.to(BF))
        out = torch.full((n, k + 5), 7.0, device=DEV)
        acid.acid_q4_dequantize(q, out=out[:, 2:-3])
        assert torch.equal(out[:, 2:-3], got) and (out[:, :2] == 7).all() and (out[:, -3:] == 7).all()


@pytest.mark.parametrize("wdt,scale_dtype", [(BF, BF), (BF, F32), (F32, BF), (F32, F32)])
@pytest.mark.parametrize("zeros", [False, True])
def test_quantiser_at_the_middles_of_codes(acid, wdt, scale_dtype, zeros):
    """Values at halves of the scale, some a last place off them, scales from subnormal to 2^120; rows that wide loads
    can read, and their copy a column further on."""
    rng = np.random.default_rng(11)
    n, k = 126, 520
    size = np.exp2(np.arange(n) * 2.0 - 131) * (1 + rng.integers(0, 16, n) / 16)
    v = rng.integers(-14, 15, (n, k)) / 2
    v[:, ::32] = 7  # each group's largest, so that its scale is the row's size
    near = rng.integers(-1, 2, (n, k)) * (rng.random((n, k)) < 0.3)
    w = torch.from_numpy((v * (1 + near * 2.0 ** -23) * size[:, None]).astype(np.float32)).to(DEV, wdt)
    rnd = lambda s: torch.from_numpy(s).to(scale_dtype).float().numpy()  # noqa: E731
    for group in (32, 64, 128):
        codes, scales, zs = O.q4_quantize(w.float().cpu().numpy(), group, zeros, rnd)
        for shift in (0, 1):
            there = torch.zeros(n, k + 8, device=DEV, dtype=wdt)[:, shift:shift + k]
            there.copy_(w)
            q = acid.acid_q4_quantize(there, group, zeros=zeros, scale_dtype=scale_dtype)
            assert (q.scales.float().cpu().numpy() == scales).all()
            assert (O.q4_unpack(q.packed.cpu().numpy(), k) == codes).all()
            assert zs is None or (q.zeros.cpu().numpy() == zs).all()


def test_quantiser_of_values_that_are_not_finite(acid):
    w = randn(4, 256, seed=1)
    w[1, 3], w[2, 200], w[3, 64] = float("nan"), float("inf"), -float("inf")
    for zeros in (False, True):
        q = acid.acid_q4_quantize(w, 64, zeros=zeros, scale_dtype=F32)
        bad = ~torch.isfinite(q.scales)
        assert bad.nonzero().tolist() == [[1, 0], [2, 3], [3, 1]]


def test_memory_of_a_given_stream(acid):
    """A call on a stream that is not the current one takes its outputs and workspace from that stream's memory, whether
    the stream is given as an object or by its handle."""
    def pool(t):
        return next(b["stream"] for b in torch.cuda.memory_snapshot()
                    if b["address"] <= t.data_ptr() < b["address"] + b["total_size"])

    side, x = torch.cuda.Stream(), randn(20, 256, seed=3)
    y = x.to(BF)
    gate = randn(1, 256, seed=4)
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        q = acid.acid_q4_quantize(randn(64, 256, seed=5), 64, True, stream=stream)
        torch.cuda.synchronize()
        w = acid.acid_q4_dequantize(q, stream=stream)
        out = acid.acid_q4_linear_forward(x, q, stream=stream)
        dx, db = acid.acid_q4_linear_backward(out, q, stream=stream)
        r, u = acid.acid_norm_site_forward(x, y, gate=gate, stream=stream)
        g = acid.acid_norm_site_backward(u, r, y, gate=gate, stream=stream)
        torch.cuda.synchronize()
        for t in (q.packed, q.scales, q.zeros, w, out, dx, db, r, u, *g.values()):
            assert pool(t) == side.cuda_stream
        close(out, f64(x) @ f64(w).T, TOL[F32])
        assert torch.equal(r, acid.acid_norm_site_forward(x, y, gate=gate)[0])
    assert pool(acid.acid_q4_linear_forward(x, q)) == torch.cuda.current_stream().cuda_stream


def test_empty_and_refusals(acid):
    q, w = weight(acid, 96, 128, 64, True)
    n = acid.launch_count()
    assert acid.acid_q4_linear_forward(torch.zeros(0, 128, device=DEV), q).shape == (0, 96)
    dx, db = acid.acid_q4_linear_backward(torch.zeros(0, 96, device=DEV), q)
    assert dx.shape == (0, 128) and (db == 0).all() and acid.launch_count() == n
    x = torch.zeros(2, 128, device=DEV)
    for call in (lambda: acid.acid_q4_linear_forward(x[:, :64], q), lambda: acid.acid_q4_linear_forward(x.half(), q),
                 lambda: acid.acid_q4_linear_forward(x, q, torch.zeros(95, device=DEV)),
                 lambda: acid.acid_q4_linear_forward(x, q, out=torch.zeros(3, 96, device=DEV)),
                 lambda: acid.acid_q4_linear_backward(torch.zeros(2, 96, device=DEV), q, silu=True),
                 lambda: acid.Q4Weight(q.packed[:, :32], q.scales, None, 96, 128, 64),
                 lambda: acid.Q4Weight(q.packed, q.scales[:, :1], None, 96, 128, 64),
                 lambda: acid.acid_q4_quantize(x, 48), lambda: acid.acid_q4_quantize(x.t()[::2])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(acid.A.AcidError):
        acid.acid_q4_linear_backward(torch.zeros(2, 96, device=DEV), q,
                                     workspace=torch.empty(0, dtype=torch.uint8, device=DEV))
