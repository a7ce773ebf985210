"""4-bit projections where single values decide: scales of very different sizes, what is not finite, results near the
largest number.  Tolerances are those of test_gpu_q4.py."""

import numpy as np
import pytest

import oracle.adaln_oracle as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_q4 import BF, DEV, F32, TOL, acid, close, f64, fp32_by_default, randn, weight  # noqa: E402, F401

KINDS = [(128, False, BF), (64, True, BF), (32, False, F32), (64, True, F32)]  # of scales and zero points


def test_rows_that_overlap_are_refused(acid):
    """Operands whose rows share memory (one row expanded to many, or rows closer than their length) are refused: the
    kernels take a row stride of at least the row."""
    q, _ = weight(acid, 96, 128, 64, True)
    wide = torch.zeros(7 * 128, device=DEV)

    def rows(n, cols):
        return [torch.zeros(1, cols, device=DEV).expand(n, cols), torch.as_strided(wide, (n, cols), (cols - 1, 1))]

    for m in (3, 6):
        x, g = torch.zeros(m, 128, device=DEV), torch.zeros(m, 96, device=DEV)
        for bad in rows(m, 128):
            for call in (lambda: acid.acid_q4_linear_forward(bad, q),
                         lambda: acid.acid_q4_linear_backward(g, q, bad, silu=True),
                         lambda: acid.acid_q4_linear_backward(g, q, dx=bad), lambda: acid.acid_q4_quantize(bad)):
                with pytest.raises(acid.A.AcidError, match="row stride"):
                    call()
        for bad in rows(m, 96):
            for call in (lambda: acid.acid_q4_linear_forward(x, q, out=bad), lambda: acid.acid_q4_linear_backward(bad, q)):
                with pytest.raises(acid.A.AcidError, match="row stride"):
                    call()
    with pytest.raises(acid.A.AcidError, match="row stride"):
        acid.acid_q4_dequantize(q, out=torch.zeros(1, 128, device=DEV).expand(96, 128))


@pytest.mark.parametrize("m", [2, 65])
@pytest.mark.parametrize("group,zeros,scale_dtype", KINDS)
def test_first_scales_far_above_the_last(acid, m, group, zeros, scale_dtype):
    """The gradient's last block of 128 rows is not full; the weight's first scales are 2^12 times those of its rows."""
    q, w = weight(acid, 700, 100, group, zeros, scale_dtype, seed=3)
    q.scales[0] *= 4096.0
    w[0] *= 4096.0
    g = randn(m, 700, seed=1)
    g[:, 0] = 0.0
    close(acid.acid_q4_linear_backward(g, q)[0], O.q4_linear_grad(f64(g), w)[0], TOL[F32])


@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 17])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("silu", [False, True])
def test_inputs_that_are_not_finite(acid, m, group, zeros, silu):
    """An infinity gives what the definition gives, whatever its code and zero point, and the other rows keep their bits."""
    for n, k in ((40, 100), (40, 400)):
        q, w = weight(acid, n, k, group, zeros, F32, seed=k)
        x = randn(m, k, seed=m)
        ref = acid.acid_q4_linear_forward(x, q, silu=silu)
        bad = x.clone()
        bad[0, 7] = float("inf")
        if m > 2:
            bad[1, 64], bad[1, k - 1] = -float("inf"), float("inf")
        if m > 3:
            bad[2, 33] = float("nan")
        got = acid.acid_q4_linear_forward(bad, q, silu=silu)
        with np.errstate(invalid="ignore"):
            want = O.q4_linear(f64(bad), w, silu=silu)
        rows = ~torch.isfinite(bad).all(1).cpu().numpy()
        np.testing.assert_array_equal(f64(got)[rows], want[rows])
        assert (f64(got)[~rows] == f64(ref)[~rows]).all()


@pytest.mark.parametrize("m", [1, 2, 5, 65])
@pytest.mark.parametrize("group,zeros,scale_dtype", KINDS)
def test_gradients_that_are_not_finite(acid, m, group, zeros, scale_dtype):
    """The same for the gradient of the output: rows of dx that meet an infinity or a NaN, and the others' bits."""
    for n, k in ((300, 200), (700, 100)):
        q, w = weight(acid, n, k, group, zeros, scale_dtype, seed=n)
        g = randn(m, n, seed=m)
        ref, ref_bias = acid.acid_q4_linear_backward(g, q)
        bad = g.clone()
        bad[0, 3] = float("inf")
        if m > 1:
            bad[m - 1, 5], bad[m - 1, n - 1] = float("inf"), -float("inf")
        if m > 2:
            bad[1, 129] = float("nan")
        dx, db = acid.acid_q4_linear_backward(bad, q)
        with np.errstate(invalid="ignore"):
            want, want_bias = O.q4_linear_grad(f64(bad), w)
        rows = ~torch.isfinite(bad).all(1).cpu().numpy()
        np.testing.assert_array_equal(f64(dx)[rows], want[rows])
        assert (f64(dx)[~rows] == f64(ref)[~rows]).all()
        cols = ~np.isfinite(want_bias)
        np.testing.assert_array_equal(f64(db)[cols], want_bias[cols])
        assert (f64(db)[~cols] == f64(ref_bias)[~cols]).all()


def positive(acid, n, k, group, zeros, scale_dtype):
    """A weight of positive values, 0.005 to 0.05, and the values."""
    rng = np.random.default_rng(n + k)
    per_row = -(-k // group)
    z = np.full((n, per_row), 5 if zeros else 8)
    codes = rng.integers(9, 16, (n, k))
    scales = torch.full((n, per_row), 0.005, device=DEV).to(scale_dtype)
    q = acid.Q4Weight(torch.from_numpy(O.q4_pack(codes)).to(DEV), scales,
                      torch.from_numpy(z.astype(np.uint8)).to(DEV) if zeros else None, n, k, group)
    return q, O.q4_values(codes, f64(scales), z, group)


@pytest.mark.parametrize("m", [1, 2, 4, 5])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_products_near_the_largest_number(acid, m, group, zeros):
    """Results of 1e38, whose sums before the scales would be past the largest number."""
    for n, k in ((40, 100), (40, 256)):
        q, w = positive(acid, n, k, group, zeros, F32)
        x = 1e37 * (0.5 + 0.5 * torch.rand(m, k, device=DEV, generator=torch.Generator(DEV).manual_seed(m)))
        close(acid.acid_q4_linear_forward(x, q), O.q4_linear(f64(x), w), TOL[F32], (n, k))
        close(acid.acid_q4_linear_forward(-x, q), O.q4_linear(f64(-x), w), TOL[F32], (n, k))


@pytest.mark.parametrize("m", [1, 2, 65])
@pytest.mark.parametrize("group,zeros,scale_dtype", KINDS)
def test_gradients_near_the_largest_number(acid, m, group, zeros, scale_dtype):
    """The same for the input's gradient."""
    for n, k in ((40, 100), (300, 200)):
        q, w = positive(acid, n, k, group, zeros, scale_dtype)
        g = 1e37 * (0.5 + 0.5 * torch.rand(m, n, device=DEV, generator=torch.Generator(DEV).manual_seed(m)))
        for v in (g, -g):
            close(acid.acid_q4_linear_backward(v, q, want_dbias=False)[0], O.q4_linear_grad(f64(v), w)[0], TOL[F32], (n, k))


def test_default_stream_by_its_handle(acid):
    """Handle 0 is the default stream, and its memory is what a call on it takes, whatever stream is current."""
    def pool(t):
        return next(b["stream"] for b in torch.cuda.memory_snapshot()
                    if b["address"] <= t.data_ptr() < b["address"] + b["total_size"])

    x, y, gate = randn(20, 256, seed=3), randn(20, 256, dtype=BF, seed=2), randn(1, 256, seed=4)
    wf = randn(64, 256, seed=5)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for stream in (0, torch.cuda.default_stream()):
            q = acid.acid_q4_quantize(wf, 64, True, stream=stream)
            w = acid.acid_q4_dequantize(q, stream=stream)
            out = acid.acid_q4_linear_forward(x, q, stream=stream)
            dx, db = acid.acid_q4_linear_backward(out, q, stream=stream)
            r, u = acid.acid_norm_site_forward(x, y, gate=gate, stream=stream)
            g = acid.acid_norm_site_backward(u, r, y, gate=gate, stream=stream)
            torch.cuda.synchronize()
            for t in (q.packed, q.scales, q.zeros, w, out, dx, db, r, u, *g.values()):
                assert pool(t) == 0
            close(out, f64(x) @ f64(w).T, TOL[F32])


def test_gradient_of_no_rows(acid):
    """Without rows dx is empty, and may be all that is asked for."""
    q, _ = weight(acid, 96, 128, 64, True)
    dx, db = acid.acid_q4_linear_backward(torch.zeros(0, 96, device=DEV), q, want_dbias=False)
    assert dx.shape == (0, 128) and db is None


@pytest.mark.parametrize("m,n,k", [(5, 300, 1000), (34, 700, 384), (130, 129, 256), (2, 96, 16384)])
def test_product_stays_in_its_workspace(acid, m, n, k):
    """The bytes of acid_q4_linear_forward_workspace_size are enough, and none past them is written."""
    q, w = weight(acid, n, k, 64, True)
    x = randn(m, k, seed=m)
    size = acid.q4_linear_forward_workspace_size(q, m)
    assert 0 < size <= acid.q4_linear_workspace_size(q, m)
    ws = torch.full((size + 4096,), 77, dtype=torch.uint8, device=DEV)
    out = acid.acid_q4_linear_forward(x, q, workspace=ws[:size])
    close(out, O.q4_linear(f64(x), w), TOL[F32])
    assert (ws[size:] == 77).all() and torch.equal(out, acid.acid_q4_linear_forward(x, q))
