"""4-bit projections of many rows as deep as their pipelines go: CTAs that take several sets of weight rows and tiles that
are not full (the product), several blocks of 128 rows to a share (the gradient), each over several slabs of columns,
against products in 64 bits of the values that the layout describes.

Tolerances are those of test_gpu_q4, whose terms hold here too: the tensor cores' sums end after a group (the product)
or 128 rows (the gradient) and shrink each partial sum by at most 16 x 2^-23 of itself, so that their total is off by
that part of itself, 2e-6; the up to 64 fp32 additions of partial sums behind them are off by sqrt(64) 2^-24 of the
result's size where terms have either sign; inputs enter to within 2^-22 of their largest value, 1.2e-6."""

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_q4 import BF, DEV, F32, TOL, acid, close, f64, fp32_by_default, randn  # noqa: E402, F401

KINDS = [(128, False, BF), (64, False, BF), (32, False, BF), (128, True, BF), (64, True, BF), (32, True, BF), (128, True, F32),
         (64, True, F32), (32, False, F32)]  # group, zero points, type of the scales
# 155 and 313 sets of 256 rows of the weight for 152 CTAs, the last one of 76 and of 129 rows
SIZES = [(39500, 384), (39500, 1000), (80001, 384), (80001, 1000)]


def weight(acid, n, k, group, zeros, scale_dtype):
    """A weight of random codes and its values in 64 bits, by the layout of include/acid.h."""
    gen = torch.Generator(device=DEV).manual_seed(n + k + group)
    per_row = -(-k // group)
    packed = torch.randint(0, 256, (n, 64 * -(-k // 128)), device=DEV, generator=gen, dtype=torch.uint8)
    scales = torch.empty(n, per_row, device=DEV).uniform_(0.003, 0.009, generator=gen).to(scale_dtype)
    z = torch.randint(0, 16, (n, per_row), device=DEV, generator=gen, dtype=torch.uint8) if zeros else None
    col = torch.arange(k, device=DEV)
    byte = 64 * (col // 128) + 4 * (4 * (col % 32 // 8) + col % 128 // 32) + col % 8 // 2
    codes = packed[:, byte].int() >> (4 * (col % 2)).int() & 15
    w = (codes - (8 if z is None else z.int()[:, col // group])).double() * scales.double()[:, col // group]
    return acid.Q4Weight(packed, scales, z, n, k, group), w


@pytest.mark.parametrize("group,zeros,scale_dtype", KINDS)
@pytest.mark.parametrize("n,k", SIZES)
def test_products(acid, n, k, group, zeros, scale_dtype):
    q, w = weight(acid, n, k, group, zeros, scale_dtype)
    b = randn(n, std=0.02, seed=n)
    for m in (1, 3, 5, 17, 34, 64, 70):
        x = randn(m, k, seed=m)
        out = acid.acid_q4_linear_forward(x, q, b)
        want = x.double() @ w.T + b.double()
        close(out, f64(want), TOL[F32], m)
        # the rows of the last tiles by themselves: a tile's fault is small in the norm of all
        for rows in (slice(0, 256), slice(n - 300, n)):
            close(out[:, rows], f64(want[:, rows]), TOL[F32], (m, rows))


@pytest.mark.parametrize("group,zeros,scale_dtype", KINDS)
@pytest.mark.parametrize("n,k", SIZES)
def test_gradients(acid, n, k, group, zeros, scale_dtype):
    q, w = weight(acid, n, k, group, zeros, scale_dtype)
    for m in (1, 2, 33, 64, 65):
        g = randn(m, n, seed=m, std=0.01)
        dx, db = acid.acid_q4_linear_backward(g, q)
        close(dx, f64(g.double() @ w), TOL[F32], m)
        close(db, f64(g.double().sum(0)), 5e-6, m)
        # one row of the weight at a time, at the ends of blocks and of the weight
        for row in (0, 127, 128, 895, 896, n - 1):
            one = torch.zeros_like(g)
            one[:, row] = g[:, row]
            close(acid.acid_q4_linear_backward(one, q, want_dbias=False)[0], f64(one.double() @ w), TOL[F32], (m, row))


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("m", [1, 3])
def test_special_values_in_every_set(acid, m, zeros):
    """What is formed value by value reaches the weight rows of all of a CTA's turns."""
    n, k = 160001, 256
    q, w = weight(acid, n, k, 64, zeros, F32)
    x = randn(m, k, seed=m)
    x[0, 70] = float("inf")
    out = acid.acid_q4_linear_forward(x, q)
    one = torch.zeros(1, k, device=DEV, dtype=torch.float64)
    one[0, 70] = 1.0
    sign = (one @ w.T).sign()[0]
    assert torch.equal(out[0].isnan(), sign == 0) and torch.equal(out[0].sign()[sign != 0], sign[sign != 0].float())
    assert out[0].isinf()[sign != 0].all()
    if m > 1:
        close(out[1:], f64(x[1:].double() @ w.T), TOL[F32])
    big = 2e37 * torch.rand(m, k, device=DEV, generator=torch.Generator(DEV).manual_seed(m))
    close(acid.acid_q4_linear_forward(big, q), f64(big.double() @ w.T), TOL[F32])
