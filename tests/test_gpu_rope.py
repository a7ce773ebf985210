"""Rotary positions with several axes, and their gradient, against the definition in 64 bits.

Tolerances: a result is a sum of two products in fp32, off by 3 w of |x1| + |x2| (w = 2^-24) and, for the angle's own
error of 2^-22 of a turn and the 2 w of its sine and cosine, by (2^-22 2 pi + 2 w) (|x1| + |x2|); its rounding is u of
itself (bf16 2^-8, fp32 2^-24)."""

import numpy as np
import pytest

from oracle import mha_oracle as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"
B, F = torch.bfloat16, torch.float32
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


def operand(rows, width, dtype, seed):
    t = torch.from_numpy(np.random.default_rng(seed).normal(size=(rows, width + 24))).to(dtype).to(DEV)
    return t[:, 8:8 + width]


def agree(got, x, heads, axes, positions, dtype, **how):
    xs = x.double().cpu().numpy()
    want = O.rope(xs, heads, axes, positions, **how)
    # |x1| + |x2| of each pair bounds both of its results' terms: twice the largest, for every column of the head
    size = np.abs(xs).reshape(len(xs), heads, -1).max(2, keepdims=True) * 2
    u = 2.0 ** -8 if dtype == B else W
    tol = (5 * W + 2.0 ** -22 * 2 * np.pi) * size + u * np.abs(want).reshape(size.shape[0], heads, -1)
    off = np.abs(got.double().cpu().numpy() - want).reshape(tol.shape)
    assert (off <= 1.01 * tol).all(), float((off - tol).max())


CASES = [
    # rows, heads, head_dim, axes, grid, first, halves
    (1, 1, 8, (8,), (1,), 0, False),
    (1, 24, 128, (44, 42, 42), (1, 1, 1), 0, False),
    (301, 24, 128, (44, 42, 42), (3, 5, 7), 0, False),
    (77, 5, 64, (24, 20, 20), (2, 6, 5), 13, False),
    (130, 3, 64, (16, 24, 24), (9, 3, 5), 0, True),
    (50, 7, 128, (16, 24, 24), (50, 1, 1), 50, True),
    (64, 2, 96, (8, 12, 12), (4, 4, 4), 1, True),
    (64, 2, 96, (8, 12, 12), (4, 4, 4), 1, False),
    (33, 4, 256, (64, 64, 64, 64), (2, 2, 2, 5), 0, True),
    (2000, 3, 64, (2, 6, 8), (40, 50, 2), 5, False),
]


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("case", [c for c in CASES])
def test_grid(acid, case, dtype):
    rows, heads, d, axes, grid, first, halves = case
    origin = tuple(3.0 * i for i in range(len(axes)))
    x = operand(rows, heads * d, dtype, 1)
    how = dict(first_rows=first, halves=halves)
    at = O.grid_positions(rows, grid, origin, first)
    got = acid.acid_rope_forward(x, heads, axes, grid=grid, origin=origin, **how)
    agree(got, x, heads, axes, at, dtype, **how)
    assert torch.equal(got[:first], x[:first])
    back = acid.acid_rope_backward(x, heads, axes, grid=grid, origin=origin, **how)
    agree(back, x, heads, axes, at, dtype, backward=True, **how)


@pytest.mark.parametrize("far", [3.0, 1e4, 1.6e7])
@pytest.mark.parametrize("halves", [False, True])
def test_positions_near_and_far(acid, far, halves):
    rows, heads, axes = 123, 2, (16, 24, 24)
    x = operand(rows, heads * 64, F, 2)
    wide = torch.rand(rows, 5, device=DEV, generator=torch.Generator(DEV).manual_seed(1)) * far - far / 3
    at = wide[:, 1:4]
    got = acid.acid_rope_forward(x, heads, axes, theta=(1e4, 100.0, 5e5), positions=at, first_rows=9, halves=halves)
    agree(got, x, heads, axes, at.double().cpu().numpy(), F, theta=(1e4, 100.0, 5e5), first_rows=9, halves=halves)


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", [B, F])
def test_in_place(acid, dtype, halves):
    x = operand(90, 4 * 64, dtype, 3)
    how = dict(grid=(10, 3, 2), first_rows=30, halves=halves)
    want = acid.acid_rope_forward(x, 4, (16, 16, 16), **how)
    got = acid.acid_rope_forward(x, 4, (16, 16, 16), out=x, **how)
    assert got.data_ptr() == x.data_ptr() and torch.equal(got, want)


def test_gradient_is_the_transpose(acid):
    """<R x, g> = <x, R^T g>: the rotation of fp32 values, to the rounding of both sides' 2 n products."""
    x, g = operand(200, 3 * 128, F, 4), operand(200, 3 * 128, F, 5)
    how = dict(grid=(5, 8, 5), first_rows=0)
    a = (acid.acid_rope_forward(x, 3, (44, 42, 42), **how).double() * g.double()).sum()
    b = (x.double() * acid.acid_rope_backward(g, 3, (44, 42, 42), **how).double()).sum()
    size = float(x.double().norm() * g.double().norm())
    assert abs(float(a - b)) <= 2 * (5 * W + 2.0 ** -22 * 2 * np.pi) * 2 * size


def test_no_rows(acid):
    x = torch.empty(0, 128, device=DEV)
    assert acid.acid_rope_forward(x, 2, (64,), grid=(4,)).shape == (0, 128)
