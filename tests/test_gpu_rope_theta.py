"""Rotary positions whose pairs turn by more than a radian a place (theta below 1), as far as the statement about the
angle goes: positions below 2^24 theta.  Tolerances as in test_gpu_rope."""

import pytest

from test_gpu_rope import DEV, F, acid, agree, fp32_by_default, operand  # noqa: F401 (fixtures among them)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("theta", [0.5, 1e-2, 1e-4])
@pytest.mark.parametrize("halves", [False, True])
def test_fast_pairs(acid, theta, halves):  # noqa: F811
    rows, heads, axes = 123, 2, (16, 48)
    x = operand(rows, heads * 64, F, 7)
    at = torch.rand(rows, 2, device=DEV, generator=torch.Generator(DEV).manual_seed(2)) * (2.0 ** 24 * theta)
    got = acid.acid_rope_forward(x, heads, axes, theta=theta, positions=at, halves=halves)
    agree(got, x, heads, axes, at.double().cpu().numpy(), F, theta=theta, halves=halves)
