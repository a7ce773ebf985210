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
