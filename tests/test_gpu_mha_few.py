"""Attention of a few query rows on both sides of the rule that chooses its kernel: one key fewer or more, one row more than
the sequences, rows spread evenly or all in one sequence.  Tolerances as in test_gpu_mha, which grant the rounding of the
probabilities in bf16 that only one of the kernels makes."""

import pytest

from test_gpu_mha import Case, acid, backward, forward, fp32_by_default  # noqa: F401 (fixtures among them)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
B, F = torch.bfloat16, torch.float32

CASES = {
    "four rows, most keys": ((B, 12, 12, 128, [4], [5461]), {}),
    "four rows, a key more": ((B, 12, 12, 128, [4], [5462]), {}),
    "two rows, shared": ((B, 12, 4, 64, [2], [22000]), {}),
    "two rows": ((B, 12, 12, 64, [2], [22000]), {}),
    "three rows, shared, window": ((B, 16, 1, 128, [3], [7000]), dict(frame=500, before=9, after=0, q_first=-1)),
    "five rows": ((B, 2, 2, 64, [5], [300]), {}),
    "a row each": ((B, 8, 8, 64, [1] * 9, [700, 1, 64, 0, 129, 1000, 128, 33, 5]), {}),
    "a row each but one": ((B, 8, 8, 64, [1] * 8 + [2], [700, 1, 64, 0, 129, 1000, 128, 33, 5]), {}),
    "one long chunk among rows": ((B, 12, 4, 128, [1] * 7 + [190], [600] * 7 + [2000]), {}),
    "all rows in one sequence": ((B, 4, 4, 64, [0] * 7 + [8] + [0] * 2, [100] * 7 + [1500] + [64] * 2), {}),
    "fp32, one long chunk": ((F, 2, 2, 64, [1] * 7 + [25], [60] * 7 + [500]), {}),
}


@pytest.mark.parametrize("name", CASES)
def test_forward(acid, name):  # noqa: F811
    args, how = CASES[name]
    forward(acid, Case(*args, seed=5, **how))


@pytest.mark.parametrize("name", ["four rows, a key more", "three rows, shared, window", "one long chunk among rows"])
def test_backward(acid, name):  # noqa: F811
    args, how = CASES[name]
    backward(acid, Case(*args, seed=6, **how))
