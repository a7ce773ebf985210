"""Attention with row sums and its gradient on more items than the GPU has SMs, so that every CTA goes through several
units: items in both directions of a round, units without keys between others, shares of items that begin and end inside
one another and wrap, key heads with several query heads.  Tolerances as in test_gpu_mha."""

import pytest

from test_gpu_mha import Case, acid, backward, forward, fp32_by_default  # noqa: F401 (fixtures among them)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
B = torch.bfloat16

FORWARD = {
    # three rounds of CTAs, causal: items get shorter, and some of a round end before others
    "causal rounds": ((B, 110, 110, 128, [600], [600]), dict(frame=60, after=0)),
    # packed, of uneven lengths, one of them without keys: its rows are written between other units
    "packed rounds": ((B, 60, 20, 64, [500, 130, 300, 0, 400], [500, 0, 450, 70, 129]), {}),
    # units of one key tile, some whose rows see nothing
    "short units": ((B, 120, 60, 64, [700], [300]), dict(frame=10, before=3, after=0)),
    # two CTAs on an SM, keys of 64 a tile
    "short keys": ((B, 130, 130, 64, [600], [100]), {}),
    # whole items, and a last wave that is split along its keys
    "split wave": ((B, 40, 40, 64, [1060], [1100]), {}),
}
BACKWARD = {
    "whole items, causal": ((B, 70, 70, 128, [600], [600]), dict(frame=60, after=0)),
    "whole items, packed": ((B, 60, 20, 64, [500, 130, 300, 0, 400], [500, 0, 450, 70, 129]), {}),
    # whole items and a last wave whose steps are shared out
    "last wave": ((B, 36, 36, 64, [1100], [1100]), {}),
    "last wave, 128, queries": ((B, 40, 40, 128, [520], [1100]), {}),
    # few items: all steps shared out, shares that begin inside items and wrap round their ends
    "shares": ((B, 3, 3, 128, [1500], [400]), {}),
    "shares, shared heads": ((B, 8, 2, 64, [1500], [600]), {}),
    "shares, packed": ((B, 6, 2, 128, [900, 0, 410, 150], [300, 64, 200, 0]), {}),
    "shares, windows": ((B, 6, 3, 64, [900, 700], [900, 700]), dict(frame=50, before=4, after=1)),
    "shares, long keys": ((B, 4, 4, 128, [260], [2300]), {}),
}


@pytest.mark.parametrize("name", FORWARD)
def test_forward(acid, name):  # noqa: F811
    args, how = FORWARD[name]
    forward(acid, Case(*args, seed=2, **how))


@pytest.mark.parametrize("name", BACKWARD)
def test_backward(acid, name):  # noqa: F811
    args, how = BACKWARD[name]
    backward(acid, Case(*args, seed=3, **how))


@pytest.mark.parametrize("name", ["whole items, causal", "last wave", "shares, packed", "shares, windows"])
def test_same_bits_again(acid, name):  # noqa: F811
    args, how = BACKWARD[name]
    c = Case(*args, seed=4, **how)
    q, k, v, g = c.gpu(c.q), c.gpu(c.k), c.gpu(c.v), c.gpu(c.g)

    def once():
        out, lse = acid.acid_mha_forward(q, k, v, c.heads, **c.how(acid))
        return (out, lse) + acid.acid_mha_backward(g, q, k, v, out, lse, c.heads, **c.how(acid))

    first = [t.clone() for t in once()]
    for _ in range(3):
        for a, b in zip(first, once()):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
