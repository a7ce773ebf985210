"""What the binding of the attention branch's operators hands to the library, seen on the CPU through a stand-in for it."""

from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def acid(monkeypatch):
    import __graft_entry__ as g

    g.build()
    from paper_2607_12358_gb300 import acid as a

    monkeypatch.setattr(a, "_rows_of", lambda name, t, rows, d, dtype: d)  # tensors of the CPU
    monkeypatch.setattr(a, "_stream", lambda stream=None: 0)
    return a


@pytest.mark.parametrize("name", ["axes", "theta", "grid", "origin"])
def test_rotation_of_values_that_change_in_place(acid, monkeypatch, name):
    """A chunk's place along the clip kept in a tensor that is counted up: each call has the numbers of its time."""
    seen = []

    def call(desc, *args):
        d = desc._obj
        seen.append([list(getattr(d, n))[:2] for n in ("axis_dim", "theta", "grid", "origin")])
        return 0

    monkeypatch.setattr(acid, "load", lambda: SimpleNamespace(acid_rope_forward=call, acid_rope_backward=call))
    x = torch.zeros(6, 128, dtype=torch.bfloat16)
    how = dict(axes=(32, 32), theta=(100.0, 200.0), grid=(2, 3), origin=(1.0, 2.0))
    moving = torch.tensor(how[name][0])
    how[name] = (moving, how[name][1])
    want = [[32, 32], [100.0, 200.0], [2, 3], [1.0, 2.0]]
    at = ["axes", "theta", "grid", "origin"].index(name)
    for f in (acid.acid_rope_forward, acid.acid_rope_backward):
        for _ in range(3):
            f(x, 2, how["axes"], theta=how["theta"], grid=how["grid"], origin=how["origin"], out=x)
            want[at][0] = moving.item()
            assert seen.pop() == want
            moving += 2
