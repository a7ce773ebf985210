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


def sizes(nq, nk, heads, kv_heads, d, backward, sequences=1):
    """Bytes that the library asks for, of each call on such operands."""
    from paper_2607_12358_gb300 import _capi as A, acid

    bounded = [(8, 8)] if sequences > 1 else [(None, None), (8, None), (None, 8), (8, 8)]  # (addresses that nothing reads)
    for q, k in bounded:
        for window in (dict(frames_before=-1, frames_after=-1), dict(frame_rows=7, frames_before=1, frames_after=0)):
            m = A.acid_mha(nq=nq, nk=nk, dtype=A.ACID_BF16, heads=heads, kv_heads=kv_heads, head_dim=d, scale=1.0,
                           sequences=sequences, q_bounds=q, k_bounds=k, **window)
            yield acid.mha_workspace_size(m, backward)


def bounds(sequences):
    """What the binding looks at of a tensor of bounds on a GPU."""
    return SimpleNamespace(dtype=torch.int32, is_cuda=True, shape=(sequences, 2), dim=lambda: 2, is_contiguous=lambda: True,
                           data_ptr=lambda: 8)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("heads, kv_heads, d", [(4, 4, 128), (8, 4, 64), (1, 1, 64)])
def test_workspace_covers_every_call(acid, heads, kv_heads, d, backward):
    """Bounds add a slot to the items.  Where the items reach the number of SMs with it no scratch is needed, while the
    call without bounds, which has fewer, shares out all its steps: the helper's workspace does for both."""
    rows = [1, 3, 77, 8192]
    for sms in (148, 152):  # (148 stands for them where there is no GPU to ask)
        rows += [128 * n for h in {heads, kv_heads} for n in (sms // h - 1, sms // h, sms // h + 1)]
    for nq in rows:
        q = torch.empty(nq, heads * d, dtype=torch.bfloat16)
        for nk in [0] + rows:
            k = torch.empty(nk, kv_heads * d, dtype=torch.bfloat16)
            for given in ({}, dict(q_bounds=bounds(1)), dict(k_bounds=bounds(1)), dict(q_bounds=bounds(1), k_bounds=bounds(1))):
                room = acid.mha_workspace(q, k, heads, backward=backward, **given)
                assert room.numel() >= max(sizes(nq, nk, heads, kv_heads, d, backward)), (nq, nk, list(given))
            for given in (dict(q_bounds=bounds(3)), dict(k_bounds=bounds(3))):
                room = acid.mha_workspace(q, k, heads, backward=backward, **given)
                assert room.numel() >= max(sizes(nq, nk, heads, kv_heads, d, backward, 3)), (nq, nk, list(given))


def test_workspace_of_the_device_that_the_call_runs_on(acid, monkeypatch):
    """The size goes by the GPU's SMs: a second GPU's is its own, for the same shape."""
    needs, given, device = {0: 1024, 1: 4096}, [], 0
    lib = SimpleNamespace(acid_mha_forward=lambda *args: given.append(args[11]) or 0)
    monkeypatch.setattr(acid, "load", lambda: lib)
    monkeypatch.setattr(acid, "mha_workspace_size", lambda desc, backward=False: needs[device])
    monkeypatch.setattr(acid, "_current_device", lambda: device)
    x = torch.empty(200, 192, dtype=torch.bfloat16)
    for device in (0, 1, 0, 1):
        acid.acid_mha_forward(x, x, x, 3)
        assert given.pop() == needs[device]
