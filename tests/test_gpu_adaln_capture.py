"""The norm sites and the 4-bit projections with their gradients captured into a caller's CUDA graph, a second stream
among them: replayed on changing inputs, the graph gives what the same calls give one by one, bit for bit."""

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"


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


@pytest.mark.parametrize("groups", [1, 12])
def test_captured_calls_equal_eager_calls(acid, groups):
    d, rows = 1536, 600
    gen = torch.Generator(device=DEV).manual_seed(9)
    rand = lambda *s, dt=torch.float32, std=1.0: (std * torch.randn(*s, device=DEV, dtype=torch.float32, generator=gen)).to(dt)  # noqa: E731
    temb, x, y = rand(groups, d), rand(rows, d), rand(rows, d, dt=torch.bfloat16)
    q = acid.acid_q4_quantize(rand(3 * d, d, std=0.02), 64, True)
    bias, w, other = rand(3 * d, std=0.1), rand(d), torch.cuda.Stream()
    new = lambda *s, dt=torch.float32: torch.empty(*s, device=DEV, dtype=dt)  # noqa: E731
    mod, r, u, dtemb, back = new(groups, 3 * d), new(rows, d), new(rows, d, dt=torch.bfloat16), new(groups, d), {}
    ws = new(acid.q4_linear_workspace_size(q, groups), dt=torch.uint8)

    def calls():
        acid.acid_q4_linear_forward(temb, q, bias, silu=True, out=mod, workspace=ws)
        v = dict(shift=mod[:, :d], scale=mod[:, d:2 * d], gate=mod[:, 2 * d:], post_w=w, group_rows=rows // groups)
        acid.acid_norm_site_forward(x, y, r=r, u=u, **v)
        fork = torch.cuda.Event()
        fork.record()
        other.wait_event(fork)
        with torch.cuda.stream(other):
            back["values"] = acid.acid_q4_dequantize(q)
        back.update(acid.acid_norm_site_backward(u, r, y, dr=x, **v))
        dmod = torch.cat([back["dshift"], back["dscale"], back["dgate"]], 1)
        back["dbias"] = acid.acid_q4_linear_backward(dmod, q, temb, silu=True, dx=dtemb, workspace=ws)[1]
        join = torch.cuda.Event()
        join.record(other)
        torch.cuda.current_stream().wait_event(join)

    calls()  # sets the kernels up
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    held = dict(back)  # the graph's own outputs
    for seed in (1, 2, 3):
        temb.copy_(rand(groups, d))
        x.copy_(rand(rows, d))
        calls()
        torch.cuda.synchronize()
        want = [t.clone() for t in (mod, r, u, dtemb, *back.values())]
        got = [mod, r, u, dtemb, *held.values()]
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        graph.replay()  # a replay right behind another
        torch.cuda.synchronize()
        acid.check_device_error()
        for name, a, b in zip(["mod", "r", "u", "dtemb", *held], got, want):
            assert torch.isfinite(b.double()).all() and torch.equal(a, b), (seed, name)
