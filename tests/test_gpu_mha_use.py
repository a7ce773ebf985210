"""The attention branch's operators as they are used together and around each other: rotation, attention, gradients and
the rotation taken back on one matrix of queries, keys and values; in a CUDA graph; on other streams; with workspaces
that calls share; rows far apart in memory; sequences beside one that is not finite; bounds outside the operands."""

import numpy as np
import pytest

from oracle import mha_oracle as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda"
B, F = torch.bfloat16, torch.float32


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


def normal(*shape, dtype=B, seed=0, std=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (std * torch.randn(*shape, device=DEV, dtype=F, generator=gen)).to(dtype)


HEADS, KV, D = 4, 2, 64
AXES, GRID = (16, 24, 24), (5, 6, 7)
WINDOW = dict(frame_rows=42, frames_before=2, frames_after=0)


def split(t):
    return t[:, :HEADS * D], t[:, HEADS * D:(HEADS + KV) * D], t[:, (HEADS + KV) * D:]


def branch(acid, qkv, g, dqkv, rope, room):
    """out, lse of the attention of rotated queries and keys (in place), and the gradient of all of qkv."""
    q, k, v = split(qkv)
    turned = qkv[:, :(HEADS + KV) * D]
    acid.acid_rope_forward(turned, HEADS + KV, AXES, grid=GRID, first_rows=rope, out=turned)
    out, lse = acid.acid_mha_forward(q, k, v, HEADS, workspace=room[0], **WINDOW)
    dq, dk, dv = split(dqkv)
    acid.acid_mha_backward(g, q, k, v, out, lse, HEADS, dq=dq, dk=dk, dv=dv, workspace=room[1], **WINDOW)
    turned = dqkv[:, :(HEADS + KV) * D]
    acid.acid_rope_backward(turned, HEADS + KV, AXES, grid=GRID, first_rows=rope, out=turned)
    return out, lse


@pytest.mark.parametrize("dtype", [B, F])
def test_branch_and_its_gradient(acid, dtype):
    """The whole branch's gradient against differences of its loss in 64 bits, along random directions.  The gradient
    goes through five roundings to the type (rotated values, probabilities, their gradient, the sums, the rotation
    back), each off by u of itself in independent directions: 8 u of its norm bounds the error along one direction
    six times over (the error along it is u sqrt(5) of the norm over sqrt(columns x rows))."""
    rows, first, u = 252, 42, 2.0 ** -8 if dtype == B else 2.0 ** -24
    qkv, g = normal(rows, (HEADS + 2 * KV) * D, dtype=dtype, seed=1), normal(rows, HEADS * D, dtype=dtype, seed=2)
    start, g64 = qkv.double().cpu().numpy(), g.double().cpu().numpy()
    dqkv = torch.full_like(qkv, 7)
    out, lse = branch(acid, qkv, g, dqkv, first, (None, None))
    at = O.grid_positions(rows, GRID, first_rows=first)
    window = dict(frame=42, before=2, after=0)

    def loss(t):
        turned = O.rope(t[:, :(HEADS + KV) * D], HEADS + KV, AXES, at, first_rows=first)
        r = O.forward(turned[:, :HEADS * D], turned[:, HEADS * D:], t[:, (HEADS + KV) * D:], HEADS, KV, [(0, rows)],
                      [(0, rows)], D ** -0.5, **window)
        return r, (r["out"] * g64).sum()

    r, _ = loss(start)
    err = np.abs(out.double().cpu().numpy() - r["out"]).max()
    assert err <= 16 * u * np.abs(r["out"]).max()
    assert np.abs(lse.double().cpu().numpy() - r["lse"]).max() <= 16 * u * np.abs(start).max()
    grad, rng, h = dqkv.double().cpu().numpy(), np.random.default_rng(0), 1e-5
    for part in range(3):
        step = np.zeros_like(start)
        c = [slice(0, HEADS * D), slice(HEADS * D, (HEADS + KV) * D), slice((HEADS + KV) * D, None)][part]
        step[:, c] = rng.normal(size=step[:, c].shape)
        along = (loss(start + h * step)[1] - loss(start - h * step)[1]) / (2 * h)
        size = np.linalg.norm(grad[:, c])
        assert abs(along - (grad * step).sum()) <= 8 * u * size + 1e-6 * size


@pytest.mark.parametrize("dtype", [B, F])
def test_captured_and_replayed(acid, dtype):
    rows = 210
    new = [(normal(rows, (HEADS + 2 * KV) * D, dtype=dtype, seed=s), normal(rows, HEADS * D, dtype=dtype, seed=s + 50))
           for s in range(3)]
    qkv, g = new[0][0].clone(), new[0][1].clone()
    dqkv = torch.empty_like(qkv)
    room = [acid.mha_workspace(qkv[:, :HEADS * D], qkv[:, :KV * D], HEADS, backward=b) for b in (False, True)]
    got = branch(acid, qkv, g, dqkv, 0, room)  # sets the kernels up
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):  # two graphs over one workspace, replayed in turn
        qkv.copy_(new[0][0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = branch(acid, qkv, g, dqkv, 0, room)
        graphs.append((graph, got))
    for i, (x, y) in enumerate(new * 2):
        qkv.copy_(x)
        g.copy_(y)
        graph, got = graphs[i % 2]
        graph.replay()
        torch.cuda.synchronize()
        x2, want = x.clone(), torch.empty_like(x)
        out, lse = branch(acid, x2, y, want, 0, (None, None))
        assert torch.equal(dqkv, want) and torch.equal(got[0], out) and torch.equal(got[1], lse)


@pytest.mark.parametrize("as_handle", [False, True])
def test_other_streams(acid, as_handle):
    """Calls given a stream run there, whatever the current one; two at once with workspaces of their own."""
    q, k, v = (normal(600, 256, seed=s) for s in (1, 2, 3))
    g = normal(600, 256, seed=4)
    x = normal(600, 256, seed=5)
    out, lse = acid.acid_mha_forward(q, k, v, 4)
    want = acid.acid_mha_backward(g, q, k, v, out, lse, 4)
    turned = acid.acid_rope_forward(x, 4, (64,), grid=(600,))
    bounds = torch.tensor([[0, 300]], dtype=torch.int32, device=DEV)
    part = acid.acid_mha_forward(q, k, v, 4, q_bounds=bounds, k_bounds=bounds)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    results = []
    for _ in range(3):
        for s in streams:
            how = dict(stream=s.cuda_stream if as_handle else s)
            o, l = acid.acid_mha_forward(q, k, v, 4, **how)
            results.append((o, l, *acid.acid_mha_backward(g, q, k, v, o, l, 4, **how),
                            acid.acid_rope_forward(x, 4, (64,), grid=(600,), **how),
                            *acid.acid_mha_forward(q, k, v, 4, q_bounds=bounds, k_bounds=bounds, **how)))
    torch.cuda.synchronize()
    for r in results:
        for a, b in zip(r, (out, lse, *want, turned, *part)):
            assert torch.equal(a, b)


def test_rows_far_apart(acid):
    """Row strides that put elements past 2^31: the same bits as from packed operands."""
    heads, d, ld = 1, 64, 1 << 20
    rows = 2100  # 2100 x 2^20 elements are past 2^31; the matrices are column blocks of one
    big = torch.zeros(rows, ld, dtype=B, device=DEV)
    cut = [big[:, i * 128:i * 128 + d] for i in range(8)]
    packed = [normal(rows, d, seed=i) for i in range(4)]
    for a, b in zip(cut, packed):
        a.copy_(b)
    q, k, v, g = packed
    for n in (rows, 3):  # tiles, and a few rows
        out, lse = acid.acid_mha_forward(q[-n:], k, v, heads, frame_rows=1, frames_after=0, q_first=-1)
        acid.acid_mha_forward(cut[0][-n:], cut[1], cut[2], heads, frame_rows=1, frames_after=0, q_first=-1, out=cut[4][-n:])
        assert torch.equal(cut[4][-n:], out)
    out, lse = acid.acid_mha_forward(q, k, v, heads)
    cut[4].copy_(out)
    want = acid.acid_mha_backward(g, q, k, v, out, lse, heads)
    acid.acid_mha_backward(cut[3], cut[0], cut[1], cut[2], cut[4], lse, heads, dq=cut[5], dk=cut[6], dv=cut[7])
    for a, b in zip(cut[5:], want):
        assert torch.equal(a, b)
    turned = acid.acid_rope_forward(q, 1, (64,), grid=(rows,))
    acid.acid_rope_forward(cut[0], 1, (64,), grid=(rows,), out=cut[5])
    assert torch.equal(cut[5], turned)


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("lengths", [[100, 37, 150], [1, 1, 1]])
def test_a_sequence_that_is_not_finite_keeps_to_itself(acid, dtype, lengths):
    """NaN and infinities in the middle sequence: the others' results are the bits that they are without it."""
    bounds = acid.sequence_bounds(lengths)
    n, (a, e) = sum(lengths), bounds[1].tolist()
    q, k, v, g = (normal(n, 128, dtype=dtype, seed=s) for s in range(4))
    how = dict(q_bounds=bounds, k_bounds=bounds)

    def run():
        out, lse = acid.acid_mha_forward(q, k, v, 2, **how)
        clean = torch.nan_to_num(out)
        return (out, lse.T, *acid.acid_mha_backward(g, q, k, v, clean, torch.nan_to_num(lse), 2, **how))

    want = run()
    for t in (q, k, v, g):
        t[a:e:2] = float("nan")
        t[a + 1:e:2] = float("inf")
    got = run()
    for x, y in zip(got, want):
        assert torch.equal(x[:a], y[:a]) and torch.equal(x[e:], y[e:])


def test_bounds_outside_the_operands_are_cut(acid):
    q, k, v, g = (normal(200, 128, seed=s) for s in range(4))
    out, lse = acid.acid_mha_forward(q, k, v, 2)
    want = acid.acid_mha_backward(g, q, k, v, out, lse, 2)
    b = torch.tensor([[-7, 100000]], dtype=torch.int32, device=DEV)
    o, l = acid.acid_mha_forward(q, k, v, 2, q_bounds=b, k_bounds=b)
    got = acid.acid_mha_backward(g, q, k, v, o, l, 2, q_bounds=b, k_bounds=b)
    for x, y in zip((o, l, *got), (out, lse, *want)):
        assert torch.allclose(x.float(), y.float(), atol=2.0 ** -7 * float(y.float().abs().max()))


def test_results_in_given_buffers(acid):
    """Results given as column blocks of one matrix; what lies beside them is left alone."""
    q, k, v, g = (normal(150, 128, seed=s) for s in range(4))
    out, lse = acid.acid_mha_forward(q, k, v, 2)
    want = acid.acid_mha_backward(g, q, k, v, out, lse, 2)
    wide = torch.full((150, 5 * 128 + 64), 3.0, dtype=B, device=DEV)
    cut = [wide[:, 16 + i * 144:16 + i * 144 + 128] for i in range(4)]
    acid.acid_mha_forward(q, k, v, 2, out=cut[3])
    acid.acid_mha_backward(g, q, k, v, out, lse, 2, dq=cut[0], dk=cut[1], dv=cut[2])
    for a, b in zip(cut, (*want, out)):
        assert torch.equal(a, b)
        a.fill_(3.0)
    assert (wide == 3.0).all()
