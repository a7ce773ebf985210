"""Operands of the norm sites and the 4-bit operators that their kernels cannot take, through the Python binding on the
CPU: stand-ins for tensors, whose addresses nothing reads, because the call is refused first."""

import math

import pytest

torch = pytest.importorskip("torch")
BF, F32 = torch.bfloat16, torch.float32


class Operand:
    """What the binding asks of a CUDA tensor."""

    is_cuda, device = True, torch.device("cpu")

    def __init__(self, shape, stride=None, dtype=F32):
        self.shape, self.dtype = torch.Size(shape), dtype
        self.strides = stride or (*(math.prod(shape[i + 1:]) for i in range(len(shape) - 1)), 1)

    def stride(self):
        return self.strides

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def data_ptr(self):
        return 0x10000000


@pytest.fixture()
def acid(monkeypatch):
    import __graft_entry__ as g

    g.build()
    from paper_2607_12358_gb300 import acid as a

    monkeypatch.setattr(a, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(a, "_current_device", lambda: 0)
    return a


def test_rows_that_overlap(acid):
    """One row expanded to many has a row stride of 0; the kernels step by at least a row."""
    q = acid.Q4Weight(Operand((96, 64), dtype=torch.uint8), Operand((96, 2)), None, 96, 128, 64)
    ws = Operand((1 << 20,), dtype=torch.uint8)
    for m in (3, 34):
        x, out = Operand((m, 128)), Operand((m, 96))
        for stride in ((0, 1), (95, 1)):
            row, wide = Operand((m, 96), stride), Operand((m, 128), stride)
            for call in (lambda: acid.acid_q4_linear_forward(wide, q, out=out, workspace=ws),
                         lambda: acid.acid_q4_linear_forward(x, q, out=row, workspace=ws),
                         lambda: acid.acid_q4_linear_backward(row, q, dx=x, want_dbias=False, workspace=ws),
                         lambda: acid.acid_q4_linear_backward(out, q, wide, silu=True, dx=x, want_dbias=False, workspace=ws),
                         lambda: acid.acid_q4_linear_backward(out, q, dx=wide, want_dbias=False, workspace=ws),
                         lambda: acid.acid_q4_quantize(wide), lambda: acid.acid_q4_dequantize(q, out=Operand((96, 128), stride))):
                with pytest.raises(acid.A.AcidError, match="row stride"):
                    call()


@pytest.mark.parametrize("first", [0, 1, 2])
def test_vectors_that_repeat_by_their_stride(acid, first):
    """A vector of stride 0 beside one of another stride: one stride is given for both."""
    names = ("gate", "scale", "shift")
    x, y = Operand((12, 256)), Operand((12, 256), dtype=BF)
    vec = {n: Operand((3, 256), (0, 1) if i == first else (768, 1)) for i, n in enumerate(names)}
    for some in (names, (names[first], names[first - 1])):
        with pytest.raises(ValueError, match="one row stride"):
            acid.acid_norm_site_forward(x, y, r=x, u=y, group_rows=4, **{n: vec[n] for n in some})
    with pytest.raises(acid.A.AcidError, match="ld_mod"):
        acid.acid_norm_site_forward(x, y, r=x, u=y, group_rows=4, **{names[first]: vec[names[first]]})


def test_groups_longer_than_the_rows(acid):
    """Lengths up to the largest number count like the rows that there are, in the library as in the binding."""
    A, n = acid.A, acid.C.c_int64()
    for rows, first, group in ((10, 0, 10), (10, 0, 1 << 62), (10, 0, (1 << 63) - 1), (10, 1, (1 << 63) - 1),
                               (10, 10, (1 << 63) - 1), (1 << 39, 5, (1 << 63) - 1), (0, 0, (1 << 63) - 1)):
        site = A.acid_norm_site(rows=rows, d=256, first_rows=first, group_rows=group)
        acid.check(acid.load().acid_norm_site_groups(acid.C.byref(site), acid.C.byref(n)))
        assert n.value == acid.norm_site_groups(rows, first, group) == (first > 0) + (rows > first), (rows, first, group)


def test_workspaces_on_the_host(acid):
    """A workspace that the GPU cannot write as one piece is refused like any other operand."""
    q = acid.Q4Weight(Operand((96, 64), dtype=torch.uint8), Operand((96, 2)), None, 96, 128, 64)
    x, g, row = Operand((34, 128)), Operand((34, 96)), Operand((34, 256))
    for bad in ("is_cuda", "is_contiguous"):
        ws = Operand((1 << 20,), dtype=torch.uint8)
        setattr(ws, bad, False if bad == "is_cuda" else lambda: False)
        for call in (lambda: acid.acid_q4_linear_forward(x, q, out=g, workspace=ws),
                     lambda: acid.acid_q4_linear_backward(g, q, dx=x, want_dbias=False, workspace=ws),
                     lambda: acid.acid_norm_site_backward(row, row, row, dx=row, dy=row, workspace=ws)):
            with pytest.raises(ValueError, match="workspace must be"):
                call()


def test_workspace_of_a_site(acid):
    """Slots of the CTAs that a width lets run, some 34 MB at most."""
    b = acid.C.c_size_t()
    for d in (8, 256, 264, 512, 1000, 1536, 1920, 4096):
        site = acid.A.acid_norm_site(rows=1 << 39, d=d)
        acid.check(acid.load().acid_norm_site_workspace_size(acid.C.byref(site), acid.C.byref(b)))
        assert 0 < b.value <= 34 << 20, d


def test_workspace_of_a_product(acid):
    """The parts of its input, whatever the weight's rows, and not the sums and parts of its gradient."""
    A, b = acid.A, acid.C.c_size_t()
    for n, k, m in ((36864, 1920, 34), (276480, 1536, 64), (36864, 1920, 2048), (9216, 1536, 5)):
        w = A.acid_q4_weight(n=n, k=k, group=64)
        acid.check(acid.load().acid_q4_linear_forward_workspace_size(acid.C.byref(w), m, acid.C.byref(b)))
        most = (m + 64) * (-(-k // 128) * 512 + 4)  # two halves of each value, whole tiles
        assert m * k * 4 <= b.value <= most, (n, k, m)
        acid.check(acid.load().acid_q4_linear_workspace_size(acid.C.byref(w), m, acid.C.byref(b)))
        assert b.value > most  # the gradient's too
    for m, want in ((0, 0), (1, 0), (4, 0), (-1, None), (32769, None)):
        status = acid.load().acid_q4_linear_forward_workspace_size(acid.C.byref(w), m, acid.C.byref(b))
        assert status == (A.ACID_ERR_INVALID_ARG if want is None else A.ACID_OK) and (want is None or b.value == want)


def test_types_of_results(acid):
    """A type that no kernel writes is refused as the other calls refuse it."""
    q = acid.Q4Weight(Operand((96, 64), dtype=torch.uint8), Operand((96, 2)), None, 96, 128, 64)
    x, g, ws = Operand((34, 128)), Operand((34, 96)), Operand((1 << 20,), dtype=torch.uint8)
    for call in (lambda: acid.acid_q4_linear_forward(x, q, out_dtype=torch.float16, workspace=ws),
                 lambda: acid.acid_q4_linear_backward(g, q, dx_dtype=torch.float16, workspace=ws),
                 lambda: acid.acid_q4_dequantize(q, torch.float16)):
        with pytest.raises(TypeError, match="unsupported dtype"):
            call()
