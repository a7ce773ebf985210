"""What the rotation and the attention with row sums refuse, checked on the CPU before any device work (the pointer values
are never read), the structs' layout, and the sizes that they report."""

import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000000  # nothing reads it


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__ as g

    g.build()
    from paper_2607_12358_gb300 import _capi

    return _capi


def test_struct_layouts(tmp_path, lib):
    src = tmp_path / "p.c"
    src.write_text("""
#include <stdio.h>
#include <stddef.h>
#include "acid.h"
#define P(T) printf(#T " %zu\\n", sizeof(T));
#define O(T, f) printf(#T "." #f " %zu\\n", offsetof(T, f));
int main(void) {
  P(acid_rope) O(acid_rope, axis_dim) O(acid_rope, theta) O(acid_rope, first_rows) O(acid_rope, ld_pos) O(acid_rope, origin)
  P(acid_mha) O(acid_mha, dtype) O(acid_mha, scale) O(acid_mha, q_bounds) O(acid_mha, frame_rows) O(acid_mha, q_first)
  P(acid_mha_grads) O(acid_mha_grads, dk) O(acid_mha_grads, lddv)
  return 0;
}""")
    exe = tmp_path / "p"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split("\n"):
        if line:
            key, val = line.split()
            t, _, f = key.partition(".")
            got = getattr(getattr(lib, t), f).offset if f else C.sizeof(getattr(lib, t))
            assert got == int(val), key


def rope(A, **kw):
    a = dict(rows=100, heads=4, head_dim=64, dtype=A.ACID_BF16, axes=3, axis_dim=(24, 20, 20), theta=(1e4,) * 3, halves=0,
             first_rows=0, positions=None, ld_pos=0, grid=(5, 4, 5), origin=(0,) * 3)
    a.update(kw)
    for n, t in (("axis_dim", C.c_int32), ("theta", C.c_float), ("grid", C.c_int32), ("origin", C.c_float)):
        a[n] = (t * 4)(*a[n])
    return A.acid_rope(**a)


INVALID, UNSUPPORTED, WORKSPACE = "ACID_ERR_INVALID_ARG", "ACID_ERR_UNSUPPORTED", "ACID_ERR_WORKSPACE"


@pytest.mark.parametrize("change, status", [
    (dict(dtype=7), INVALID), (dict(rows=-1), INVALID), (dict(rows=2 ** 31 + 1), UNSUPPORTED), (dict(heads=0), INVALID),
    (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=264), UNSUPPORTED), (dict(axes=0), INVALID), (dict(axes=5), INVALID),
    (dict(axis_dim=(24, 20, 22)), INVALID), (dict(axis_dim=(24, 20, 19)), INVALID), (dict(axis_dim=(24, 20, 0)), INVALID),
    (dict(axis_dim=(24, 20, 2)), UNSUPPORTED), (dict(axis_dim=(24, 20, 12), halves=1), UNSUPPORTED),
    (dict(theta=(1e4, 0, 1e4)), INVALID), (dict(theta=(1e4, float("inf"), 1e4)), INVALID), (dict(first_rows=101), INVALID),
    (dict(first_rows=-1), INVALID), (dict(grid=(5, 0, 5)), INVALID), (dict(grid=(2 ** 20, 2 ** 20, 2)), INVALID),
    (dict(origin=(0, float("nan"), 0)), INVALID), (dict(positions=P, ld_pos=2), INVALID),
    (dict(positions=P + 2, ld_pos=3), INVALID)])
@pytest.mark.parametrize("call", ["acid_rope_forward", "acid_rope_backward"])
def test_rope_refuses(lib, call, change, status):
    f = getattr(lib.load(), call)
    assert lib.STATUS_NAMES[f(C.byref(rope(lib, **change)), P, 512, P, 512, None)] == status
    assert b"rope" in lib.load().acid_last_error()


@pytest.mark.parametrize("args, status", [
    ((None, 512, P, 512), INVALID), ((P, 512, None, 512), INVALID), ((P, 255, P, 512), INVALID), ((P, 512, P, 255), INVALID),
    ((P + 8, 512, P, 512), UNSUPPORTED), ((P, 512, P + 8, 512), UNSUPPORTED), ((P, 513, P, 512), UNSUPPORTED),
    ((P, 512, P, 516), UNSUPPORTED), ((P, 512, P, 520), INVALID)])
def test_rope_refuses_operands(lib, args, status):
    f = lib.load().acid_rope_forward
    assert lib.STATUS_NAMES[f(C.byref(rope(lib)), *args, None)] == status
    assert f(None, P, 512, P, 512, None) == lib.ACID_ERR_INVALID_ARG
    assert f(C.byref(rope(lib, rows=0)), None, 512, None, 512, None) == lib.ACID_OK  # no launch


def mha(A, **kw):
    a = dict(nq=100, nk=80, dtype=A.ACID_BF16, heads=4, kv_heads=2, head_dim=64, scale=0.125, sequences=1, q_bounds=None,
             k_bounds=None, frame_rows=0, frames_before=-1, frames_after=-1, q_first=0)
    a.update(kw)
    return A.acid_mha(**a)


MHA = [(dict(dtype=3), INVALID), (dict(nq=-1), INVALID), (dict(nk=-1), INVALID), (dict(nk=2 ** 30 + 1), UNSUPPORTED),
       (dict(heads=0), INVALID), (dict(kv_heads=3), INVALID), (dict(heads=65536 * 2, kv_heads=2), UNSUPPORTED),
       (dict(head_dim=32), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(dtype=1, head_dim=48), UNSUPPORTED),
       (dict(dtype=1, head_dim=160), UNSUPPORTED), (dict(scale=float("nan")), INVALID), (dict(sequences=0), INVALID),
       (dict(sequences=65536, q_bounds=P, k_bounds=P), INVALID), (dict(sequences=2), INVALID),
       (dict(sequences=2, q_bounds=P), INVALID), (dict(sequences=2, q_bounds=P + 4, k_bounds=P), UNSUPPORTED),
       (dict(frame_rows=-1), INVALID), (dict(frame_rows=2 ** 31), INVALID), (dict(frames_before=-2), INVALID),
       (dict(frames_after=-2), INVALID), (dict(q_first=-2), INVALID), (dict(q_first=2 ** 31), INVALID)]


def forward(A, m, q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, out=P, ldo=256, lse=P, ws=P, nws=1 << 40):
    return A.STATUS_NAMES[A.load().acid_mha_forward(C.byref(m), q, ldq, k, ldk, v, ldv, out, ldo, lse, ws, nws, None)]


def backward(A, m, dout=P, lddo=256, q=P, ldq=256, k=P, ldk=128, v=P, ldv=128, out=P, ldo=256, lse=P, dq=P, lddq=256, dk=P,
             lddk=128, dv=P, lddv=128, ws=P, nws=1 << 40):
    g = A.acid_mha_grads(dq, lddq, dk, lddk, dv, lddv)
    return A.STATUS_NAMES[A.load().acid_mha_backward(C.byref(m), dout, lddo, q, ldq, k, ldk, v, ldv, out, ldo, lse,
                                                     C.byref(g), ws, nws, None)]


@pytest.mark.parametrize("change, status", MHA)
def test_mha_refuses(lib, change, status):
    m = mha(lib, **change)
    assert forward(lib, m) == status and backward(lib, m) == status
    b = C.c_size_t()
    for f in (lib.load().acid_mha_forward_workspace_size, lib.load().acid_mha_backward_workspace_size):
        assert lib.STATUS_NAMES[f(C.byref(m), C.byref(b))] == status
    assert b"mha" in lib.load().acid_last_error()


@pytest.mark.parametrize("name", ["q", "k", "v", "out"])
def test_mha_refuses_operands(lib, name):
    m, ld = mha(lib), "ldo" if name == "out" else "ld" + name
    width = 256 if name in ("q", "out") else 128
    for call in (forward, backward):
        assert call(lib, m, **{name: None}) == INVALID
        assert call(lib, m, **{ld: width - 8}) == INVALID
        assert call(lib, m, **{ld: width + 4}) == UNSUPPORTED
        assert call(lib, m, **{name: P + 8}) == UNSUPPORTED
        assert call(lib, m, lse=None) == INVALID and call(lib, m, lse=P + 2) == INVALID


@pytest.mark.parametrize("name", ["dout", "dq", "dk", "dv"])
def test_mha_backward_refuses_gradients(lib, name):
    m, ld = mha(lib), "lddo" if name == "dout" else "ld" + name
    width = 256 if name in ("dout", "dq") else 128
    assert backward(lib, m, **{ld: width - 8}) == INVALID
    assert backward(lib, m, **{ld: width + 4}) == UNSUPPORTED
    assert backward(lib, m, **{name: P + 8}) == UNSUPPORTED
    assert backward(lib, m, dq=None, dk=None, dv=None) == INVALID
    assert backward(lib, m, dout=None) == INVALID
    assert lib.load().acid_mha_backward(C.byref(m), P, 256, P, 256, P, 128, P, 128, P, 256, P, None, P, 1 << 40,
                                        None) == lib.ACID_ERR_INVALID_ARG


def size(A, m, back):
    b = C.c_size_t()
    f = A.load().acid_mha_backward_workspace_size if back else A.load().acid_mha_forward_workspace_size
    assert f(C.byref(m), C.byref(b)) == A.ACID_OK
    return b.value


@pytest.mark.parametrize("shape", [dict(), dict(nq=1, nk=5000), dict(dtype=1), dict(nq=5000, nk=512, head_dim=128),
                                   dict(sequences=3, q_bounds=P, k_bounds=P)])
def test_mha_refuses_workspaces(lib, shape):
    m = mha(lib, **shape)
    lds = dict(ldq=512, ldk=256, ldv=256, ldo=512)
    for back in (False, True):
        need, call = size(lib, m, back), backward if back else forward
        more = dict(lds, lddo=512, lddq=512, lddk=256, lddv=256) if back else lds
        assert not back or need > 0
        if need:
            assert call(lib, m, **more, nws=need - 1) == WORKSPACE
            assert call(lib, m, **more, ws=None) == WORKSPACE
            assert call(lib, m, **more, ws=P + 8) == WORKSPACE


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    from paper_2607_12358_gb300 import acid

    x = torch.zeros(4, 128, dtype=torch.bfloat16)
    for bad in (dict(grid=(2, 2), positions=x), dict(), dict(grid=(2,)), dict(grid=(2, 2), theta=(1.0,)),
                dict(grid=(2, 2), origin=(0,))):
        with pytest.raises(ValueError):
            acid.acid_rope_forward(x, 2, (32, 32), **bad)
    with pytest.raises(ValueError):
        acid.acid_rope_forward(x, 3, (32, 32), grid=(2, 2))
    with pytest.raises(ValueError, match="CUDA"):  # on the CPU
        acid.acid_rope_forward(x, 2, (32, 32), grid=(2, 2))
    with pytest.raises(ValueError, match="CUDA"):
        acid.acid_mha_forward(x, x, x, 2)
    for heads, k in ((3, x), (2, x[:, :96]), (2, torch.zeros(4, 256, dtype=torch.bfloat16)), (0, x)):
        with pytest.raises(ValueError):
            acid.acid_mha_forward(x, k, k, heads)
    with pytest.raises(ValueError, match="int32"):
        acid.acid_mha_forward(x, x, x, 2, q_bounds=torch.zeros(1, 2, dtype=torch.int64))
    assert acid.sequence_bounds([3, 0, 5], device="cpu").tolist() == [[0, 3], [3, 3], [3, 8]]
    assert acid.sequence_bounds([3, 2], 4, device="cpu").tolist() == [[0, 3], [4, 6]]
    with pytest.raises(ValueError):
        acid.sequence_bounds([5], 4, device="cpu")


def test_clearing_of_padding_refuses(lib):
    def call(m, keys=0, a=P, lda=256, b=None, ldb=0, lse=None):
        return lib.STATUS_NAMES[lib.load().acid_mha_clear_padding(C.byref(m), keys, a, lda, b, ldb, lse, None)]

    m = mha(lib, heads=4, kv_heads=2, head_dim=64, sequences=2, q_bounds=P, k_bounds=P)
    assert call(m, lda=255) == "ACID_ERR_INVALID_ARG"
    assert call(m, lda=260) == "ACID_ERR_UNSUPPORTED"
    assert call(m, a=P + 8) == "ACID_ERR_UNSUPPORTED"
    assert call(m, b=P, ldb=128) == "ACID_ERR_INVALID_ARG"
    assert call(m, lse=P + 2) == "ACID_ERR_INVALID_ARG"
    assert call(m, keys=1, a=P, lda=128, lse=P) == "ACID_ERR_INVALID_ARG"
    assert call(mha(lib, head_dim=80)) == "ACID_ERR_UNSUPPORTED"
    assert call(m, a=None) == "ACID_OK"  # nothing to clear
    assert call(mha(lib, heads=4, kv_heads=2, head_dim=64)) == "ACID_OK"  # no padding
