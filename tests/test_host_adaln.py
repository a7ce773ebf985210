"""What the norm-site and 4-bit entry points refuse, checked on the CPU before
any device work (the pointer values are never read), and the sizes that they report."""

import ctypes as C
import math
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__ as g

    g.build()
    from paper_2607_12358_gb300 import _capi

    return _capi


P = 0x10000000  # nothing reads it


def site(A, **kw):
    a = dict(rows=100, d=256, stream_dtype=A.ACID_FP32, branch_dtype=A.ACID_BF16, post_norm=1, pre_norm=2, gate_tanh=0,
             eps=1e-6, res_scale=1.0, branch_scale=1.0, first_rows=0, group_rows=0, gate=P, scale=P, shift=P, ld_mod=256,
             post_w=None, pre_w=None)
    a.update(kw)
    return A.acid_norm_site(**a)


def test_struct_layouts(tmp_path, lib):
    src = tmp_path / "p.c"
    src.write_text("""
#include <stdio.h>
#include <stddef.h>
#include "acid.h"
#define P(T) printf(#T " %zu\\n", sizeof(T));
#define O(T, f) printf(#T "." #f " %zu\\n", offsetof(T, f));
int main(void) {
  P(acid_norm_site) O(acid_norm_site, first_rows) O(acid_norm_site, gate) O(acid_norm_site, ld_mod) O(acid_norm_site, pre_w)
  P(acid_norm_site_grads) O(acid_norm_site_grads, dgate) O(acid_norm_site_grads, dpre_w)
  P(acid_q4_weight) O(acid_q4_weight, n) O(acid_q4_weight, scale_dtype)
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


def test_groups_and_workspace(lib):
    A, L = lib, lib.load()
    n, b = C.c_int64(), C.c_size_t()
    for kw, want in ((dict(), 1), (dict(first_rows=100), 1), (dict(first_rows=99), 2), (dict(group_rows=30), 4),
                     (dict(first_rows=10, group_rows=30), 4), (dict(rows=0), 0), (dict(group_rows=1), 100)):
        assert L.acid_norm_site_groups(C.byref(site(A, **kw)), C.byref(n)) == A.ACID_OK and n.value == want, kw
    assert L.acid_norm_site_workspace_size(C.byref(site(A, rows=1 << 39)), C.byref(b)) == A.ACID_OK
    assert 0 < b.value < 1 << 28
    assert L.acid_norm_site_groups(C.byref(site(A)), None) == A.ACID_ERR_INVALID_ARG
    assert L.acid_norm_site_workspace_size(None, C.byref(b)) == A.ACID_ERR_INVALID_ARG
    for k, want in ((1, 64), (128, 64), (129, 128), (1536, 768)):
        assert L.acid_q4_row_bytes(k, C.byref(b)) == A.ACID_OK and b.value == want
    assert L.acid_q4_row_bytes(0, C.byref(b)) == A.ACID_ERR_INVALID_ARG


def test_site_refusals(lib):
    A, L = lib, lib.load()
    INV, UNS, WS = A.ACID_ERR_INVALID_ARG, A.ACID_ERR_UNSUPPORTED, A.ACID_ERR_WORKSPACE

    def fwd(x=P, ldx=256, y=P, ldy=256, r=P, ldr=256, u=P, ldu=256, **kw):
        return L.acid_norm_site_forward(C.byref(site(A, **kw)), x, ldx, y, ldy, r, ldr, u, ldu, None)

    bad = [(dict(stream_dtype=2), INV), (dict(branch_dtype=-1), INV), (dict(post_norm=3), INV), (dict(pre_norm=-1), INV),
           (dict(rows=-1), INV), (dict(d=0), INV), (dict(d=250), UNS), (dict(d=4104), UNS), (dict(first_rows=101), INV),
           (dict(first_rows=-1), INV), (dict(group_rows=-1), INV), (dict(eps=-1e-6), INV), (dict(eps=math.nan), INV),
           (dict(group_rows=50, ld_mod=255), INV), (dict(group_rows=50, ld_mod=258), INV), (dict(gate=P + 4), UNS),
           (dict(pre_w=P + 8), UNS)]
    for kw, want in bad:
        assert fwd(**kw) == want, kw
        assert L.acid_last_error()
    assert L.acid_norm_site_forward(None, P, 256, P, 256, P, 256, P, 256, None) == INV
    for kw, want in ((dict(x=None), INV), (dict(r=None, u=None), INV), (dict(ldx=255), INV), (dict(ldu=200), INV),
                     (dict(x=P + 8), UNS), (dict(ldy=260), UNS), (dict(u=P + 2), UNS)):
        assert fwd(**kw) == want, kw
    assert fwd(rows=0, x=None, y=None, r=None, u=None) == A.ACID_OK

    def bwd(du=P, r=P, y=P, dr=P, ld=256, ws=P, n=1 << 30, grads=None, **kw):
        o = dict(dx=P, lddx=256, dy=P, lddy=256, dgate=P, dscale=P, dshift=P, ld_dmod=256, dpost_w=P, dpre_w=P)
        o.update(grads or {})
        return L.acid_norm_site_backward(C.byref(site(A, **kw)), du, ld, r, 256, y, 256, dr, 256,
                                         C.byref(A.acid_norm_site_grads(**o)), ws, n, None)

    for kw, want in ((dict(du=None, dr=None), INV), (dict(du=None), INV), (dict(r=None), INV), (dict(y=None), INV),
                     (dict(ld=8), INV), (dict(ws=None), WS), (dict(ws=P + 4), WS), (dict(n=100), WS),
                     (dict(group_rows=50, grads=dict(ld_dmod=100)), INV), (dict(grads=dict(dgate=P + 4)), UNS),
                     (dict(grads=dict(lddx=250)), INV), (dict(grads=dict(dy=P + 8)), UNS)):
        assert bwd(**kw) == want, kw
    assert L.acid_norm_site_backward(C.byref(site(A)), P, 256, P, 256, P, 256, P, 256, None, P, 1 << 30, None) == INV


def test_q4_refusals(lib):
    A, L = lib, lib.load()
    INV, UNS, WS = A.ACID_ERR_INVALID_ARG, A.ACID_ERR_UNSUPPORTED, A.ACID_ERR_WORKSPACE

    def weight(**kw):
        a = dict(packed=P, scales=P, zeros=None, n=100, k=256, group=64, scale_dtype=A.ACID_BF16)
        a.update(kw)
        return C.byref(A.acid_q4_weight(**a))

    def fwd(xt=A.ACID_FP32, x=P, ldx=256, m=3, bias=None, ot=A.ACID_FP32, out=P, ldo=100, ws=None, nws=0, **kw):
        return L.acid_q4_linear_forward(xt, x, ldx, m, weight(**kw), bias, 1, ot, out, ldo, ws, nws, None)

    for kw, want in ((dict(n=0), INV), (dict(n=1 << 31), INV), (dict(k=0), INV), (dict(k=65537), INV),
                     (dict(group=48), UNS), (dict(group=0), UNS), (dict(scale_dtype=3), INV), (dict(packed=None), INV),
                     (dict(scales=None), INV), (dict(packed=P + 4), UNS), (dict(scales=P + 1), UNS),
                     (dict(n=(1 << 31) - 1, k=65536, ldx=65536, ldo=1 << 31), UNS), (dict(xt=5), INV), (dict(x=None), INV),
                     (dict(x=P + 2), UNS), (dict(ldx=255), INV), (dict(m=-1), INV), (dict(m=32769), INV),
                     (dict(ot=7), INV), (dict(out=None), INV), (dict(ldo=99), INV), (dict(bias=P + 2), UNS),
                     (dict(m=5), WS), (dict(m=5, ws=P + 8, nws=1 << 20), WS), (dict(m=5, ws=P, nws=100), WS)):
        assert fwd(**kw) == want, kw
        assert L.acid_last_error()
    assert fwd(m=0, x=None, out=None) == A.ACID_OK
    assert L.acid_q4_linear_forward(A.ACID_FP32, P, 256, 3, None, None, 0, A.ACID_FP32, P, 100, None, 0, None) == INV
    b = C.c_size_t()
    assert L.acid_q4_linear_workspace_size(weight(), 5, C.byref(b)) == A.ACID_OK and b.value > 0
    assert L.acid_q4_linear_workspace_size(weight(), -1, C.byref(b)) == INV
    need = b.value

    def bwd(gt=A.ACID_FP32, g=P, ldg=100, m=5, xt=A.ACID_FP32, x=P, ldx=256, silu=1, dx=P, lddx=256, db=P, ws=P, n=need,
            **kw):
        return L.acid_q4_linear_backward(gt, g, ldg, m, weight(**kw), xt, x, ldx, silu, dx, lddx, db, ws, n, None)

    for kw, want in ((dict(gt=9), INV), (dict(g=None), INV), (dict(ldg=99), INV), (dict(m=-1), INV), (dict(x=None), INV),
                     (dict(dx=None, db=None), INV), (dict(lddx=255), INV), (dict(dx=P + 1), UNS), (dict(db=P + 1), UNS),
                     (dict(ws=None), WS), (dict(ws=P + 8), WS), (dict(n=need - 1), WS), (dict(packed=None), INV)):
        assert bwd(**kw) == want, kw
    for call in (lambda **kw: L.acid_q4_quantize(A.ACID_BF16, P, 256, weight(**kw), None),
                 lambda **kw: L.acid_q4_dequantize(weight(**kw), A.ACID_BF16, P, 256, None)):
        for kw, want in ((dict(group=16), UNS), (dict(packed=None), INV), (dict(n=-4), INV), (dict(packed=P + 8), UNS)):
            assert call(**kw) == want, kw
    assert L.acid_q4_quantize(A.ACID_BF16, P, 255, weight(), None) == INV
    assert L.acid_q4_quantize(4, P, 256, weight(), None) == INV
    assert L.acid_q4_dequantize(weight(), A.ACID_FP32, None, 256, None) == INV
