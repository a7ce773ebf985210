"""CPU checks of how the norm sites and the 4-bit operators are launched, on the stand-in runtime."""

from test_host_launches import libs, run  # noqa: F401

CALLS = r"""
def site(rows, d, ts, tb, groups):
    return A.acid_norm_site(rows=rows, d=d, stream_dtype=ts, branch_dtype=tb, post_norm=1, pre_norm=2, gate_tanh=0, eps=1e-6,
                            res_scale=1.0, branch_scale=1.0, first_rows=0, group_rows=-(-rows // groups) if groups > 1 else 0,
                            gate=p[6], scale=p[7], shift=p[8], ld_mod=d, post_w=p[9], pre_w=p[10])
def forward(rows, d, ts=A.ACID_FP32, tb=A.ACID_BF16, groups=1, y=True):
    s = site(rows, d, ts, tb, groups)
    return lib.acid_norm_site_forward(C.byref(s), p[0], d, p[1] if y else None, d, p[2], d, p[3], d, None)
def backward(rows, d, ts=A.ACID_FP32, tb=A.ACID_BF16, groups=1):
    s = site(rows, d, ts, tb, groups)
    g = A.acid_norm_site_grads(p[4], d, p[5], d, p[11], p[12], p[13], d, p[14], p[15])
    return lib.acid_norm_site_backward(C.byref(s), p[0], d, p[1], d, p[2], d, p[3], d, C.byref(g), p[6], 1 << 40, None)
def weight(n, k, group, zeros, sdt): return A.acid_q4_weight(p[1], p[2], p[3] if zeros else None, n, k, group, sdt)
def linear4(m, n, k, group=128, zeros=False, sdt=A.ACID_BF16, t=A.ACID_FP32):
    w = weight(n, k, group, zeros, sdt)
    return lib.acid_q4_linear_forward(t, p[0], k, m, C.byref(w), p[4], 1, t, p[5], n, p[6], 1 << 40, None)
def linear4_back(m, n, k, group=128, zeros=False, sdt=A.ACID_BF16, t=A.ACID_FP32):
    w = weight(n, k, group, zeros, sdt)
    return lib.acid_q4_linear_backward(t, p[0], n, m, C.byref(w), t, p[4], k, 1, p[5], k, p[7], p[6], 1 << 40, None)
B, F = A.ACID_BF16, A.ACID_FP32
"""


def test_shared_memory_opt_in_on_every_device(libs):  # noqa: F811
    """Every kernel's opt-in is made on each device that it is launched on, and made again after it failed."""
    run(CALLS + """
calls = [lambda d=d, i=i, o=o, y=y: forward(5000, d, i, o, 3, y) for d in (256, 1536, 4096) for i in (B, F) for o in (B, F) for y in (0, 1)]
calls += [lambda d=d, i=i, o=o: backward(5000, d, i, o, 3) for d in (256, 1536, 4096) for i in (B, F) for o in (B, F)]
for f in (linear4, linear4_back):
    calls += [lambda f=f, m=m, g=g, z=z, s=s, t=t: f(m, 520, 1536, g, z, s, t) for m in (1, 4, 5, 17, 34, 65, 200)
              for g in (32, 64, 128) for z in (0, 1) for s in (B, F) for t in (B, F)]
fk.attribute_error = 1
for i, f in enumerate(calls):
    assert f() in (A.ACID_OK, A.ACID_ERR_CUDA), i  # below 48 KB nothing has to be asked for
fk.attribute_error = 0
for dev in (0, 1, 0):
    fk.device = dev
    for i, f in enumerate(calls):
        assert f() == A.ACID_OK, (dev, i, lib.acid_last_error())
""", *libs)


def test_grids_follow_the_device(libs):  # noqa: F811
    """Persistent grids are sized to the SMs of the device that the call runs on."""
    run(CALLS + """
for dev, sms in ((0, 152), (1, 100), (0, 152)):
    fk.device = dev
    fk.launches = 0
    assert forward(1000000, 4096) == A.ACID_OK and fk.grid % sms == 0 and fk.launches == 1
""", *libs)


def test_small_and_empty_calls(libs):  # noqa: F811
    """One launch for a few rows, which need no workspace; none where there is nothing to do."""
    run(CALLS + """
w = weight(9216, 1536, 128, False, B)
call = lambda m, ws, size: lib.acid_q4_linear_forward(F, p[0], 1536, m, C.byref(w), p[4], 1, F, p[5], 9216, ws, size, None)
assert call(1, None, 0) == A.ACID_OK and call(4, None, 0) == A.ACID_OK and fk.launches == 2
assert call(5, None, 0) == A.ACID_ERR_WORKSPACE and call(5, p[6], 16) == A.ACID_ERR_WORKSPACE and fk.launches == 2
fk.launches = 0
assert call(0, None, 0) == A.ACID_OK and forward(0, 256) == A.ACID_OK and fk.launches == 0
""", *libs)
