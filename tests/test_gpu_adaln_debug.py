"""The norm sites and the 4-bit operators in the debug build, which checks every hand-computed memory index against
its extent: ragged sizes of each kernel and type, results against the 64-bit definitions, and no check may fire."""

import os
import subprocess
import sys
import textwrap

import pytest

pytestmark = pytest.mark.gpu
pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = textwrap.dedent(
    r"""
    import torch

    import test_gpu_norm_site as N
    import test_gpu_q4 as Q
    from paper_2607_12358_gb300 import acid

    assert acid.bounds_report()["checked"]
    acid.selftest_bounds()
    rep = acid.bounds_report()
    assert (rep["site"], rep["index"], rep["extent"]) == (99, 1000, 1000), rep

    BF, F32 = torch.bfloat16, torch.float32
    for types in N.TYPES:
        for rows, d in ((1, 8), (37, 264), (300, 256), (45, 1920), (19, 3072), (5, 4096)):
            t, vec = N.make(rows, d, types, seed=d)
            N.both(acid, t, vec, dict(post_norm="layer", pre_norm="layer"), what=(types, rows, d))
        for rows, first, group in ((700, 3, 1), (700, 50, 33), (311, 1, 1000)):
            t, vec = N.make(rows, 520, types, seed=rows, groups=acid.norm_site_groups(rows, first, group))
            N.both(acid, t, vec, dict(first_rows=first, group_rows=group, gate_tanh=True), what=(types, rows, group))
    for m in (1, 3, 4, 5, 17, 34, 65, 130):
        for n, k, group, zeros, sdt in ((1, 31, 32, True, BF), (300, 1000, 64, False, F32), (129, 129, 128, True, BF),
                                        (520, 384, 128, False, F32), (9217, 256, 32, True, BF)):
            Q.check_both(acid, m, n, k, group, zeros, sdt, F32, F32, True)
            Q.check_both(acid, m, n, k, group, zeros, sdt, BF, BF, False, bias=False)
    for wdt in (F32, BF):
        for group in (32, 64, 128):
            for zeros in (False, True):
                Q.test_quantiser(acid, wdt, BF, group, zeros)
    acid.check_device_error()
    rep = acid.bounds_report()
    assert rep["site"] == 0, rep
    print("bounds ok")
    """
)


def test_debug_build_index_checks():
    from paper_2607_12358_gb300 import build as b

    b.build(debug=True)
    path = os.pathsep.join([ROOT, os.path.join(ROOT, "tests"), os.environ.get("PYTHONPATH", "")])
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, env=dict(os.environ, ACID_LIBRARY="debug", PYTHONPATH=path),
                       capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and "bounds ok" in r.stdout, r.stdout[-3000:] + r.stderr[-3000:]
