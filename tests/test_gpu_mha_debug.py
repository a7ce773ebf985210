"""Rotary positions and attention with row sums in the debug build, which checks every hand-computed memory index
against its extent: the value tests' cases, and no check may fire."""

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

    import test_gpu_mha as M
    import test_gpu_rope as R
    from paper_2607_12358_gb300 import acid

    assert acid.bounds_report()["checked"]
    acid.selftest_bounds()
    rep = acid.bounds_report()
    assert (rep["site"], rep["index"], rep["extent"]) == (99, 1000, 1000), rep
    for args, how in M.CASES.values():
        M.forward(acid, M.Case(*args, **how))
        M.backward(acid, M.Case(*args, seed=1, **how))
    for case in R.CASES:
        for dtype in (torch.bfloat16, torch.float32):
            R.test_grid(acid, case, dtype)
    R.test_in_place(acid, torch.bfloat16, True)
    R.test_positions_near_and_far(acid, 1e4, False)
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
