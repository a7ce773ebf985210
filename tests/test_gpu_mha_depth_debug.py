"""Attention with row sums and its gradient in the debug build on more items than the GPU has SMs: several units of every
CTA, shares of items, the last wave, parts and their joins, with every index checked."""

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

    import test_gpu_mha_depth as D
    import test_gpu_mha_use as U
    from paper_2607_12358_gb300 import acid

    assert acid.bounds_report()["checked"]
    torch.set_default_dtype(torch.float32)
    for args, how in D.FORWARD.values():
        D.forward(acid, D.Case(*args, seed=2, **how))
    for args, how in D.BACKWARD.values():
        D.backward(acid, D.Case(*args, seed=3, **how))
    U.test_rows_far_apart(acid)
    U.test_bounds_outside_the_operands_are_cut(acid)
    for dtype in (torch.bfloat16, torch.float32):
        U.test_a_sequence_that_is_not_finite_keeps_to_itself(acid, dtype, [1, 1, 1])
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
