"""Client operators at edges: what earlier launches left in shared memory, first calls
on many threads, gradients that are not finite."""

import pytest

from test_gpu_client import _c, draws, make, routed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [3, 8, 40, 41, 64])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_narrow_gradients_whatever_ran_before(D, norm, dtype):
    """Rows of up to 64 columns, four to a warp, where some of the four are fewer rows
    than the others: their gradients do not depend on the statistics that other rows
    (of NaN, of zeros) left in every SM's shared memory."""
    import torch
    c = _c()

    def leave(value):
        a, dh, dz = make(8 * 152 * 16 * 4, D, dtype, norm, groups=1)
        a["x"].fill_(value)
        a["y"].fill_(value)
        j = c.join(**a, norm=norm)
        return lambda: c.join_grad(j, dh, dz)

    nans, zeros = leave(float("nan")), leave(0.0)
    for R, groups in ((1, 1), (2, 1), (3, 1), (5, 1), (33, 1), (1001, 1), (9733, 1), (21, 3), (655, 5), (13, 13),
                      (3 * 65, 3), (7 * 1031, 7)):
        a, dh, dz = make(R, D, dtype, norm, groups=groups)
        j = c.join(**a, norm=norm, draws=draws(0.2))
        zeros()
        want = c.join_grad(j, dh, dz)
        nans()
        got = c.join_grad(j, dh, dz)
        for name, w, g in zip(want._fields, want, got):
            if w is not None:
                assert torch.isfinite(g.float()).all() and torch.equal(g, w), (R, groups, name)


FIRST_CALLS = r"""
import sys, threading, torch
sys.path.insert(0, "tests")
from test_gpu_client import make
from paper_1601_04033_gb300 import client as c
sets = []
for D in (4096, 264, 2048, 1024, 4088, 520, 8192, 5000):      # what they need of shared memory differs
    for dtype in ("float32", "bfloat16"):
        for norm in ("rms", "layer"):
            sets.append((norm, *make(40, D, dtype, norm, groups=1)))
            sets.append((norm, *make(40, D, dtype, norm, groups=1, pad=3)))
torch.cuda.synchronize()
out, errors, meet = [None] * len(sets), [], threading.Barrier(len(sets))

def call(i):
    norm, a, dh, dz = sets[i]
    try:
        meet.wait(60)
        j = c.join(**a, norm=norm)
        out[i] = [j.h, j.z, *c.join_grad(j, dh, dz)]
    except Exception as e:
        errors.append((i, e))

threads = [threading.Thread(target=call, args=(i,)) for i in range(len(sets))]
[t.start() for t in threads]
[t.join() for t in threads]
assert not errors, errors
for i, (norm, a, dh, dz) in enumerate(sets):
    j = c.join(**a, norm=norm)
    for got, want in zip(out[i], [j.h, j.z, *c.join_grad(j, dh, dz)]):
        assert got is want is None or torch.equal(got, want), i
print("same")
"""


def test_first_calls_of_many_threads():
    """A process whose first joins come on many threads at once, of widths that need
    more and less shared memory of the same kernels."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.endswith("same\n"), r.stderr[-3000:]


@pytest.mark.parametrize("E, pad", [(5, 0), (8, 0), (60, 0), (60, 3), (256, 0), (500, 4), (1024, 0)])
@pytest.mark.parametrize("up", [float("inf"), float("nan")])
def test_rows_that_take_no_part_have_no_gradient_whatever_it_is_times(E, pad, up):
    """The gradient of a row that is not valid is 0, not upstream * 0."""
    import torch
    for dtype in ("float32", "bfloat16"):
        for groups in (1, 3):
            logits, chosen, valid = routed(120, E, 2, dtype, groups=groups, ragged=groups > 1, pad=pad)
            if valid is None:
                valid = torch.arange(120, device="cuda") % 3 > 0
            b = _c().balance(logits, chosen, groups=groups, valid=valid, z=0.1,
                             upstream=torch.full((1,), up, device="cuda"))
            assert (b.dlogits[~valid] == 0).all() and not torch.isfinite(b.dlogits[valid]).all()
            assert torch.isfinite(b.loss).all()
