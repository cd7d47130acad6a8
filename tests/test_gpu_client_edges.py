"""Client operators at edges that one call alone does not show: what earlier launches
left in shared memory."""

import pytest

from test_gpu_client import _c, draws, make

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
