"""The score of few classes over more rows than its blocks take in one turn."""

import pytest

from test_gpu_client import _c
from test_gpu_score import TYPES, case, check

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, cols, classes", [(1216 * 5 + 3, 45, 10), (1216 * 2, 97, 32), (1217, 1, 2)])
def test_turns_over_the_rows(rows, cols, classes, dtype):
    """Half of the rows have no label, so that a warp's next row is one that it does not look at: either
    gradient alone, and both from what is known, are what the whole call gives, bit for bit."""
    c = _c()
    z, w, labels = case(rows, cols, classes, dtype, False, drop=0.5)
    s = check(c, z, w, labels)
    e = c.score(z, w, labels, grad=False)
    assert torch.equal(e.loss, s.loss) and torch.equal(e.rows, s.rows)
    for known in (None, e):
        for _ in range(5):
            only = c.score(z, w, labels, grads=(True, False), known=known)
            assert only.dw is None and torch.equal(only.dz, s.dz)
        only = c.score(z, w, labels, grads=(False, True), known=known)
        assert only.dz is None and torch.equal(only.dw, s.dw)
        t = c.score(z, w, labels, known=known)
        assert torch.equal(t.dz, s.dz) and torch.equal(t.dw, s.dw)
    leaf = z.detach().requires_grad_(True)
    c.scored(leaf, w, labels)[0].backward()
    assert torch.equal(leaf.grad, s.dz)
