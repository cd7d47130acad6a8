"""Infinities in products and scores: large fp32 products, which go by planes, make of them what
small ones and the definition make."""

import pytest

from test_gpu_client import _c

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U23 = 2.0 ** -23


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def signs(t):
    """What is infinite, of which sign, and what is not a number."""
    return torch.where(t.isnan(), 2.0, torch.where(t.isinf(), t.sign(), 0.0)).float()


@pytest.mark.parametrize("rows", [40, 1103])
@pytest.mark.parametrize("flip", [False, True])
def test_infinities_are_fp32s(flip, rows):
    """Of small products and large ones: an infinity times a number is an infinity of the sign that it
    should have; NaN comes of infinities that meet a zero or each other, as in the definition."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(7)
    K, N = 516, 520
    x, dy = torch.randn(rows, K, generator=g, device="cuda"), torch.randn(rows, N, generator=g, device="cuda")
    w = torch.randn(2, *((N, K) if flip else (K, N)), generator=g, device="cuda")
    w = w.transpose(1, 2) if flip else w
    first = rows * 2 // 3
    inf = float("inf")
    w[0, 7, 50], w[0, 7, 51], w[0, 7, 52], w[0, 7, 53] = 1.0, -0.5, 0.0, 1.0 + 2.0 ** -20
    x[5, 7], x[6, 8], x[7, 9], x[7, 10] = inf, -inf, inf, -inf
    w[0, 11, 60], w[1, 12, 61] = -inf, inf
    x[8, 11], x[9, 11] = 0.0, 2.0
    dy[first + 2, 30], dy[3, 31] = inf, -inf
    x[first + 2, 40], w[1, 41, 30] = 3.0, 0.0
    offsets = torch.tensor([0, first, rows], dtype=torch.int32, device="cuda")
    y, (dx, dw) = c.multiply(x, w, offsets), c.multiply_grad(x, w, offsets, dy)
    for e, (a, b) in enumerate(((0, first), (first, rows))):
        xe, we, de = x[a:b].double(), w[e].double(), dy[a:b].double()
        for got, want in ((y[a:b], xe @ we), (dx[a:b], de @ we.t()), (dw[e], xe.t() @ de)):
            assert torch.equal(signs(got), signs(want)) and bool(signs(want).any())


@pytest.mark.parametrize("flip", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [64, 4096])
def test_classes_that_are_shut(rows, dtype, flip):
    """A column of ones in z and -inf under it in w shut a class: it takes no part in the losses, nor in
    gradients but those of the ones, where 0 times -inf is NaN."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(8)
    D, V = 128, 520
    w = (torch.randn(*((V, D) if flip else (D, V)), generator=g, device="cuda") * D ** -0.5).to(dtype)
    w = w.t() if flip else w
    z = torch.randn(rows, D, generator=g, device="cuda").to(dtype)
    z[:, 5] = 1.0
    shut = torch.rand(V, generator=g, device="cuda") < 0.3
    shut[300:400] = True
    w[5, shut] = -float("inf")
    open_ = torch.nonzero(~shut)[:, 0]
    labels = open_[torch.randint(0, open_.numel(), (rows,), generator=g, device="cuda")]
    s = c.score(z, w, labels)
    logits = z.double() @ w[:, open_].double()
    want = torch.logsumexp(logits, 1) - logits.gather(1, torch.searchsorted(open_, labels)[:, None])[:, 0]
    # D 2^-23 sum |z| |w| for s, twice; some 2^-20 for the log-sum-exp's parts.
    bound = 2 * D * U23 * (z.double().abs() @ w[:, open_].double().abs()).max(1).values + 2.0 ** -20 * (1 + want)
    assert bool(((s.rows.double() - want).abs() <= bound).all())
    p = torch.softmax(logits, 1)
    p[torch.arange(rows, device="cuda"), torch.searchsorted(open_, labels)] -= 1.0
    dw, rest = z.double().t() @ p / rows, torch.arange(D, device="cuda") != 5
    dz = p @ w[:, open_].double().t() / rows
    # g's and the results' roundings, in the 2-norm.
    u = 2 * torch.finfo(dtype).eps / 2 + 1e-5
    assert not s.dw[:, shut].any() and off(s.dw[:, open_], dw) <= u
    assert s.dz[:, 5].isnan().all() and off(s.dz[:, rest], dz[:, rest]) <= u


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows, cols, classes", [(40, 24, 10), (64, 128, 520), (700, 128, 3100), (4096, 128, 520)])
def test_losses_of_infinite_values(rows, cols, classes, dtype):
    """A class of infinite value: the loss of another one is infinite, its own is no number, and rows that it
    shuts or leaves alone have theirs; whichever kernels the size takes."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(9)
    w = (torch.randn(cols, classes, generator=g, device="cuda") * cols ** -0.5).to(dtype)
    z = torch.randn(rows, cols, generator=g, device="cuda").to(dtype)
    w[5, 7], w[5, 8:] = float("inf"), 0.0
    z[:, 5] = torch.tensor([1.0, -1.0], device="cuda").repeat(rows // 2).to(dtype)
    w[5, :7] = 0.0
    labels = torch.randint(0, 7, (rows,), generator=g, device="cuda")
    labels[:8] = 7
    labels[8:12] = classes - 1
    s = c.score(z, w, labels, grad=False)
    logits = z.double() @ w.double()
    want = torch.logsumexp(logits, 1) - logits.gather(1, labels[:, None])[:, 0]
    assert torch.equal(signs(s.rows), signs(want))
    assert want[0].isnan() and want[1].isposinf() and want[8].isposinf() and want[9].isfinite()
    on = want.isfinite()
    rest = torch.arange(cols, device="cuda") != 5
    size = z[:, rest].double().abs() @ w[rest].double().abs()
    bound = 2 * cols * U23 * size.max(1).values + 2.0 ** -20 * (1 + want.abs())
    assert bool(((s.rows.double() - want).abs() <= bound)[on].all()) and bool(on.any())
    assert s.loss.isnan().all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows, classes", [(40, 10), (64, 520), (500, 4200), (700, 3100), (4096, 520)])
def test_shut_classes_and_rows_without_labels(rows, classes, dtype):
    """Rows without a label take no part where classes are shut either: the gradients are those of the
    others' alone, and zeros in their place."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(10)
    cols = 128
    w = (torch.randn(cols, classes, generator=g, device="cuda") * cols ** -0.5).to(dtype)
    z = torch.randn(rows, cols, generator=g, device="cuda").to(dtype)
    z[:, 5] = 1.0
    shut = torch.arange(classes, device="cuda") % 3 == 1
    w[5, shut] = -float("inf")
    labels = torch.randint(0, (classes - 1) // 3, (rows,), generator=g, device="cuda") * 3
    labels[torch.rand(rows, generator=g, device="cuda") < 0.3] = -1
    on = labels >= 0
    s = c.score(z, w, labels)
    logits = z[on].double() @ w[:, ~shut].double()
    p = torch.softmax(logits, 1)
    at = torch.cumsum(~shut, 0)[labels[on]] - 1
    p[torch.arange(p.shape[0], device="cuda"), at] -= 1.0
    n, rest = p.shape[0], torch.arange(cols, device="cuda") != 5
    # g's and the results' roundings, in the 2-norm.
    u = 2 * torch.finfo(dtype).eps / 2 + 1e-5
    assert s.rows.isfinite().all() and not s.rows[~on].any()
    assert not s.dw[:, shut].any() and off(s.dw[:, ~shut], z[on].double().t() @ p / n) <= u
    assert not s.dz[~on].any() and off(s.dz[on][:, rest], (p @ w[:, ~shut].double().t() / n)[:, rest]) <= u
