"""fp32 products that are large enough to go by planes are as accurate as fp32's.

Accuracy, in the 2-norm, of sums of terms of either sign.  A value is the sum of three planes of 8 bits;
of their products those of 2^-24 and less are left out, 2^-25 of the result.  The sums are
taken out of an accumulator every 256 k; a step of 16 k cuts up to 2^-23 of what is there, half of that
on average, and after i of n steps that is some (i / n)^1/2 of the sum: (1/3) n 2^-23 for a part of n <= 16
steps, 6.4e-7.  How much each cuts varies by 12^-1/2 2^-23 of it, 16 of them by 1.2 2^-23; adding the parts up
rounds by 2^-24 of a sum each, to either side: 3 2^-23 for all of this.  Each of the three smallest
products that are taken along is some 2e-6 of the result."""

import pytest

from test_gpu_client import _c

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U23 = 2.0 ** -23


def most(steps):
    return (1 / 3 * min(16, steps) + 3) * U23


def planes(t):
    """The three planes of fp32 values, in 64 bits."""
    out, rest = [], t.double()
    for _ in range(3):
        out.append(rest.to(torch.bfloat16).double())
        rest = rest - out[-1]
    return out


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def without(a, b):
    """What a product in 64 bits loses with any one of the smallest pairs of planes that take part."""
    a3, b3 = planes(a), planes(b)
    want = a.double() @ b.double()
    return min(float((a3[i] @ b3[j]).norm() / want.norm()) for i, j in ((2, 0), (0, 2), (1, 1)))


@pytest.mark.parametrize("flip", [False, True])
def test_products_are_fp32s(flip):
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(3)
    sizes, before, behind, K, N = [700, 0, 333, 65], 3, 2, 516, 520
    n = before + sum(sizes) + behind
    assert n * K * N >= 1 << 28
    bounds = [before + sum(sizes[:e]) for e in range(len(sizes) + 1)]
    x, dy = torch.randn(n, K, generator=g, device="cuda"), torch.randn(n, N, generator=g, device="cuda")
    w = torch.randn(len(sizes), *((N, K) if flip else (K, N)), generator=g, device="cuda")
    w = w.transpose(1, 2) if flip else w
    offsets = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    y, (dx, dw) = c.multiply(x, w, offsets), c.multiply_grad(x, w, offsets, dy)
    want = [torch.zeros_like(t, dtype=torch.float64) for t in (y, dx, dw)]
    for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
        xe, we, de = x[a:b].double(), w[e].double(), dy[a:b].double()
        want[0][a:b], want[1][a:b], want[2][e] = xe @ we, de @ we.t(), xe.t() @ de
    for got, ref, steps in zip((y, dx, dw), want, (K / 16, N / 16, 700 / 16)):
        assert off(got, ref) <= most(steps), (off(got, ref), most(steps))
    assert without(x[:700], w[0]) > most(16) and without(x[:700].t(), dy[:700]) > most(16)


@pytest.mark.parametrize("w_dtype", [torch.float32, torch.bfloat16])
def test_long_sums_of_one_sign_are_fp32s(w_dtype):
    """8,192 terms: one accumulator would lose 8,192 / 32 2^-24 = 1.5e-5 of them (a step half of 2^-23 on
    average); parts of 256 lose at most 8.5 2^-23 (1 to 16 sixteenths of a part at each of 16 steps), and
    their sum 32 2^-25 or so."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(4)
    n, K, N = 8192, 256, 512
    dtype = torch.float32 if w_dtype is torch.float32 else torch.bfloat16
    x, dy = ((torch.rand(n, d, generator=g, device="cuda") + 0.5).to(dtype) for d in (K, N))
    w = torch.zeros(1, K, N, device="cuda")                  # fp32, and so is its gradient
    dw = c.multiply_grad(x, w, torch.tensor([0, n], dtype=torch.int32, device="cuda"), dy, grads=(False, True)).w[0]
    want = x.double().t() @ dy.double()
    assert float((dw.double() / want - 1.0).abs().max()) <= 8.5 * U23 + 32 * 2.0 ** -25


@pytest.mark.parametrize("flip", [False, True])
def test_losses_are_fp32s(flip):
    """Losses of some 27 made of values s of some 8 in 8 steps: of s that are off by 2/3 8 2^-23 of themselves, the
    own class's (8) and the largest (25); and the log-sum-exp's and the loss's own roundings, 2^-24 of 25 and
    27 each and exp's and log's."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(5)
    R, D, V = 4096, 128, 520
    w = torch.randn(*((V, D) if flip else (D, V)), generator=g, device="cuda") * 8.0 * D ** -0.5
    w = w.t() if flip else w
    z = torch.randn(R, D, generator=g, device="cuda")
    labels = torch.randint(0, V, (R,), generator=g, device="cuda")
    logits = z.double() @ w.double()
    want = torch.logsumexp(logits, 1) - logits.gather(1, labels[:, None])[:, 0]
    s = c.score(z, w, labels, grad=False)
    bound = (2 / 3 * 8 * U23 * (8 ** 2 + 25 ** 2) ** 0.5 + 2.0 ** -22) / 27 + 2.0 ** -23
    assert off(s.rows, want) <= bound, off(s.rows, want)
    z3, w3 = planes(z), planes(w)
    for i, j in ((2, 0), (0, 2), (1, 1)):
        less = logits - z3[i] @ w3[j]
        assert off(torch.logsumexp(less, 1) - less.gather(1, labels[:, None])[:, 0], want) > bound


@pytest.mark.parametrize("flip", [False, True])
def test_gradients_of_losses_are_fp32s(flip):
    """g is a label's -1 and, of a sixth of its size, 33 probabilities, which s, exp and the log-sum-exp make some 2^-20 off; dz
    is a sum of 3 steps of it, dw one of 256, in parts of 16."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(6)
    R, D, V = 4096, 2048, 33
    w = torch.randn(*((V, D) if flip else (D, V)), generator=g, device="cuda") * 0.3 * D ** -0.5
    w = w.t() if flip else w
    z = torch.randn(R, D, generator=g, device="cuda")
    labels = torch.randint(0, V, (R,), generator=g, device="cuda")
    p = torch.softmax(z.double() @ w.double(), 1)
    p[torch.arange(R, device="cuda"), labels] -= 1.0
    s = c.score(z, w, labels)
    assert off(s.dz, p @ w.double().t() / R) <= most(3) + 2.0 ** -20 / 6 + U23
    assert off(s.dw, z.double().t() @ p / R) <= most(16) + 2.0 ** -20 / 6 + U23
    assert without(z.t(), p.float()) > most(16) + 2.0 ** -20 / 6 + U23


def test_pieces_are_fp32s():
    """Several pieces of the classes in fp32: sums over pieces, and a short last piece."""
    from paper_1601_04033_gb300 import fasgd
    from test_gpu_score import case
    c = _c()
    R, D, V = 30000, 24, 9001
    z, w, labels = case(R, D, V, torch.float32, False)
    assert R * V * 6 > 2 * fasgd.SCORE_PIECE
    s = c.score(z, w, labels)
    dz, dw = torch.zeros(R, D, dtype=torch.float64, device="cuda"), torch.zeros(D, V, dtype=torch.float64, device="cuda")
    n = int((labels >= 0).sum())
    for a in range(0, R, 4000):
        k = torch.nonzero(labels[a:a + 4000] >= 0)[:, 0] + a
        g = torch.softmax(z[k].double() @ w.double(), 1)
        g[torch.arange(k.numel(), device="cuda"), labels[k]] -= 1.0
        dz[k] = g @ w.double().t() / n
        dw += z[k].double().t() @ g / n
    for got, want in ((s.dz, dz), (s.dw, dw)):
        assert off(got, want) <= most(16) + 2.0 ** -20, off(got, want)
