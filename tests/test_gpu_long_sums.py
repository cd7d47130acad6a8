"""Sums of hundreds of thousands of terms of one sign, which an accumulator that cuts bits off
makes too small: as they leave the experts' products in 16 bits, and inside the score.

A sum of n terms, each addition of which cuts up to 2^-24 of what is there, is off by at most n / 2 2^-24 of
itself, and by a quarter of that as a rule.  A product of more than 16,384 terms begins a new accumulator after
2,048 (1,024 2^-24 = 512 2^-23 = 6.1e-5), the score after 256 (8 2^-23).  What is stored rounds to
either side by half a step of the type at most: over 4,096 values its mean is off by a 64th of that."""

import pytest

from client_util import UNIT
from test_gpu_client import _c

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def positive(g, *shape, dtype, scale=1.0):
    return ((torch.rand(*shape, generator=g, device="cuda") + 0.5) * scale).to(dtype)


def bias(got, want):
    return abs(float((got.double() / want - 1.0).mean()))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_long_sums_in_16_bits(dtype):
    """131,072 terms in one accumulator (two parts of 262,144) would lose 4e-4."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(1)
    n, K, N = 1 << 18, 4096, 2048
    x, dy = positive(g, n, K, dtype=dtype, scale=2.0 ** -5), positive(g, n, N, dtype=dtype, scale=2.0 ** -5)
    offsets = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    most = 512 * 2.0 ** -23 + UNIT[dtype] / 64
    w = torch.zeros(1, K, N, dtype=dtype, device="cuda")
    dw = c.multiply_grad(x, w, offsets, dy, grads=(False, True)).w[0]
    assert bias(dw[:64, :64], x[:, :64].double().t() @ dy[:, :64].double()) <= most
    # As long a sum in y: the same rows as columns.
    y = c.multiply(x.t().contiguous(), dy[None], torch.tensor([0, K], dtype=torch.int32, device="cuda"))
    assert bias(y[:64, :64], x[:, :64].double().t() @ dy[:, :64].double()) <= most


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_probabilities_of_long_rows(dtype):
    """524,288 columns, every s near 20: one accumulator would make s 2e-2 and with it every
    probability 2 % too small.  Off by 8 2^-23 20 for s and as much for the log-sum-exp, 2^-20 for exp, what
    holding and storing gradients rounds, and the roundings of 2,048 parts' sum, each up to 2^-20 to either
    side: six times 2,048^1/2 2^-20 / 3^1/2."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(2)
    R, D, V = 256, 1 << 19, 2048
    z, w = positive(g, R, D, dtype=dtype, scale=2.0 ** -8), positive(g, V, D, dtype=dtype, scale=20.0 * 2.0 ** -11)
    labels = torch.zeros(R, dtype=torch.int64, device="cuda")
    s = c.score(z, w.t(), labels, upstream=torch.tensor([4096.0], device="cuda"))
    step = 1 << 16
    logits = sum(z[:, a:a + step].double() @ w[:, a:a + step].double().t() for a in range(0, D, step))
    p = torch.softmax(logits, 1)
    off = 2 * 8 * 2.0 ** -23 * 21 + 6 * (2048 / 3) ** 0.5 * 2.0 ** -20
    assert float((s.rows.double() + torch.log(p[:, 0])).abs().max()) <= off + 2.0 ** -18
    want = z[:, :512].double().t() @ p[:, 1:] * (4096.0 / R)
    assert bias(s.dw[:512, 1:], want) <= off + 2.0 ** -20 + 2 * UNIT[dtype] / 64


def test_small_products_in_fp32():
    """Sums of 4,000 terms of either sign on the ordinary cores, in parts of 256.  An addition rounds by 2^-24 of
    what is there at most, a half of that in the root of the mean square; after i terms that is i^1/2 terms, in all
    (n / 2)^1/2 2^-25 of a part of n and as much of the 16 parts: 4.2e-7 (one after the other: 1.3e-6)."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(3)
    E, K, N = 40, 4000, 256
    x, w = torch.randn(4 * E, K, generator=g, device="cuda"), torch.randn(E, K, N, generator=g, device="cuda")
    y = c.multiply(x, w, torch.arange(0, 4 * E + 1, 4, dtype=torch.int32, device="cuda"))
    want = torch.bmm(x.double().reshape(E, 4, K), w.double()).reshape(4 * E, N)
    assert float((y.double() - want).norm() / want.norm()) <= ((256 / 2) ** 0.5 + (16 / 2) ** 0.5) * 2.0 ** -25


def test_gradients_of_few_rows_in_fp32():
    """g is -1 for one class and some 1e-5 for each of the others: whatever is added after that one's part rounds by
    2^-24 of it at most.  256 such roundings to either side are 16 / 3^1/2 2^-24, the parts' sum (54 in each of 16)
    less than as much again, and g itself is off by some 2^-22."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(4)
    R, D, V = 3, 24, 220561
    w = torch.randn(D, V, generator=g, device="cuda") * 0.3
    z = torch.randn(R, D, generator=g, device="cuda")
    labels = torch.tensor([3, 100000, 220560], device="cuda")
    s = c.score(z, w, labels)
    p = torch.softmax(z.double() @ w.double(), 1)
    p[torch.arange(R), labels] -= 1.0
    want = p @ w.double().t() / R
    assert float((s.dz.double() - want).norm() / want.norm()) <= 2 * 16 / 3 ** 0.5 * 2.0 ** -24 + 2.0 ** -22
