"""fasgd_score (softmax cross entropy from the last product on) against its definition in
64 bits.

Bounds.  s is off by ds = D 2^-23 sum |z| |w| (a sum of D products in fp32, additions that
round or cut), and so is the log-sum-exp, to which exp and log add some 2^-21 of 1 and of
the values' size.  A g = exp(s - lse) - [label] is off by p (2 ds + 2^-20 + 2^-22 |lse|), and
for 16-bit types by its rounding; the products' sums of V and R terms as any sum."""

import pytest

from client_util import TINY, UNIT
from test_gpu_client import _c

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = [torch.float32, torch.bfloat16, torch.float16]
U23 = 2.0 ** -23


def case(R, D, V, dtype, flip, pad=0, drop=0.1, scale=2.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + R + D + V)
    w = (torch.randn(*((V, D) if flip else (D, V)), generator=g, device="cuda") * scale * D ** -0.5).to(dtype)
    w = w.t() if flip else w
    labels = torch.randint(0, V, (R,), generator=g, device="cuda")
    z = torch.randn(R, D, generator=g, device="cuda") + torch.rand(R, 1, generator=g, device="cuda") * 3.0 * w[:, labels].t().float()
    wide = torch.full((R, D + pad), float("nan"), device="cuda", dtype=dtype)
    wide[:, :D] = z
    if drop:
        labels[torch.rand(R, generator=g, device="cuda") < drop] = -1
    return wide[:, :D], w, labels


def check(c, z, w, labels, upstream=None):
    V, R, D = w.shape[1], z.shape[0], z.shape[1]
    up = None if upstream is None else torch.tensor([upstream], device="cuda")
    s = c.score(z, w, labels, upstream=up)
    kept = (labels >= 0) & (labels < V)
    k = torch.nonzero(kept)[:, 0]
    z64, w64, y = z[k].double(), w.double(), labels[k]
    logits = z64 @ w64
    ds = D * U23 * (z64.abs() @ w64.abs())
    lse = torch.logsumexp(logits, 1)
    p = torch.exp(logits - lse[:, None])
    at = logits.gather(1, y[:, None])[:, 0]
    want = lse - at
    dlse = (p * ds).sum(1) + 2.0 ** -21 * (1 + lse.abs())
    off = dlse + ds.gather(1, y[:, None])[:, 0] + 2.0 ** -22 * (lse.abs() + at.abs() + 1)
    rows = s.rows.double()
    assert not rows[~kept].any()
    assert bool(((rows[k] - want).abs() <= off).all()), float(((rows[k] - want).abs() - off).max())
    assert bool(((s.lse.double()[k] - lse).abs() <= off).all())
    assert s.dz.isfinite().all() and s.dw.isfinite().all()
    n = max(1, k.numel())
    assert abs(float(s.loss) - float(want.sum() / n)) <= float(off.sum() / n + 2.0 ** -20 * (want.abs().sum() / n)) + 1e-30
    # gradients
    u = UNIT[z.dtype]
    share = (1.0 if upstream is None else upstream) / n if k.numel() else 0.0
    g = p.clone()
    g[torch.arange(k.numel(), device="cuda"), y] -= 1.0
    dg = p * (ds + dlse[:, None] + 2.0 ** -20) + (0.0 if z.dtype is torch.float32 else u * g.abs() + TINY[z.dtype] / 16384) + 2.0 ** -23 * g.abs()
    dz, dw = torch.zeros(R, D, dtype=torch.float64, device="cuda"), z64.t() @ g * share
    bz = torch.zeros_like(dz)
    dz[k] = g @ w64.t() * share
    bz[k] = (dg @ w64.abs().t() + (V + 8) * U23 * (g.abs() @ w64.abs().t())) * abs(share)
    bw = (z64.abs().t() @ dg + (R + 8) * U23 * (z64.abs().t() @ g.abs())) * abs(share)
    assert not s.dz[~kept].any()
    for name, got, ref, b in (("dz", s.dz, dz, bz), ("dw", s.dw, dw, bw)):
        bound = b * (1 + u) + u * ref.abs() + TINY[got.dtype]
        off = (got.double() - ref).abs()
        assert bool((off <= bound).all()), (name, float((off - bound).max()), float(off.max()))
    assert s.dw.stride() == torch.empty_like(w).stride()
    return s


SIZES = [(1, 1, 2), (1, 64, 1), (1, 4096, 1000), (2, 8, 9), (128, 200, 10), (127, 96, 64), (129, 72, 257), (300, 129, 1021), (64, 1000, 512),
         (513, 40, 3000), (5, 256, 20000), (1000, 264, 255), (259, 517, 1555)]


@pytest.mark.parametrize("flip", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_score(size, dtype, flip):
    check(_c(), *case(*size, dtype, flip))


@pytest.mark.parametrize("dtype", TYPES)
def test_layouts(dtype):
    """Rows apart, odd addresses, gradients into other layouts, an upstream value."""
    c = _c()
    for pad in (3, 8):
        z, w, labels = case(200, 136, 520, dtype, False, pad)
        s = check(c, z, w, labels, 2.5)
        wide = torch.full((137, 600), float("nan"), device="cuda", dtype=dtype)
        inner = wide[:136, pad:pad + 520]
        inner.copy_(w)
        into = torch.empty(200, 150, device="cuda", dtype=dtype)[:, 7:143], torch.empty(136, 531, device="cuda", dtype=dtype)[:, 1:521]
        t = c.score(z, inner, labels, upstream=torch.tensor([2.5], device="cuda"), into=into)
        assert t.dz is into[0] and all(torch.equal(p, q) for p, q in zip(s, t))
        turned = torch.empty(520, 136, device="cuda", dtype=dtype).t()
        t = c.score(z, w, labels, upstream=torch.tensor([2.5], device="cuda"), grads=(False, True), into=(None, turned))
        assert t.dz is None
        u = UNIT[dtype]
        assert bool(((turned.double() - s.dw.double()).abs() <= 2 * u * s.dw.double().abs() + 300 * U23 * s.dw.abs().max()).all())
        t = c.score(z, w, labels, upstream=torch.tensor([2.5], device="cuda"), grads=(True, False))
        assert t.dw is None and torch.equal(t.dz, s.dz)


@pytest.mark.parametrize("dtype", TYPES)
def test_in_two_steps(dtype):
    """Loss first, gradients with the known log-sum-exps: the same bits."""
    c = _c()
    z, w, labels = case(333, 200, 1500, dtype, True)
    s = c.score(z, w, labels)
    loss = c.score(z, w, labels, grad=False)
    assert loss.dz is None and torch.equal(loss.loss, s.loss) and torch.equal(loss.rows, s.rows)
    # Rows without a label are copied as zeros before gradients, and their log-sum-exp is any value.
    kept = labels >= 0
    assert torch.equal(loss.lse[kept], s.lse[kept])
    t = c.score(z, w, labels, known=loss)
    assert t.loss is loss.loss and t.rows is loss.rows and torch.equal(t.dz, s.dz) and torch.equal(t.dw, s.dw)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_without_labels(dtype):
    """Whatever they hold, they take no part; all of them: zeros."""
    c = _c()
    z, w, labels = case(150, 80, 300, dtype, False)
    labels[3], labels[4], labels[5] = 300, 1 << 40, -100
    s = c.score(z, w, labels, upstream=torch.tensor([float("inf")], device="cuda"))
    assert not s.dz[labels < 0].any() and not s.dz[3:5].any()
    s = c.score(z, w, labels)
    out = (labels < 0) | (labels >= 300)
    z[out] = float("nan")
    z[3] = float("inf")
    t = c.score(z, w, labels)
    assert torch.equal(t.loss, s.loss) and torch.equal(t.rows, s.rows) and torch.equal(t.dz, s.dz) and torch.equal(t.dw, s.dw)
    e = c.score(z, w, labels, grad=False)
    assert torch.equal(e.loss, s.loss) and torch.equal(e.rows, s.rows)
    t = c.score(z, w, torch.full_like(labels, -1))
    assert float(t.loss) == 0.0 and not t.rows.any() and not t.dz.any() and not t.dw.any()


@pytest.mark.parametrize("kept", [0, 1, 63, 64, 256, 512, 700, 1299])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_without_labels(dtype, kept):
    """Any number of many rows that have labels, anywhere among NaNs: their results, zeros elsewhere, and
    the same from what is known of them."""
    c = _c()
    z, w, labels = case(1299, 264, 1000, dtype, True, 8, drop=0.0)
    out = torch.randperm(1299, generator=torch.Generator().manual_seed(kept))[kept:].cuda()
    labels[out] = torch.where(out % 2 == 0, -1, 1 << 33)
    zeroed = z.clone()
    zeroed[out] = 0.0
    s = check(c, zeroed, w, labels)
    z[out] = float("nan")
    t = c.score(z, w, labels)
    on = labels.lt(1000) & labels.ge(0)
    assert all(torch.equal(p, q) for p, q in zip(s[:4], t[:4])) and torch.equal(s.lse[on], t.lse[on])
    e = c.score(z, w, labels, grad=False)
    assert torch.equal(e.loss, s.loss) and torch.equal(e.rows, s.rows)
    again = c.score(z, w, labels, known=e)
    assert torch.equal(again.dz, s.dz) and torch.equal(again.dw, s.dw)


def test_no_rows():
    c = _c()
    for dtype in TYPES:
        s = c.score(torch.empty(0, 40, dtype=dtype, device="cuda"), torch.ones(40, 24, dtype=dtype, device="cuda"),
                    torch.empty(0, dtype=torch.int64, device="cuda"))
        assert float(s.loss) == 0.0 and s.dz.shape == (0, 40) and not s.dw.any()
        for flip in (False, True):
            w = torch.ones(1000, 300, dtype=dtype, device="cuda").t() if flip else torch.ones(300, 1000, dtype=dtype, device="cuda")
            s = c.score(torch.empty(0, 300, dtype=dtype, device="cuda"), w, torch.empty(0, dtype=torch.int64, device="cuda"))
            assert float(s.loss) == 0.0 and s.dz.shape == (0, 300) and not s.dw.any()


@pytest.mark.parametrize("dtype", TYPES)
def test_sure_and_hopeless_rows(dtype):
    """Logits of hundreds: no overflow, a loss of 0 or of hundreds, and gradients that fit it."""
    c = _c()
    D, V = 64, 700
    w = torch.zeros(D, V, dtype=dtype, device="cuda")
    w[torch.arange(D), torch.arange(D)] = 16.0
    z = torch.zeros(3, D, dtype=dtype, device="cuda")
    z[:, 5] = 32.0                                     # class 5: 512, the others 0
    labels = torch.tensor([5, 6, 699], device="cuda")
    s = c.score(z, w, labels)
    assert torch.equal(s.rows.cpu(), torch.tensor([0.0, 512.0, 512.0]))
    third = torch.tensor([0.0, 16.0, 16.0], device="cuda") / 3
    assert torch.equal(s.dz[:, 5].float(), third.to(dtype).float())
    assert float(s.dz[1, 6]) == float(torch.tensor(-16.0 / 3).to(dtype)) and not s.dz[0].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_sure_rows(dtype):
    """Rows that are nearly certain of their class, 1 - p of some 1e-4: their gradients are made of s - lse,
    whose error is the fp32 sums' and not that of a rounded or cut one.  With |s| near 24 that is 512 2^-23
    sum |z| |w| in the worst case; the sums of the formula's random signs stay below 2^-17 of it in all."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(7)
    R, D, V = 256, 2048, 1024
    w = (torch.randn(V, D, generator=g, device="cuda") * D ** -0.5).to(dtype)
    labels = torch.randint(0, V, (R,), generator=g, device="cuda")
    z = (torch.randn(R, D, generator=g, device="cuda") * 0.5 + 17.0 * w[labels].float()).to(dtype)
    logits = z.double() @ w.double().t()
    p = torch.softmax(logits, 1)
    sure = 1.0 - p.gather(1, labels[:, None])[:, 0]
    assert 1e-6 < float(sure.median()) < 1e-2
    p[torch.arange(R, device="cuda"), labels] -= 1.0
    # s - lse is off by some 2^-17: as much of 1 - p relative to 1 - p itself, which is 1e-4 or so, would be
    # 8 %; the sums' actual errors are a few 2^-24 of 17.  fp16 values this small (1e-8) lie between
    # multiples of 2^-24, off by up to half of it each, unless the loss is scaled up as it is for fp16.
    for scale in (1.0, 65536.0):
        s = c.score(z, w.t(), labels, upstream=torch.tensor([scale], device="cuda"))
        dz = p @ w.double() / R * scale
        off = (s.dz.double() - dz).norm() / dz.norm()
        steps = TINY[dtype] / 2 * dz.numel() ** 0.5 / float(dz.norm())
        assert float(off) <= 2 * UNIT[dtype] + 64 * 2.0 ** -24 * 17 / float(sure.square().mean().sqrt()) + steps


def test_pieces(monkeypatch):
    """Several pieces of the classes: the sums over them, and a last piece that is short."""
    from paper_1601_04033_gb300 import fasgd
    c = _c()
    for dtype, R, V in ((torch.bfloat16, 40000, 14001), (torch.float32, 30000, 9001)):
        z, w, labels = case(R, 24, V, dtype, dtype is torch.bfloat16)
        assert R * V * z.element_size() > 2 * fasgd.SCORE_PIECE
        s = c.score(z, w, labels)
        dz, dw = torch.zeros(R, 24, dtype=torch.float64, device="cuda"), torch.zeros(24, V, dtype=torch.float64, device="cuda")
        n = int((labels >= 0).sum())
        for a in range(0, R, 4000):
            k = torch.nonzero(labels[a:a + 4000] >= 0)[:, 0] + a
            g = torch.softmax(z[k].double() @ w.double(), 1)
            g[torch.arange(k.numel(), device="cuda"), labels[k]] -= 1.0
            dz[k] = g @ w.double().t() / n
            dw += z[k].double().t() @ g / n
        # Roundings of g, uncorrelated, and of the result: relative to the whole, in the 2-norm.
        for got, want in ((s.dz, dz), (s.dw, dw)):
            assert float((got.double() - want).norm() / want.norm()) <= (2 * UNIT[dtype] if dtype is torch.bfloat16 else 1e-5)
        assert torch.equal(c.score(z, w, labels).dw, s.dw)


def test_differentiates_and_replays():
    c = _c()
    z, w, labels = case(200, 96, 1000, torch.float32, True)
    za, wa = z.detach().clone().requires_grad_(True), w.detach().clone().requires_grad_(True)
    loss, rows = c.scored(za, wa, labels)
    (loss * 3.0).backward()
    want = c.score(z, w, labels, upstream=torch.tensor([3.0], device="cuda"))
    assert torch.equal(loss.detach().reshape(1), want.loss) and not rows.requires_grad
    assert torch.equal(za.grad, want.dz) and torch.equal(wa.grad, want.dw)
    # torch's own, in 64 bits, and differences along the gradient.
    ref = [t.detach().double().requires_grad_(True) for t in (z, w)]

    def loss64(a, b):
        return torch.nn.functional.cross_entropy(a @ b, labels, ignore_index=-1)

    g = torch.autograd.grad(3.0 * loss64(*ref), ref)
    for got, d in zip((za.grad, wa.grad), g):
        assert (got - d).abs().max() <= 1000 * U23 * d.abs().max()
    for i in range(2):
        moved = [[t.detach() + s * 1e-5 * (g[j] if i == j else 0.0) for j, t in enumerate(ref)] for s in (1, -1)]
        rise = 3.0 * (loss64(*moved[0]) - loss64(*moved[1])) / 2e-5
        assert abs(rise - (g[i] ** 2).sum()) <= 1e-5 * (g[i] ** 2).sum()
    with pytest.raises(RuntimeError, match="second derivatives"):
        d, = torch.autograd.grad(c.scored(za, wa, labels)[0], za, create_graph=True)
        d.sum().backward()
    # Captured, on other inputs, next to calls on another stream.
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = c.score(z, w, labels)
    z.mul_(0.5)
    labels.copy_(labels.roll(1))
    graph.replay()
    got = [t.clone() for t in kept]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        again = c.score(z, w, labels)
    here = c.score(z, w, labels)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(got, again, here))
