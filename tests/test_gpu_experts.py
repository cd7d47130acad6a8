"""The routed experts' operators (routes, rows to their experts and back, the experts'
products) against their definitions in 64 bits.

Bounds.  A sum of K products in fp32, in any order and with additions that round or cut,
is off by at most K 2^-23 sum |a| |b|: each addition by 2^-23 of a partial sum that
sum |a| |b| bounds, products of 16-bit values being exact and those of fp32 values off by
2^-24 once.  fp32 products by planes add, for each term, five partial products of 2^-8 of the
term's size (5 K 2^-8 2^-23) and drop 2^-25 of it; and sums of 256 k (of six pairs: 6 K / 256
of them, at least one and the begun one) are added up in fp32, each off by 2^-24: together less than
(K / 32 + 2) 2^-23 more.  Storing rounds by half a step of the type."""

import random

import pytest

from client_util import TINY, UNIT
from test_gpu_client import _c

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = [torch.float32, torch.bfloat16, torch.float16]
U23 = 2.0 ** -23


def near(got, want, size, terms, what=""):
    """got of a type against want in 64 bits, a sum of `terms` products of which the sizes add up to `size`."""
    u = UNIT[got.dtype]
    bound = (terms * (33 / 32) + 2) * U23 * size * (1 + u) + u * want.abs() + TINY[got.dtype]
    off = (got.double() - want).abs()
    worst = (off - bound).max() if off.numel() else torch.zeros(())
    assert bool((off <= bound).all()), (what, float(worst), float(off.max()))


def choices(g, T, top, E, drop=0.1):
    c = torch.randint(0, E, (T, top), generator=g, device="cuda", dtype=torch.int32)
    if drop:
        c[torch.rand(T, top, generator=g, device="cuda") < drop] = -1
    return c


def route64(chosen, E):
    flat = chosen.reshape(-1).tolist()
    by = [[a for a, c in enumerate(flat) if c == e] for e in range(E)]
    order = [a for entries in by for a in entries]
    place = [-1] * len(flat)
    for i, a in enumerate(order):
        place[a] = i
    offsets = [0]
    for entries in by:
        offsets.append(offsets[-1] + len(entries))
    order += [-1] * (len(flat) - len(order))
    return [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (offsets, order, place)]


@pytest.mark.parametrize("T,top,E", [(1, 1, 1), (1, 8, 8), (128, 2, 4), (0, 2, 3), (33, 3, 1024), (4096, 1, 300), (8000, 2, 320),
                                     (2500, 7, 321), (2048, 2, 512), (40000, 3, 17), (70000, 1, 1024)])
def test_routes(T, top, E):
    g = torch.Generator(device="cuda").manual_seed(T + E)
    chosen = choices(g, T, top, E)
    if T > 40:
        chosen[5:9] = E                       # beyond the last expert
        chosen[9:12] = 1 << 30
        chosen[30:] = torch.where(chosen[30:] == 0, -7, chosen[30:])      # an expert nearly without rows
    r = _c().route(chosen, E)
    for got, want in zip(r, route64(chosen, E)):
        assert torch.equal(got.reshape(-1), want)
    again = _c().route(chosen, E)
    assert all(torch.equal(x, y) for x, y in zip(r, again))


def test_routes_with_nothing_chosen():
    r = _c().route(torch.full((50, 3), -1, dtype=torch.int32, device="cuda"), 5)
    assert not r.offsets.any() and (r.order == -1).all() and (r.place == -1).all()


def matrix(g, R, D, dtype, pad=0, scale=1.0):
    t = torch.full((R, D + pad), float("nan"), device="cuda", dtype=dtype)
    t[:, :D] = torch.randn(R, D, generator=g, device="cuda") * scale
    return t[:, :D]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,top,E,D,pad", [(128, 2, 4, 96, 0), (1, 8, 16, 2048, 0), (1, 1, 1, 1, 0), (37, 3, 5, 61, 0), (200, 9, 13, 264, 8),
                                           (500, 2, 7, 1021, 3), (64, 17, 40, 8192, 0), (0, 2, 3, 40, 0),
                                           (41, 3, 4, 1030, 0), (30, 9, 11, 260, 6), (2100, 2, 3, 515, 1)])
def test_rows_to_places_and_back(dtype, T, top, E, D, pad):
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(D)
    chosen = choices(g, T, top, E, 0.3)
    if T > 3:
        chosen[2] = -1                        # a row that goes nowhere
    r = c.route(chosen, E)
    n = T * top
    x, dout = matrix(g, T, D, dtype, pad), matrix(g, T, D, dtype, pad)
    y = matrix(g, n, D, dtype, pad)
    y[int(r.offsets[-1]):] = float("nan")    # places of no entry are not read
    weight = torch.rand(T, top, generator=g, device="cuda")
    at = r.place.reshape(-1).long()
    entries = torch.nonzero(at >= 0)[:, 0]
    at, t = at[entries], entries // top
    xs = c.gather(x, r)
    want = torch.zeros(n, D, dtype=dtype, device="cuda")
    want[at] = x[t]
    assert torch.equal(xs, want)
    for w in (weight, None):
        w64 = torch.ones(n, device="cuda", dtype=torch.float64)[entries] if w is None else w.reshape(-1).double()[entries]
        terms = y.double()[at] * w64[:, None]
        zero = torch.zeros(T, D, dtype=torch.float64, device="cuda")
        near(c.combine(y, r, w), zero.index_add(0, t, terms), zero.index_add(0, t, terms.abs()), top, "out")
    dy, dweight = c.combine_grad(y, r, weight, dout)
    terms = dout.double()[t] * weight.reshape(-1).double()[entries][:, None]
    want = torch.zeros(n, D, dtype=torch.float64, device="cuda").index_copy(0, at, terms)
    near(dy, want, want.abs(), 1, "dy")
    prod = dout.double()[t] * y.double()[at]
    zero = torch.zeros(n, dtype=torch.float64, device="cuda")
    near(dweight.reshape(-1), zero.index_copy(0, entries, prod.sum(1)), zero.index_copy(0, entries, prod.abs().sum(1)), D, "dweight")
    # Into the caller's tensors, rows apart.
    outs = matrix(g, n, D, dtype, 5), matrix(g, T, D, dtype, 5), matrix(g, n, D, dtype, 5)
    assert c.gather(x, r, out=outs[0]) is outs[0] and torch.equal(outs[0], xs)
    assert torch.equal(c.combine(y, r, weight, out=outs[1]), c.combine(y, r, weight))
    dw2 = torch.empty_like(weight)
    c.combine_grad(y, r, weight, dout, into=c.CombineGrads(outs[2], dw2))
    assert torch.equal(outs[2], dy)
    near(dw2.reshape(-1), zero.index_copy(0, entries, prod.sum(1)), zero.index_copy(0, entries, prod.abs().sum(1)), D, "dweight")


def test_routes_that_are_not_ones_stay_in_bounds():
    """Entries outside [0, n) stand for nowhere, whatever they are."""
    c = _c()
    T, top, D = 40, 2, 64
    x = torch.randn(T, D, device="cuda")
    y = torch.randn(T * top, D, device="cuda")
    odd = torch.tensor([-5, T * top, 1 << 30, -(1 << 31)], dtype=torch.int32, device="cuda").repeat(T * top // 4)
    r = c.Route(torch.zeros(2, dtype=torch.int32, device="cuda"), odd, odd.reshape(T, top))
    assert not c.gather(x, r).any() and not c.combine(y, r).any()
    dy, dw = c.combine_grad(y, r, torch.ones(T, top, device="cuda"), x)
    assert not dy.any() and not dw.any()


# sizes of the groups, rows of no expert before and behind, inputs, outputs
PRODUCTS = [
    ([1], 0, 0, 1, 1), ([1, 0, 2], 0, 0, 8, 8), ([3], 0, 2, 64, 128), ([0, 0], 0, 3, 16, 24), ([130, 64, 62], 0, 0, 96, 64),
    ([1, 1, 1, 1, 1, 1, 1, 1], 0, 0, 512, 256), ([300, 0, 17, 129, 1], 0, 5, 200, 136), ([257, 255], 3, 4, 129, 61),
    ([63, 65, 15, 16, 17], 0, 0, 72, 1021), ([1000, 24], 0, 0, 520, 264), ([31] * 40, 0, 9, 40, 80), ([513], 7, 0, 64, 320),
    ([0, 0, 5, 0], 2, 1, 33, 7), ([4], 0, 0, 2048, 40), ([2, 700], 0, 0, 264, 24), ([200, 56], 0, 0, 1000, 10),
    ([700, 0, 333, 1], 2, 3, 517, 261), ([65, 1500], 0, 0, 320, 1032), ([3, 0, 1], 0, 2, 5000, 4100),
]


def product_case(g, sizes, before, behind, K, N, dtype, w_dtype, flip, pad=0):
    n = before + sum(sizes) + behind
    offsets = [before]
    for s in sizes:
        offsets.append(offsets[-1] + s)
    offsets = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    x, dy = matrix(g, n, K, dtype, pad), matrix(g, n, N, dtype, pad)
    for t in (x, dy):                         # rows that no expert has are not read
        t[:before] = float("nan")
        t[n - behind:] = float("inf")
    w = torch.randn(len(sizes), *((N, K) if flip else (K, N)), generator=g, device="cuda").to(w_dtype)
    return x, w.transpose(1, 2) if flip else w, offsets, dy


def check_products(c, x, w, offsets, dy, **kw):
    y = c.multiply(x, w, offsets)
    dx, dw = c.multiply_grad(x, w, offsets, dy)
    K, N = w.shape[1:]
    n, bounds = x.shape[0], offsets.tolist()
    assert dw.dtype == w.dtype and dw.stride() == torch.empty_like(w).stride()

    def zeros(*shape):
        return torch.zeros(*shape, dtype=torch.float64, device="cuda")

    want = [zeros(n, N), zeros(n, K), zeros(*w.shape)]
    size = [zeros(n, N), zeros(n, K), zeros(*w.shape)]
    terms = zeros(w.shape[0], 1, 1)
    for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
        xe, we, de = x[a:b].double(), w[e].to(x.dtype).double(), dy[a:b].double()
        for of, f in ((want, lambda t: t), (size, torch.abs)):
            of[0][a:b] = f(xe) @ f(we)
            of[1][a:b] = f(de) @ f(we).t()
            of[2][e] = f(xe).t() @ f(de)
        terms[e] = b - a
    near(y, want[0], size[0], K, "y")
    near(dx, want[1], size[1], N, "dx")
    near(dw, want[2], size[2], terms, "dw")
    return y, dx, dw


@pytest.mark.parametrize("flip", [False, True])
@pytest.mark.parametrize("types", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16),
                                   (torch.bfloat16, torch.float32), (torch.float16, torch.float32)])
@pytest.mark.parametrize("case", PRODUCTS, ids=lambda c: f"{len(c[0])}x{sum(c[0])}x{c[3]}x{c[4]}")
def test_products(case, types, flip):
    g = torch.Generator(device="cuda").manual_seed(sum(case[0]) + case[3])
    check_products(_c(), *product_case(g, *case, *types, flip))


@pytest.mark.parametrize("pad", [3, 8])
@pytest.mark.parametrize("dtype", TYPES)
def test_products_of_rows_apart(dtype, pad):
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(pad)
    for case in (PRODUCTS[6], PRODUCTS[9]):
        x, w, offsets, dy = product_case(g, *case, dtype, dtype, False, pad)
        y, dx, dw = check_products(c, x, w, offsets, dy)
        # The experts' matrices in a wider buffer, an odd address, an odd step between them.
        E, K, N = w.shape
        wide = torch.full((E, K + 1, N + pad), float("nan"), device="cuda", dtype=dtype)
        inner = wide[:, :K, 1:N + 1] if pad == 3 else wide[:, :K, :N]
        inner.copy_(w)
        assert torch.equal(c.multiply(x, inner, offsets), y)
        out = matrix(g, x.shape[0], N, dtype, pad)
        into = c.MultiplyGrads(matrix(g, x.shape[0], K, dtype, pad), torch.full_like(wide, 7.0)[:, :K, 1:N + 1])
        assert c.multiply(x, w, offsets, out=out) is out and torch.equal(out, y)
        c.multiply_grad(x, w, offsets, dy, into=into)
        assert torch.equal(into.x, dx) and torch.equal(into.w, dw)
        # The other layout of the gradient, and one gradient alone.
        turned = torch.empty(E, N, K, dtype=dtype, device="cuda").transpose(1, 2)
        only = c.multiply_grad(x, w, offsets, dy, grads=(False, True), into=c.MultiplyGrads(None, turned))
        assert only.x is None
        near(turned, dw.double(), dw.double().abs() + 1, sum(case[0]))
        only = c.multiply_grad(x, w, offsets, dy, grads=(True, False))
        assert only.w is None and torch.equal(only.x, dx)


@pytest.mark.parametrize("dtype", TYPES)
def test_odd_offsets_stay_in_bounds(dtype):
    """Offsets that leave the rows or fall are cut: what is not an expert's is 0, guards around
    the outputs stay."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(1)
    n, K, N = 100, 72, 136
    x, dy = matrix(g, n, K, dtype), matrix(g, n, N, dtype)
    w = torch.randn(3, K, N, generator=g, device="cuda").to(dtype)
    for offsets, kept in (([-50, 20, 1 << 30, 1 << 30], None), ([60, 20, 20, 20], 0), ([0, 100, 40, 1000], None),
                          ([1 << 30] * 4, 0), ([-9] * 4, 0), ([100, 50, 0, -3], 0)):
        guard = torch.full((n + 64, N), 3.0, dtype=dtype, device="cuda")
        o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        c.multiply(x, w, o, out=guard[32:-32])
        dx, dw = c.multiply_grad(x, w, o, dy)
        assert (guard[:32] == 3.0).all() and (guard[-32:] == 3.0).all()
        if kept == 0:
            assert not guard[32:-32].any() and not dx.any() and not dw.any()


def test_products_without_rows():
    c = _c()
    for dtype in TYPES:
        x, w = torch.empty(0, 40, dtype=dtype, device="cuda"), torch.ones(3, 40, 24, dtype=dtype, device="cuda")
        offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
        assert c.multiply(x, w, offsets).shape == (0, 24)
        dx, dw = c.multiply_grad(x, w, offsets, torch.empty(0, 24, dtype=dtype, device="cuda"))
        assert dx.shape == (0, 40) and not dw.any() and dw.shape == w.shape


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_special_values_stay_in_their_rows(dtype):
    """A row of NaN or infinities reaches its own results and its expert's gradient, no others."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w, offsets, dy = product_case(g, [70, 10, 50], 0, 0, 80, 96, dtype, dtype, False)
    clean = c.multiply(x, w, offsets), *c.multiply_grad(x, w, offsets, dy)
    x[71] = float("nan")
    dy[75, 3] = float("inf")
    y, (dx, dw) = c.multiply(x, w, offsets), c.multiply_grad(x, w, offsets, dy)
    rows = torch.arange(130, device="cuda")
    assert torch.equal(y[rows != 71], clean[0][rows != 71]) and y[71].isnan().all()
    assert torch.equal(dx[rows != 75], clean[1][rows != 75]) and not dx[75].isfinite().any()
    assert torch.equal(dw[[0, 2]], clean[2][[0, 2]]) and dw[1].isnan().all()


def test_calls_on_other_streams_and_in_graphs():
    """Two products at once on two streams, and the whole way captured and replayed with new choices."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(5)
    T, top, E, D, H = 300, 2, 6, 128, 192
    x = matrix(g, T, D, torch.bfloat16)
    up, down = (torch.randn(E, *s, generator=g, device="cuda").mul_(0.1) for s in ((D, H), (H, D)))
    weight = torch.rand(T, top, generator=g, device="cuda")
    chosen = choices(g, T, top, E)

    def way():
        r = c.route(chosen, E)
        xs = c.gather(x, r)
        u = c.multiply(xs, up, r.offsets)
        y = c.multiply(u, down, r.offsets)
        out = c.combine(y, r, weight)
        dy, dweight = c.combine_grad(y, r, weight, out)
        du, ddown = c.multiply_grad(u, down, r.offsets, dy)
        dxs, dup = c.multiply_grad(xs, up, r.offsets, du)
        return [out, dweight, ddown, dup, c.combine(dxs, r)]

    first = way()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    results = []
    for s in streams:
        with torch.cuda.stream(s):
            results += [way() for _ in range(3)]
    torch.cuda.synchronize()
    for r in results:
        assert all(torch.equal(p, q) for p, q in zip(r, first))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = way()
    for seed in (1, 2):
        chosen.copy_(choices(torch.Generator(device="cuda").manual_seed(seed), T, top, E))
        graph.replay()
        replayed = [t.clone() for t in kept]
        assert all(torch.equal(p, q) for p, q in zip(replayed, way()))


def experts_plain(x, chosen, weight, up, down):
    """Every expert on every row, in 64 bits."""
    E = up.shape[0]
    chosen = chosen.long()
    share = torch.zeros(x.shape[0], E, dtype=x.dtype, device=x.device)
    share = share.index_put((torch.arange(x.shape[0], device=x.device)[:, None].expand_as(chosen)[chosen >= 0], chosen[chosen >= 0]),
                            weight[chosen >= 0], accumulate=True)
    u = torch.relu(torch.einsum("td,edh->eth", x, up))
    return torch.einsum("eth,ehd,te->td", u, down, share)


def test_the_way_through_the_experts_differentiates():
    """gathered -> multiplied -> multiplied -> combined in fp32: the gradients of rows, weights of
    the combination and experts are the formula's, and differences'."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(9)
    T, top, E, D, H = 90, 2, 5, 40, 24
    chosen = choices(g, T, top, E, 0.2)
    leaves = [torch.randn(T, D, generator=g, device="cuda"), torch.rand(T, top, generator=g, device="cuda"),
              torch.randn(E, D, H, generator=g, device="cuda") * 0.2, torch.randn(E, H, D, generator=g, device="cuda") * 0.2]
    dout = torch.randn(T, D, generator=g, device="cuda")

    def way(x, weight, up, down):
        r = c.route(chosen, E)
        u = torch.relu(c.multiplied(c.gathered(x, r), up, r.offsets))
        return c.combined(c.multiplied(u, down, r.offsets), r, weight)

    own = [t.clone().requires_grad_(True) for t in leaves]
    out = way(*own)
    got = torch.autograd.grad(out, own, dout)
    ref = [t.double().requires_grad_(True) for t in leaves]
    want_out = experts_plain(ref[0], chosen, *ref[1:])
    want = torch.autograd.grad(want_out, ref, dout.double())
    # Sums of up to D, H and T terms, one after the other: relative to the largest value.
    assert (out - want_out).abs().max() <= 200 * U23 * want_out.abs().max() * 4
    for a, b in zip(got, want):
        assert (a - b).abs().max() <= 400 * U23 * b.abs().max() * 4
    # Differences in 64 bits along the gradient's own direction confirm the formula's.
    for i in range(4):
        step = 1e-6
        moved = [[t.detach() + s * step * (a.detach().double() if i == j else 0.0) for j, (t, a) in enumerate(zip(ref, want))]
                 for s in (1, -1)]
        rise = sum(s * (experts_plain(m[0], chosen, *m[1:]) * dout.double()).sum() for s, m in zip((1, -1), moved)) / (2 * step)
        assert abs(rise - (want[i] ** 2).sum()) <= 1e-5 * (want[i] ** 2).sum()
    with pytest.raises(RuntimeError, match="second derivatives"):
        d, = torch.autograd.grad(way(*own).sum(), own[2], create_graph=True)
        d.sum().backward()


def test_gathers_differentiate_twice():
    c = _c()
    r = c.route(torch.tensor([[0, 1], [1, 1], [-1, 0]], dtype=torch.int32, device="cuda"), 2)
    x = torch.randn(3, 8, device="cuda", requires_grad=True)
    v = torch.randn(6, 8, device="cuda", requires_grad=True)
    d, = torch.autograd.grad(c.gathered(x, r), x, v, create_graph=True)
    assert torch.allclose(d, c.combine(v, r))
    again, = torch.autograd.grad(d, v, torch.ones_like(d))
    assert torch.equal(again, c.gather(torch.ones(3, 8, device="cuda"), r))
    y = torch.randn(6, 8, device="cuda", requires_grad=True)
    u = torch.randn(3, 8, device="cuda", requires_grad=True)
    d, = torch.autograd.grad(c.combined(y, r), y, u, create_graph=True)
    assert torch.equal(d, c.gather(u, r))
    again, = torch.autograd.grad(d, u, torch.ones_like(d))
    assert torch.equal(again, c.combine(torch.ones(6, 8, device="cuda"), r))


def test_many_experts():
    """As many as there may be, most with two rows, one with many, some with none."""
    g = torch.Generator(device="cuda").manual_seed(2)
    sizes = [2] * 1024
    sizes[17], sizes[500], sizes[1023] = 700, 0, 0
    for dtype in (torch.bfloat16, torch.float32):
        check_products(_c(), *product_case(g, sizes, 0, 3, 24, 40, dtype, dtype, False))


def test_rows_far_apart():
    """Offsets beyond 2^31 values: rows of a wide buffer, read, written and exchanged."""
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(4)
    R, D, far = 60000, 64, 40000
    wide = torch.empty(2, R, far, dtype=torch.bfloat16, device="cuda")
    x, out = wide[0][:, 8:8 + D], wide[1][:, 16:16 + D]
    x.copy_(torch.randn(R, D, generator=g, device="cuda"))
    w = torch.randn(3, D, D, generator=g, device="cuda").to(torch.bfloat16)
    offsets = torch.tensor([0, 20000, 59000, 59990], dtype=torch.int32, device="cuda")
    near_by = x.contiguous()
    want = c.multiply(near_by, w, offsets)
    assert torch.equal(c.multiply(x, w, offsets, out=out), want) and torch.equal(out, want)
    for p, q in zip(c.multiply_grad(x, w, offsets, out), c.multiply_grad(near_by, w, offsets, want)):
        assert torch.equal(p, q)
    r = c.route(choices(g, R, 1, 7), 7)
    assert torch.equal(c.gather(x, r, out=out), c.gather(near_by, r))
    weight = torch.rand(R, 1, generator=g, device="cuda")
    assert torch.equal(c.combine(out, r, weight), c.combine(out.contiguous(), r, weight))
    labels = torch.randint(0, 900, (R,), generator=g, device="cuda")
    classes = torch.randn(D, 900, generator=g, device="cuda").to(torch.bfloat16)
    for p, q in zip(c.score(x, classes, labels), c.score(near_by, classes, labels)):
        assert torch.equal(p, q)


def test_random_products():
    """Sizes drawn over the range of small ones, all layouts."""
    c = _c()
    rng = random.Random(11)
    g = torch.Generator(device="cuda").manual_seed(11)
    for _ in range(40):
        sizes = [rng.choice([0, 1, 7, 64, 100, 300]) for _ in range(rng.randint(1, 9))]
        dtype = rng.choice(TYPES)
        x, w, offsets, dy = product_case(g, sizes, rng.choice([0, 0, 5]), rng.choice([0, 0, 70]), rng.randint(1, 400), rng.randint(1, 400),
                                         dtype, rng.choice([dtype, torch.float32]), rng.random() < 0.5, rng.choice([0, 0, 1, 8]))
        check_products(c, x, w, offsets, dy)
