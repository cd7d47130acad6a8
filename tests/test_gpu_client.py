"""The client operators (dropout, the residual join and its gradients, the balance
loss) on the GPU, against their definitions in 64 bits: every type, both norms,
sizes where tiles, vectors and octets end, strided and unaligned rows, gates
shared by groups of rows, empty and masked rows, special values."""

import numpy as np
import pytest

from client_util import U32, Join64, factors, hold

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "bfloat16", "float16"]
SEED, CLIENT, COUNT = 0x9E37_79B9_7F4A_7C15, 11, (5 << 32) + 3


def _c():
    from paper_1601_04033_gb300 import client
    return client


def rows_of(gen, R, D, dtype, scale=1.0, shift=0.0, pad=0, offset=0):
    """[R, D] rows `pad` values apart, `offset` values into their buffer."""
    import torch
    buf = torch.full((R * (D + pad) + offset + 8,), float("nan"), device="cuda", dtype=dtype)
    t = buf[offset:offset + R * (D + pad)].view(R, D + pad)[:, :D]
    t.copy_(torch.randn(R, D, generator=gen, device="cuda") * scale + shift)
    return t


def draws(rate):
    return _c().Draws(rate, SEED, CLIENT, COUNT) if rate else None


def make(R, D, dtype, norm="rms", groups=0, post=True, pre=True, y=True, seed=1, pad=0, offset=0, gate_f32=False):
    """Arguments of a join: groups = 0: no gate, 1: a vector, else that many gates."""
    import torch
    dtype = getattr(torch, dtype) if isinstance(dtype, str) else dtype
    gen = torch.Generator(device="cuda").manual_seed(seed)
    layer = norm == "layer"

    def vec(mean, spread):
        # 4-byte aligned only, as a view into a flat vector of parameters.
        return (torch.randn(D + 1, generator=gen, device="cuda") * spread + mean)[1:]

    a = dict(x=rows_of(gen, R, D, dtype, 1.3, 0.2, pad, offset),
             y=rows_of(gen, R, D, dtype, 0.6, -0.1, pad, offset) if y else None,
             post=vec(1.0, 0.3) if post and y else None,
             post_bias=vec(0.0, 0.2) if post and y and layer else None, gate=None,
             pre=vec(1.0, 0.3) if pre else None, pre_bias=vec(0.0, 0.2) if pre and layer else None)
    if groups == 1:
        a["gate"] = vec(0.5, 0.3)
    elif groups > 1:
        a["gate"] = (torch.randn(groups, D, generator=gen, device="cuda") * 0.3 + 0.5).to(
            torch.float32 if gate_f32 else dtype)
    dh = rows_of(gen, R, D, dtype, 0.7, 0.0, pad, offset)
    dz = rows_of(gen, R, D, dtype, 0.7, 0.0, pad, offset) if pre else None
    return a, dh, dz


def check_join(a, dh, dz, norm="rms", eps=1e-5, carry=0.9, branch=0.7, rate=0.0, strided=0, use_dh=True):
    import torch
    c = _c()
    R, D = a["x"].shape
    j = c.join(**a, norm=norm, eps=eps, carry=carry, branch=branch, draws=draws(rate))
    g = c.join_grad(j, dh if use_dh else None, dz)
    want = Join64(a["x"], a["y"], a["post"], a["post_bias"], a["gate"], a["pre"], a["pre_bias"], norm == "layer",
                  eps, carry, branch, (rate, SEED, CLIENT, COUNT), dh if use_dh else None, dz)
    # h's terms; z's: a row's values over its 1/sqrt.
    scale = want.h.abs().amax(1, keepdim=True) + carry * a["x"].double().abs()
    if a["y"] is not None:
        hold(j.h, want.h, scale, "h")
    else:
        assert j.h is None
    if a["pre"] is not None:
        h = want.h
        mean = h.mean(1, keepdim=True) if norm == "layer" else 0.0
        rstd = 1 / torch.sqrt(((h - mean) ** 2).mean(1, keepdim=True) + eps)
        size = scale.amax(1, keepdim=True) * rstd
        bias = 0.0 if a["pre_bias"] is None else a["pre_bias"].double().abs()
        hold(j.z, want.z, size * a["pre"].double().abs() * (1 + size) + bias, "z")
    assert j.h is None or torch.isfinite(j.h.float()).all()
    hold(g.x, want.grads["x"], want.row * (carry if a["y"] is not None else 1.0), "dx")
    if a["y"] is not None:
        hold(g.y, want.grads["y"], want.row_y, "dy")
    for name in ("post", "post_bias", "gate", "pre", "pre_bias"):
        t = getattr(g, name)
        assert (t is None) == (a[name] is None)
        if t is not None:
            hold(t, want.grads[name], want.terms[name], "d" + name, rows=R)
    return j, g


WIDTHS = [1, 2, 7, 8, 9, 24, 63, 64, 65, 200, 255, 256, 257, 500, 512, 784, 1000, 1021, 1024, 1031, 2000, 2047,
          2048, 2056, 4096, 4099, 5000, 8184, 8191, 8192, 8193, 8200, 16384, 20001, 32768, 32776, 40001]


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_join_widths(D, dtype):
    k = WIDTHS.index(D)
    for n, R in enumerate((1, 9 + k)):
        norm = ("rms", "layer")[(k + n) % 2]
        check_join(*make(R, D, dtype, norm, groups=1), norm=norm, rate=(0.0, 0.3)[(k // 2 + n) % 2])


@pytest.mark.parametrize("R", [2, 3, 8, 31, 151, 152, 153, 303, 305, 1000, 2433, 5001])
def test_join_row_counts(R):
    for D, dtype, norm in ((40, "bfloat16", "layer"), (41, "float16", "rms"), (264, "float32", "layer"),
                           (1027, "bfloat16", "rms")):
        check_join(*make(R, D, dtype, norm, groups=1), norm=norm, rate=0.1)


@pytest.mark.parametrize("post, gate, pre, y", [(p, g, r, True) for p in (0, 1) for g in (0, 1) for r in (0, 1)]
                         + [(0, 0, 1, False)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("D", [96, 203, 9000])
def test_join_parts(post, gate, pre, y, norm, D):
    """Every part may be absent; dh may be absent where z has a gradient."""
    a, dh, dz = make(37, D, "bfloat16" if D != 203 else "float32", norm, gate, bool(post), bool(pre), y)
    check_join(a, dh, dz, norm=norm, rate=0.25)
    if pre:
        check_join(a, dh, dz, norm=norm, use_dh=False)
    if y and norm == "layer":             # a norm without its biases
        check_join({**a, "post_bias": None, "pre_bias": None}, dh, dz, norm=norm)


@pytest.mark.parametrize("groups, L", [(2, 1), (2, 40), (3, 7), (5, 300), (13, 33), (64, 8), (400, 1), (700, 3),
                                       (100, 16)])
@pytest.mark.parametrize("D, gate_f32", [(128, False), (129, True), (1030, False), (9000, True)])
def test_join_gates_of_groups(groups, L, D, gate_f32):
    norm = "layer" if D % 2 else "rms"
    if groups * L * D > 4_000_000:
        L = max(1, 4_000_000 // (groups * D))
    check_join(*make(groups * L, D, "float16" if D > 128 else "bfloat16", norm, groups, gate_f32=gate_f32),
               norm=norm, rate=0.2)


@pytest.mark.parametrize("pad, offset", [(0, 1), (0, 3), (1, 0), (3, 0), (8, 0), (16, 8), (8, 4), (5, 2)])
@pytest.mark.parametrize("D", [1, 6, 40, 200, 203, 1024, 5003])
@pytest.mark.parametrize("dtype", DTYPES)
def test_join_strides_and_alignments(pad, offset, D, dtype):
    import torch
    a, dh, dz = make(21, D, dtype, groups=1, pad=pad, offset=offset)
    j, g = check_join(a, dh, dz, rate=0.3)
    # The same values in rows without gaps.
    b = {k: None if t is None else t.clone(memory_format=torch.contiguous_format) for k, t in a.items()}
    j2, g2 = check_join(b, dh.contiguous(), dz.contiguous(), rate=0.3)
    hold(j.h, j2.h.double(), j2.h.double().abs().amax(), "h by layout")
    # Outputs into strided places leave what lies between alone.
    R = 21
    gen = torch.Generator(device="cuda").manual_seed(3)
    outs = [rows_of(gen, R, D, a["x"].dtype, pad=pad, offset=offset) for _ in range(4)]
    before = [o._base.clone() for o in outs]
    c = _c()
    s = dict(norm="rms", eps=1e-5, carry=0.9, branch=0.7, draws=draws(0.3))
    k = c.join(**a, **s, h=outs[0], z=outs[1])
    c.join_grad(k, dh, dz, into=c.JoinGrads(x=outs[2], y=outs[3]))
    for o, want, was in zip(outs, (j.h, j.z, g.x, g.y), before):
        assert torch.equal(o, want)
        o.copy_(was[offset:offset + R * (D + pad)].view(R, D + pad)[:, :D])
        assert torch.equal(o._base.view(torch.uint8), was.view(torch.uint8))


@pytest.mark.parametrize("D, pad", [(48, 3), (200, 5), (1021, 16), (2056, 3), (9001, 1)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_join_many_unaligned_rows(D, pad, norm):
    """Enough rows for every block to take several, and parts that are absent."""
    for dtype in ("bfloat16", "float32"):
        R = 1300 if D < 3000 else 400
        check_join(*make(R, D, dtype, norm, groups=1, pad=pad, offset=1), norm=norm, rate=0.2)
        check_join(*make(R, D, dtype, norm, groups=2, post=False, pad=pad), norm=norm, use_dh=False)
        check_join(*make(R, D, dtype, norm, y=False, pad=pad, offset=3), norm=norm)


def test_join_halves_of_one_matrix():
    """x and y as the two halves of one product's rows, h and z of another's."""
    import torch
    c = _c()
    a, dh, dz = make(19, 136, "bfloat16", groups=1)
    wide = torch.cat((a["x"], a["y"]), 1)
    out = torch.empty_like(wide)
    j = c.join(**{**a, "x": wide[:, :136], "y": wide[:, 136:]}, h=out[:, :136], z=out[:, 136:])
    k = c.join(**a)
    assert torch.equal(j.h, k.h) and torch.equal(j.z, k.z)
    with pytest.raises(Exception, match="share"):
        c.join(**{**a, "x": wide[:, :136], "y": wide[:, 136:]}, h=wide[:, 8:144], z=out[:, 136:])


def test_join_gradients_into_a_flat_vector():
    """Parameters and their gradients as views of flat vectors, as they are pulled
    and pushed."""
    import torch
    c = _c()
    a, dh, dz = make(50, 77, "float32", "layer", groups=1)
    names = ["post", "post_bias", "gate", "pre", "pre_bias"]
    flat = torch.full((5 * 77 + 3,), -5.0, device="cuda")
    into = c.JoinGrads(**{n: flat[3 + 77 * i:3 + 77 * (i + 1)] for i, n in enumerate(names)})
    j = c.join(**a, norm="layer")
    g = c.join_grad(j, dh, dz, into=into)
    w = c.join_grad(j, dh, dz)
    for n in names:
        assert getattr(g, n) is getattr(into, n) and torch.equal(getattr(g, n), getattr(w, n)), n
    assert (flat[:3] == -5).all()


@pytest.mark.parametrize("D", [64, 201, 9001])
def test_join_special_rows(D):
    """Rows of zeros and of one value (no variance), of huge and tiny values; a NaN
    or an infinity stays in its own row."""
    import torch
    c = _c()
    a, dh, dz = make(12, D, "float32", "layer", groups=1)
    a["x"][0] = 0
    a["y"][0] = 0
    a["x"][1] = 3
    a["y"][1] = -2
    a["y"][2] *= 1e-20
    a["y"][3] *= 1e15
    check_join(a, dh, dz, norm="layer")
    b, dh2, dz2 = make(12, D, "float32", "rms", groups=1)
    b["x"][0] = 0
    b["y"][0] = 0
    check_join(b, dh2, dz2)
    clean = c.join(**a, norm="layer")
    gc = c.join_grad(clean, dh, dz)
    bad = {k: None if t is None else t.clone() for k, t in a.items()}
    bad["x"][5, D // 2] = float("nan")
    bad["y"][7, D // 3] = float("inf")
    j = c.join(**bad, norm="layer")
    g = c.join_grad(j, dh, dz)
    ok = [r for r in range(12) if r not in (5, 7)]
    for got, want in ((j.h, clean.h), (j.z, clean.z), (g.x, gc.x), (g.y, gc.y)):
        assert torch.equal(got[ok], want[ok])
    assert j.z[5].isnan().all() and j.h[7].isnan().all() and j.h[5].isnan().sum() == 1
    assert g.x[5].isnan().all() and g.pre.isnan().all()


def test_join_rate_one_drops_the_branch_and_dropped_places_hold_anything():
    import torch
    c = _c()
    a, dh, dz = make(30, 104, "bfloat16", groups=1)
    j = c.join(**a, carry=0.5, draws=draws(1.0))
    assert torch.equal(j.h.float(), (0.5 * a["x"].float()).to(torch.bfloat16).float())
    g = c.join_grad(j, dh, dz)
    assert (g.y == 0).all() and (g.gate == 0).all() and (g.post == 0).all()
    # Without a norm a value that is dropped may be NaN.
    a["post"] = None
    m = torch.from_numpy(factors(np.arange(30 * 104), 0.4, SEED, CLIENT, COUNT).reshape(30, 104)).cuda()
    want = c.join(**a, draws=draws(0.4))
    wg = c.join_grad(want, dh, dz)
    a["y"] = torch.where(m > 0, a["y"], float("nan"))
    got = c.join(**a, draws=draws(0.4))
    gg = c.join_grad(got, dh, dz)
    assert torch.equal(got.h, want.h) and torch.equal(got.z, want.z)
    assert torch.equal(gg.x, wg.x) and torch.equal(gg.y, wg.y) and torch.equal(gg.gate, wg.gate)


@pytest.mark.parametrize("D", [136, 139])
def test_join_draws_dropouts_mask(D):
    """The mask of a join is that of dropout on the same element."""
    import torch
    c = _c()
    a, _, _ = make(40, D, "float32", post=False, pre=False)
    j = c.join(a["x"], a["y"], carry=0.0, draws=draws(0.37))
    assert torch.equal(j.h, c.dropout(a["y"], draws(0.37)))


@pytest.mark.parametrize("D, R", [(33, 6), (256, 5), (8200, 2)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_join_gradient_against_differences(D, R, norm):
    """Directional central differences of the forward kernels' own outputs, summed
    in 64 bits.  With step e the curvature leaves O(e^2) ~ 1e-4 of the third
    derivatives, the outputs' rounding 2^-24 sqrt(2 R D) / e of their size."""
    import torch
    c = _c()
    a, dh, dz = make(R, D, "float32", norm, groups=1, seed=4)
    s = dict(norm=norm, eps=1e-3, carry=0.9, branch=0.7, draws=draws(0.2))
    g = c.join_grad(c.join(**a, **s), dh, dz)
    gen = torch.Generator(device="cuda").manual_seed(9)
    e = 2.0 ** -7
    for name in ("x", "y", "post", "post_bias", "gate", "pre", "pre_bias"):
        if a[name] is None:
            continue
        way = torch.randn(a[name].shape, generator=gen, device="cuda")
        ends = []
        for sign in (1, -1):
            j = c.join(**{**a, name: a[name] + sign * e * way}, **s)
            ends.append((j.h.double() * dh.double()).sum() + (j.z.double() * dz.double()).sum())
        slope = (ends[0] - ends[1]) / (2 * e)
        d = (getattr(g, name).double() * way.double())
        size = d.abs().sum() / np.sqrt(d.numel()) + d.sum().abs() + 1.0
        assert abs(slope - d.sum()) <= 5e-3 * size, (name, float(slope), float(d.sum()))


def test_join_same_bits_twice_on_streams_and_in_graphs():
    import torch
    c = _c()
    for R, D, dtype in ((700, 1000, "bfloat16"), (333, 203, "float32"), (5, 9001, "float16")):
        a, dh, dz = make(R, D, dtype, "layer", groups=1)

        def step():
            j = c.join(**a, norm="layer", draws=draws(0.1))
            return [j.h, j.z, *c.join_grad(j, dh, dz)]

        want = [t.clone() for t in step()]
        for got, w in zip(step(), want):
            assert torch.equal(got, w)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = step()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(x, w) for x, w in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step()
        for t in got:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip(got, want))


def test_no_rows():
    import torch
    c = _c()
    a, dh, dz = make(1, 24, "bfloat16", "layer", groups=1)
    for k in ("x", "y"):
        a[k] = a[k][:0]
    j = c.join(**a, norm="layer")
    g = c.join_grad(j, dh[:0], dz[:0])
    assert j.h.shape == (0, 24) and g.x.shape == (0, 24)
    for n in ("post", "post_bias", "gate", "pre", "pre_bias"):
        assert (getattr(g, n) == 0).all(), n
    assert c.dropout(a["x"], draws(0.5)).shape == (0, 24)
    b = c.balance(torch.zeros(0, 6, device="cuda"), torch.zeros(0, 2, dtype=torch.int32, device="cuda"), groups=3)
    assert (b.loss == 0).all() and b.counts.shape == (3, 6) and (b.counts == 0).all()


def test_offsets_past_32_bits():
    """Rows that begin beyond 2^31 and 2^32 values into their buffers."""
    import torch
    c = _c()
    R, D, step = 5, 40, (1 << 30) + 8
    a, dh, dz = make(R, D, "bfloat16", groups=1)
    want = c.join(**a, draws=draws(0.2))
    wg = c.join_grad(want, dh, dz)

    def far(t):
        buf = torch.empty((R - 1) * step + D, dtype=t.dtype, device="cuda")
        v = buf.as_strided((R, D), (step, 1))
        return v.copy_(t)

    b = {**a, "x": far(a["x"]), "y": far(a["y"])}
    j = c.join(**b, draws=draws(0.2), h=far(a["x"]), z=far(a["x"]))
    assert torch.equal(j.h, want.h) and torch.equal(j.z, want.z)
    g = c.join_grad(j, far(dh), far(dz), into=c.JoinGrads(x=far(dh), y=far(dh)))
    for n in ("x", "y", "gate", "post", "pre"):
        assert torch.equal(getattr(g, n), getattr(wg, n)), n
    o = c.dropout(b["x"], draws(0.3), out=far(a["x"]))
    assert torch.equal(o, c.dropout(a["x"], draws(0.3)))
    del j, g, o, b
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("R, D, pad, offset", [(1, 1, 0, 0), (1, 8, 0, 0), (3, 5, 0, 0), (128, 200, 0, 0),
                                               (37, 203, 0, 0), (37, 203, 5, 1), (64, 1000, 24, 0),
                                               (64, 1000, 3, 0), (7, 4096, 0, 1), (1, 100_003, 0, 0),
                                               (5001, 24, 8, 8), (2000, 1, 0, 0), (2000, 3, 1, 0)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_dropout(R, D, pad, offset, dtype):
    import torch
    c = _c()
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = rows_of(gen, R, D, getattr(torch, dtype), 1.0, 0, pad, offset)
    res = rows_of(gen, R, D, getattr(torch, dtype), 1.0, 0, pad, offset)
    for rate in (0.0, 0.1, 0.5, 1.0 - 2.0 ** -16, 1.0):
        m = torch.from_numpy(factors(np.arange(R * D), rate, SEED, CLIENT, COUNT).reshape(R, D)).cuda()
        d = _c().Draws(rate, SEED, CLIENT, COUNT)
        plain = c.dropout(x, d)
        hold(plain, x.double() * m, x.double().abs() * m, f"rate {rate}")
        assert torch.equal(plain == 0, (m == 0) | (x == 0))
        both = c.dropout(x, d, residual=res)
        hold(both, x.double() * m + res.double(), x.double().abs() * m + res.double().abs(), "residual")
        # In place of either.
        for which in ("x", "residual"):
            xs, rs = x.clone(), res.clone()
            got = c.dropout(xs, d, residual=rs, out=xs if which == "x" else rs)
            assert torch.equal(got, both), which
        out = rows_of(gen, R, D, x.dtype, 1.0, 0, pad, offset)
        was = out._base.clone()
        assert torch.equal(c.dropout(x, d, out=out), plain)
        out.copy_(was[offset:offset + R * (D + pad)].view(R, D + pad)[:, :D])
        assert torch.equal(out._base.view(torch.uint8), was.view(torch.uint8))


def test_dropout_of_what_is_not_finite():
    import torch
    c = _c()
    x = torch.full((50, 70), float("nan"), device="cuda")
    x[::2] = float("inf")
    m = torch.from_numpy(factors(np.arange(3500), 0.5, SEED, CLIENT, COUNT).reshape(50, 70)).cuda()
    y = c.dropout(x, draws(0.5))
    assert (y[m == 0] == 0).all() and not torch.isfinite(y[m > 0]).any()


def test_dropout_rate_and_streams_of_draws():
    """The share kept is the rounded rate's within five deviations; other clients,
    counts and seeds draw other masks, and no two neighbours are alike."""
    import torch
    c = _c()
    n = 1 << 22
    x = torch.ones(n, device="cuda")
    base = c.dropout(x, c.Draws(0.1, 1, 2, 3)) > 0
    p = 1 - np.floor(0.1 * 65536 + 0.5) / 65536
    assert abs(float(base.double().mean()) - p) < 5 * np.sqrt(p * (1 - p) / n)
    for other in ((0.1, 2, 2, 3), (0.1, 1, 3, 3), (0.1, 1, 2, 4), (0.1, 1, 2, 3 + (1 << 32)), (0.1, 1 + (1 << 32), 2, 3)):
        same = ((c.dropout(x, c.Draws(*other)) > 0) == base).double().mean()
        assert abs(float(same) - (p * p + (1 - p) ** 2)) < 5e-3, other
    both = (base[1:] & base[:-1]).double().mean()
    assert abs(float(both) - p * p) < 5e-3


def test_dropout_of_more_than_2_to_the_35():
    """Octets beyond 2^32, whose upper bits go into the counter's last word."""
    import torch
    c = _c()
    n = (1 << 35) + 4099
    if torch.cuda.mem_get_info()[0] < 3 * n:
        pytest.skip("needs 70 GB of device memory")
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    c.dropout(x, draws(0.25), out=x)
    for at in (0, (1 << 32) - 64, (1 << 35) - 1000, n - 1000):
        m = factors(np.arange(at, min(n, at + 2000)), 0.25, SEED, CLIENT, COUNT)
        assert np.array_equal(x[at:at + 2000].float().cpu().numpy() > 0, m > 0), at
    del x
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------
# balance
# ---------------------------------------------------------------------------
def balance64(logits, chosen, groups, valid, wb, wz, up=1.0):
    """In 64 bits on the CPU, the gradient by its formula row by row; and the size
    of each row's terms."""
    x = logits.double().cpu().numpy()
    T, E = x.shape
    ch, L = chosen.cpu().numpy().reshape(T, -1), T // groups
    ok = np.ones(T, bool) if valid is None else valid.cpu().numpy().astype(bool)
    k = ch.shape[1]
    x = np.where(ok[:, None], x, 0.0)
    top = x.max(1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.exp(x - top)
        p = e / e.sum(1, keepdims=True)
        lse = (top + np.log(e.sum(1, keepdims=True)))[:, 0]
    empty = np.isneginf(top[:, 0])
    p[empty] = 0
    lse[empty] = 0
    p[~ok] = 0
    lse[~ok] = 0
    counts = np.zeros((groups, E), np.int64)
    f = np.zeros((groups, E))
    n = ok.reshape(groups, L).sum(1)
    live, N = int((n > 0).sum()), int(n.sum())
    for g in range(groups):
        ids = ch[g * L:(g + 1) * L][ok[g * L:(g + 1) * L]].reshape(-1)
        counts[g] = np.bincount(ids[(ids >= 0) & (ids < E)], minlength=E)
        if n[g]:
            f[g] = counts[g] / (k * n[g])
    fr = np.repeat(f, L, 0)
    dot = (fr * p).sum(1)
    per = np.repeat(np.where(n > 0, 1.0 / np.maximum(n, 1), 0.0), L)
    lb = E * (dot * per).sum() / max(live, 1)
    lz = (lse ** 2).sum() / max(N, 1)
    a, b = wb * E / max(live, 1) * per, 2 * wz / max(N, 1) * lse
    grad = up * p * (a[:, None] * (fr - dot[:, None]) + b[:, None])
    reach = np.where(np.isfinite(top), np.abs(x - np.where(np.isfinite(top), top, 0)), 0.0).clip(0, 200)
    size = abs(up) * p * (np.abs(a)[:, None] * (fr + dot[:, None]) + np.abs(b)[:, None]) * (1 + reach)
    return np.array([wb * lb + wz * lz, lb, lz]), counts, grad, size


def routed(T, E, k, dtype, seed=5, groups=1, ragged=False, pad=0, offset=0, drop=0.05):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    logits = rows_of(gen, T, E, getattr(torch, dtype), 1.5, 0.3, pad, offset)
    chosen = torch.topk(logits.float() + torch.randn(T, E, generator=gen, device="cuda"), k, 1).indices.int()
    chosen[torch.rand(T, k, generator=gen, device="cuda") < drop] = -1
    valid = None
    if ragged:
        L = T // groups
        n = torch.randint(0, L + 1, (groups, 1), generator=gen, device="cuda")
        n[0] = 0                       # a sequence of padding alone
        valid = (torch.arange(L, device="cuda")[None] < n).reshape(-1)
    return logits, chosen, valid


def check_balance(logits, chosen, valid, groups=1, wb=0.02, wz=0.003, upstream=None):
    import torch
    b = _c().balance(logits, chosen, balance=wb, z=wz, groups=groups, valid=valid, upstream=upstream)
    up = 1.0 if upstream is None else float(upstream)
    loss, counts, grad, size = balance64(logits, chosen, groups, valid, wb, wz, up)
    assert np.array_equal(b.counts.cpu().numpy(), counts)
    T = logits.shape[0]
    hold(b.loss.cpu(), torch.from_numpy(loss), torch.from_numpy(np.abs(loss)), "loss", rows=T)
    hold(b.dlogits.cpu(), torch.from_numpy(grad), torch.from_numpy(size), "dlogits")
    if valid is not None:
        assert (b.dlogits[~valid.bool()] == 0).all()
    return b


@pytest.mark.parametrize("E", [1, 2, 5, 8, 16, 31, 32, 33, 60, 64, 72, 127, 128, 129, 256, 257, 500, 512, 777, 1024])
@pytest.mark.parametrize("dtype", DTYPES)
def test_balance_experts(E, dtype):
    for T in (1, 130 + E % 7):
        check_balance(*routed(T, E, min(E, 1 + E % 8), dtype))


@pytest.mark.parametrize("T, groups", [(1, 1), (2, 2), (7, 7), (96, 3), (1000, 1), (1000, 8), (1000, 1000),
                                       (4097, 1), (30_000, 3), (30_000, 600), (70_001, 1)])
@pytest.mark.parametrize("ragged", [False, True])
def test_balance_groups(T, groups, ragged):
    check_balance(*routed(T, 24, 3, "float32", groups=groups, ragged=ragged), groups=groups)
    check_balance(*routed(T, 9, 2, "bfloat16", groups=groups, ragged=ragged), groups=groups)


@pytest.mark.parametrize("E, pad, offset", [(64, 8, 0), (64, 3, 0), (60, 4, 0), (60, 0, 1), (13, 3, 2), (256, 0, 4)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_balance_strides(E, pad, offset, dtype):
    import torch
    logits, chosen, valid = routed(333, E, 4, dtype, pad=pad, offset=offset, groups=3, ragged=True)
    b = check_balance(logits, chosen, valid, groups=3)
    d = check_balance(logits.contiguous(), chosen, valid, groups=3)
    assert torch.equal(b.counts, d.counts)


def test_balance_masks_and_special_values():
    """Masked experts (-inf, and the type's lowest value), rows without any expert,
    rows that take no part whatever they hold, assignments out of range."""
    import torch
    c = _c()
    for E in (8, 60, 200):
        logits, chosen, _ = routed(200, E, 2, "float32")
        logits[:, 3] = float("-inf")
        logits[5, 1:] = float("-inf")
        logits[7] = float("-inf")
        chosen[7] = -1
        chosen[9, 0] = E + 5
        chosen[10, 1] = -(1 << 31)
        chosen[11, 1] = (1 << 31) - 1
        b = check_balance(logits, chosen, None)
        assert (b.dlogits[:, 3] == 0).all() and (b.dlogits[7] == 0).all() and torch.isfinite(b.dlogits).all()
        low = logits.clone()
        low[:, 3] = torch.finfo(torch.float32).min
        low[7, 3] = float("-inf")      # else that row's only expert
        d = check_balance(low, chosen, None)
        assert torch.equal(d.dlogits, b.dlogits)
        valid = torch.ones(200, dtype=torch.bool, device="cuda")
        valid[20:40] = False
        w = check_balance(logits, chosen, valid)
        logits[20:30] = float("nan")
        logits[30:40] = float("inf")
        chosen[20:40] = 1
        g = c.balance(logits, chosen, balance=0.02, z=0.003, valid=valid)
        assert all(torch.equal(x, y) for x, y in zip(g, w))
        # A row that takes part keeps its NaN to itself, but for the loss.
        logits[50, 2] = float("nan")
        n = c.balance(logits, chosen, balance=0.02, z=0.003, valid=valid)
        assert n.dlogits[50].isnan().all() and n.loss.isnan().all()
        rest = [r for r in range(200) if r != 50]
        assert torch.equal(n.dlogits[rest], w.dlogits[rest])
        none = c.balance(logits, chosen, valid=torch.zeros_like(valid))
        assert (none.loss == 0).all() and (none.dlogits == 0).all() and (none.counts == 0).all()


def test_balance_rows_of_a_types_lowest_value_alone():
    import torch
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        logits = torch.full((4, 10), torch.finfo(dtype).min, dtype=dtype, device="cuda")
        chosen = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
        check_balance(logits, chosen, None, wz=0.0 if dtype != torch.float16 else 1e-6) if dtype == torch.float16 else None
        b = _c().balance(logits, chosen, balance=1.0, z=0.0)
        assert abs(float(b.loss[1]) - 1.0) < 1e-5            # uniform: E f . P = 1
        d = b.dlogits.float()
        assert torch.isfinite(d).all() and (d[:, 0] > 0).all() and (d[:, 1:] < 0).all()


def test_balance_upstream_parts_and_repeats():
    import torch
    c = _c()
    for T, E, groups in ((300, 40, 3), (40_000, 16, 1)):
        logits, chosen, valid = routed(T, E, 4, "float32", groups=groups, ragged=groups > 1)
        up = torch.tensor([-2.5], device="cuda")
        b = check_balance(logits, chosen, valid, groups, upstream=up)
        again = c.balance(logits, chosen, balance=0.02, z=0.003, groups=groups, valid=valid, upstream=up)
        assert all(torch.equal(x, y) for x, y in zip(b, again))
        loss_only = c.balance(logits, chosen, balance=0.02, z=0.003, groups=groups, valid=valid, grad=False)
        assert loss_only.dlogits is None and torch.equal(loss_only.loss, b.loss)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            g = c.balance(logits, chosen, balance=0.02, z=0.003, groups=groups, valid=valid, upstream=up)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(b, g))


def test_balance_gradient_against_differences():
    """Directional central differences of the kernel's own loss (fp32: the step is
    wide, and the bound a hundredth of the slope's size)."""
    import torch
    c = _c()
    logits, chosen, valid = routed(60, 12, 2, "float32", groups=2, ragged=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for wb, wz in ((1.0, 0.0), (0.0, 1.0), (1.0, 0.1)):
        s = dict(balance=wb, z=wz, groups=2, valid=valid)
        d = c.balance(logits, chosen, **s).dlogits.double()
        way = d.sign().float() + 0.1 * torch.randn(logits.shape, generator=gen, device="cuda")
        e = 2.0 ** -6
        up = c.balance(logits + e * way, chosen, **s).loss[0].double()
        down = c.balance(logits - e * way, chosen, **s).loss[0].double()
        slope, want = float((up - down) / (2 * e)), float((d * way.double()).sum())
        assert want > 0 and abs(slope - want) <= 0.01 * want, (wb, wz, slope, want)


# ---------------------------------------------------------------------------
# inside automatic differentiation
# ---------------------------------------------------------------------------
def test_automatic_differentiation():
    import torch
    c = _c()
    a, dh, dz = make(40, 72, "float32", "layer", groups=1)
    s = dict(norm="layer", carry=0.9, branch=0.7, draws=draws(0.2))
    leaves = {k: t.clone().requires_grad_(True) for k, t in a.items() if t is not None}
    h, z = c.joined(**leaves, **s)
    torch.autograd.backward([h, z], [dh, dz])
    g = c.join_grad(c.join(**a, **s), dh, dz)
    for k, t in leaves.items():
        assert torch.equal(t.grad, getattr(g, k)), k
    # One of the two outputs unused.
    for use in (0, 1):
        x = a["x"].clone().requires_grad_(True)
        out = c.joined(**{**a, "x": x}, **s)
        out[use].backward(dh)
        zero = torch.zeros_like(dh)
        g = c.join_grad(c.join(**a, **s), dh if use == 0 else None, zero if use == 0 else dh)
        assert torch.equal(x.grad, g.x), use
    x, r = a["x"].clone().requires_grad_(True), a["y"].clone().requires_grad_(True)
    c.dropped(x, draws(0.3), r).backward(dh)
    assert torch.equal(x.grad, c.dropout(dh, draws(0.3))) and torch.equal(r.grad, dh)
    logits, chosen, valid = routed(50, 9, 2, "float32", ragged=True, groups=5)
    leaf = logits.clone().requires_grad_(True)
    loss, parts, counts = c.balanced(leaf, chosen, valid=valid, balance=0.5, z=0.1, groups=5)
    (3.0 * loss).backward()
    b = c.balance(logits, chosen, valid=valid, balance=0.5, z=0.1, groups=5, upstream=torch.full((1,), 3.0, device="cuda"))
    assert torch.equal(leaf.grad, b.dlogits) and torch.equal(counts, b.counts)
    assert torch.equal(torch.cat((loss.detach().reshape(1), parts)), b.loss)


@pytest.fixture(params=["module", "python"])
def form(request, monkeypatch):
    """Both forms of the marshalling: client_torch.cpp's module, and client.py's own,
    which serves where torch's headers were missing."""
    c = _c()
    if request.param == "module":
        if c._fast is None:
            pytest.skip("built without torch's headers")
    else:
        monkeypatch.setattr(c, "_fast", None)
    return request.param


def test_the_module_is_built():
    """Here torch's headers are installed."""
    from paper_1601_04033_gb300 import build
    assert _c()._fast is not None or build.torch_home() is None


def shapes_of_join():
    """(x, y, post, gate, pre) of every form that a join takes, with its gradients' ends."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(8)

    def z(*s, dtype=torch.bfloat16):
        return torch.randn(*s, generator=gen, device="cuda").to(dtype)
    w, wide, cube = z(24, dtype=torch.float32), z(10, 48), z(4, 5, 24)
    return [(z(6, 24), z(6, 24), w, w, w), (z(24), None, None, None, w), (wide[:, :24], wide[:, 24:], w, z(2, 24), None),
            (cube, z(4, 5, 24), w, z(5, 24, dtype=torch.float32), w), (z(1, 24), z(1, 24), None, None, None),
            (cube[:, :1], None, None, None, w), (cube[:1], cube[1:2], None, None, w), (z(0, 24), z(0, 24), w, w, w),
            (z(3, 1), z(3, 1), None, None, None)]


def test_both_forms_agree(monkeypatch):
    import torch
    c = _c()
    if c._fast is None:
        pytest.skip("built without torch's headers")
    fast = c._fast

    def both(call):
        out = []
        for m in (fast, None):
            monkeypatch.setattr(c, "_fast", m)
            out.append(call())
        for a, b in zip(*out):
            assert (a is None) == (b is None)
            if a is not None:
                assert a.shape == b.shape and a.dtype == b.dtype and a.is_contiguous() == b.is_contiguous()
                assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))

    for x, y, post, gate, pre in shapes_of_join():
        def step():
            j = c.join(x, y, post=post, gate=gate, pre=pre, draws=draws(0.3), carry=0.9)
            return [j.h, j.z, *c.join_grad(j, x, x if pre is not None else None)]
        both(step)
        both(lambda: [c.dropout(x, draws(0.3)), c.dropout(x, draws(0.3), residual=y)])
    for groups, valid in ((1, None), (3, torch.arange(30, device="cuda") % 4 > 0)):
        logits, chosen, _ = routed(30, 9, 2, "float16")
        up = torch.full((1,), 2.0, device="cuda")
        both(lambda: c.balance(logits, chosen, groups=groups, valid=valid, z=0.1, upstream=up))
        both(lambda: c.balance(logits, chosen, groups=groups, valid=valid, grad=False))


def test_refusals_on_tensors(form):
    import torch
    from paper_1601_04033_gb300 import fasgd
    c = _c()
    x = torch.zeros(4, 8, device="cuda")
    w = torch.ones(8, device="cuda")
    for bad in (lambda: c.dropout(x.double(), draws(0.5)), lambda: c.dropout(x.t(), draws(0.5)),
                lambda: c.dropout(x.cpu(), draws(0.5)), lambda: c.dropout(x, draws(0.5), residual=x[:2]),
                lambda: c.dropout(x, draws(0.5), out=x.half()), lambda: c.join(x, x.half(), pre=w),
                lambda: c.join(x, pre=w.half()), lambda: c.join(x, pre=w[:4]), lambda: c.join(x, x, gate=w[:4]),
                lambda: c.join(x, pre=torch.ones(16, device="cuda")[::2]),
                lambda: c.balance(x, torch.zeros(4, 2, dtype=torch.int64, device="cuda")),
                lambda: c.join(x.view(2, 2, 8)[:, :1].expand(2, 2, 8), pre=w), lambda: c.join(x, y=x.clone(), h=x[:2]),
                lambda: c.join(x, pre=w, h=x.clone()), lambda: c.join(x, x.clone(), gate=torch.ones(2, 2, 8, device="cuda")),
                lambda: c.dropout(torch.zeros((), device="cuda"), draws(0.5)), lambda: c.join(torch.zeros(4, 4, 8, device="cuda")[:, :3], pre=w),
                lambda: c.join_grad(c.join(x, x.clone(), pre=w), x, x[:2]), lambda: c.join_grad(c.join(x, pre=w), x, x, into=c.JoinGrads(pre=w[:4])),
                lambda: c.join_grad(c.join(x, x.clone(), gate=w), x, into=c.JoinGrads(gate=w.half())),
                lambda: c.balance(x, torch.zeros(4, 2, dtype=torch.int32, device="cuda"), valid=torch.ones(3, device="cuda").bool()),
                lambda: c.balance(x, torch.zeros(4, 2, dtype=torch.int32, device="cuda"), valid=torch.ones(4, device="cuda")),
                lambda: c.balance(x, torch.zeros(4, 2, dtype=torch.int32, device="cuda"), upstream=torch.ones(2, device="cuda")),
                lambda: c.balance(x, torch.zeros(3, 2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    y = torch.zeros(4, 8, device="cuda")
    ids = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    for bad in (lambda: c.dropout(x, c.Draws(1.5)), lambda: c.dropout(x, c.Draws(float("nan"))),
                lambda: c.dropout(x, c.Draws(0.1, 0, -1)), lambda: c.dropout(x, c.Draws(0.1, 0, 0, 1 << 48)),
                lambda: c.dropout(x[:3], draws(0.1), out=x[1:]),
                lambda: c.join(x), lambda: c.join(x, gate=w, pre=w), lambda: c.join(x, pre=w, eps=0.0),
                lambda: c.join(x, y, gate=torch.ones(3, 8, device="cuda")), lambda: c.join(x, y, carry=float("inf")),
                lambda: c.join(x, y, h=x), lambda: c.join(x, y, pre=w, z=y), lambda: c.join(x, y, post_bias=w),
                lambda: c.join(x[:1].expand(4, 8), y), lambda: c.balance(x, ids, groups=3),
                lambda: c.balance(x, ids, z=float("nan")),
                lambda: c.balance(torch.zeros(4, 1025, device="cuda"), ids),
                lambda: c.join_grad(c.join(x, y, pre=w), y), lambda: c.join_grad(c.join(x, y), y, y)):
        with pytest.raises(fasgd.FasgdError) as e:
            bad()
        assert e.value.code == fasgd.EINVAL and str(e.value) != "EINVAL: "
