"""The client operators inside torch's automatic differentiation where the tensors of
the forward call are gone by the time of the backward call: activation
checkpointing and saved-tensor hooks; both forms of the marshalling."""

import pytest

from test_gpu_client import _c, draws, make

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["module", "python"])
def client(request, monkeypatch):
    c = _c()
    if request.param == "module":
        if c._fast is None:
            pytest.skip("built without torch's headers")
    else:
        monkeypatch.setattr(c, "_fast", None)
    return c


def overwrite():
    """What torch's allocator has free, written over."""
    import torch
    keep = [torch.full((n,), float("nan"), device="cuda") for n in (64, 256, 1 << 10, 1 << 14, 1 << 16, 1 << 20) * 40]
    torch.cuda.synchronize()
    del keep


def block(c, leaves, x, place, norm):
    """A residual block whose x, y and parameters are all intermediate tensors."""
    import torch
    y = torch.tanh(x @ leaves["w"]) + 0.1
    s = {k: leaves[k] * (1.0 + 0.01 * place) for k in ("post", "gate", "pre")}
    if norm == "layer":
        s.update({k: leaves[k] * 1.01 for k in ("post_bias", "pre_bias")})
    h, z = c.joined(x * 1.0, y, **s, norm=norm, carry=0.9, branch=0.7, draws=draws(0.2))
    return h + 0.5 * c.dropped(z, draws(0.3))


def gradients(c, D, dtype, norm, through):
    import torch
    a, dh, _ = make(37, D, dtype, norm, groups=1)
    gen = torch.Generator(device="cuda").manual_seed(6)
    leaves = {k: t for k, t in a.items() if t is not None and k != "y"}
    leaves["w"] = (torch.randn(D, D, generator=gen, device="cuda") * D ** -0.5).to(a["x"].dtype)
    leaves = {k: t.clone().requires_grad_(True) for k, t in leaves.items()}
    x = leaves["x"]
    for place in range(3):
        x = through(lambda x, place=place: block(c, leaves, x, place, norm), x)
    overwrite()
    x.backward(dh)
    return {k: t.grad for k, t in leaves.items()}


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("D, dtype", [(40, "float32"), (200, "bfloat16"), (203, "float32")])
def test_checkpoints_and_hooks_give_the_same_gradients(client, D, dtype, norm):
    import torch
    from torch.utils.checkpoint import checkpoint
    graph = torch.autograd.graph
    want = gradients(client, D, dtype, norm, lambda f, x: f(x))
    assert all(torch.isfinite(t).all() and (t != 0).any() for t in want.values())

    def hooked(f, x):
        with graph.saved_tensors_hooks(lambda t: t.detach().clone(), lambda t: t.clone()):
            return f(x)

    def on_cpu(f, x):
        with graph.save_on_cpu():
            return f(x)

    for through in (lambda f, x: checkpoint(f, x, use_reentrant=False), lambda f, x: checkpoint(f, x, use_reentrant=True),
                    hooked, on_cpu):
        got = gradients(client, D, dtype, norm, through)
        for k, t in want.items():
            assert torch.equal(got[k], t), k


def test_rows_that_lay_apart_come_back_without_gaps(client):
    """A hook may hand back a tensor of another layout, with gates of groups too.
    Another kernel then takes the rows: 64 roundings of 2^-24 of a row's terms, which
    are below 200 here, stay below 1e-3; what was overwritten is NaN."""
    import contextlib
    import torch
    a, dh, dz = make(24, 72, "float32", groups=3, pad=5, offset=1)

    def apart(t):
        return t._base.clone()[1:1 + 24 * 77].view(24, 77)[:, :72]

    def grads(context, gone):
        leaves = {k: apart(t) if k in ("x", "y") else t.clone() for k, t in a.items() if t is not None}
        leaves = {k: t.requires_grad_(True) for k, t in leaves.items()}
        with context:
            h, z = client.joined(**leaves, carry=0.9, draws=draws(0.2))
        if gone:
            for t in leaves.values():
                t.data.fill_(float("nan"))
            overwrite()
        torch.autograd.backward([h, z], [dh, dz])
        return {k: t.grad for k, t in leaves.items()}

    want = grads(contextlib.nullcontext(), False)
    got = grads(torch.autograd.graph.saved_tensors_hooks(
        lambda t: t.detach().clone(memory_format=torch.contiguous_format), lambda t: t), True)
    for k, t in want.items():
        torch.testing.assert_close(got[k], t, rtol=1e-3, atol=1e-3)


def test_second_derivatives_of_dropout(client):
    """Inside a graph of the backward call: d2/dx2 of sum (m x + r)^3 + x^2, on the
    diagonal 6 (m x + r) m^2 + 2; two roundings each way of 2^-24."""
    import torch
    a, _, _ = make(9, 203, "float32", post=False)
    x, r = a["x"].clone().requires_grad_(True), a["y"].clone().requires_grad_(True)
    d = draws(0.3)
    (g,) = torch.autograd.grad((client.dropped(x, d, r) ** 3).sum() + (x * x).sum(), x, create_graph=True)
    gx, gr = torch.autograd.grad(g.sum(), (x, r))
    m = client.dropout(torch.ones_like(a["x"]), d)
    u = 6 * (a["x"] * m + a["y"])
    torch.testing.assert_close(gx, u * m * m + 2, rtol=1e-5, atol=1e-5)
    torch.testing.assert_close(gr, u * m, rtol=1e-5, atol=1e-5)


def test_other_second_derivatives_are_refused(client):
    """Also where the gradient handed in is a constant; first derivatives made with a
    graph are as without one, and the other paths' second derivatives stay."""
    import torch
    a, dh, dz = make(9, 72, "float32", groups=1)

    def leaves():
        return {k: t.clone().requires_grad_(True) for k, t in a.items() if t is not None}

    v = leaves()
    plain = torch.autograd.grad([t for t in client.joined(**v)], list(v.values()), [dh, dz])
    for power in (1, 2):
        v = leaves()
        h, z = client.joined(**v)
        grads = torch.autograd.grad((h * dh).sum() + (z ** power * dz).sum(), list(v.values()), create_graph=True)
        if power == 1:
            assert all(torch.equal(g, w) for g, w in zip(grads, plain))
        for g in grads:
            assert g.requires_grad
            with pytest.raises(RuntimeError, match="second derivatives"):
                torch.autograd.grad(g.sum(), v["x"], retain_graph=True)
        with pytest.raises(RuntimeError, match="second derivatives"):
            (sum(g.sum() for g in grads) + (v["x"] ** 3).sum()).backward()
    logits = torch.randn(12, 8, device="cuda").requires_grad_(True)
    chosen = torch.zeros(12, 2, dtype=torch.int32, device="cuda")
    loss, _, _ = client.balanced(logits, chosen, z=0.1)
    (want,) = torch.autograd.grad(loss, logits, retain_graph=True)
    (g,) = torch.autograd.grad(loss, logits, create_graph=True)
    assert torch.equal(g, want)
    with pytest.raises(RuntimeError, match="second derivatives"):
        (g * g).sum().backward()
    # A graph of the backward call that is not differentiated through the operators.
    x = a["x"].clone().requires_grad_(True)
    w = a["pre"].clone().requires_grad_(True)
    h, z = client.joined(x.detach(), pre=w)
    (z.sum() + (x ** 3).sum()).backward(create_graph=True)
    (second,) = torch.autograd.grad(x.grad.sum(), x)
    assert torch.equal(second, 6 * a["x"])


def test_writes_into_saved_tensors_are_noticed(client):
    """A tensor that an earlier operation saved and a call then writes into: its backward
    raises, as after any other in-place operation."""
    import torch
    a, dh, dz = make(6, 24, "float32", groups=1)
    w = a["pre"]
    j = client.join(**a)
    calls = [lambda t, v: client.dropout(a["x"], draws(0.3), out=t), lambda t, v: client.dropout(t, draws(0.3), out=t),
             lambda t, v: client.join(**a, h=t), lambda t, v: client.join(**a, z=t)]
    for name in client.JoinGrads._fields:
        if name in ("x", "y"):
            calls.append(lambda t, v, name=name: client.join_grad(j, dh, dz, into=client.JoinGrads(**{name: t})))
        elif a[name] is not None:
            calls.append(lambda t, v, name=name: client.join_grad(j, dh, dz, into=client.JoinGrads(**{name: v})))
    assert len(calls) == 9
    for call in calls:
        leaf, vector = a["x"].clone().requires_grad_(True), w.clone().requires_grad_(True)
        t, v = leaf * 1.0, vector * 1.0
        out = (t * t).sum() + (v * v).sum()
        with torch.no_grad():
            call(t, v)
        with pytest.raises(RuntimeError, match="inplace"):
            out.backward()
    # Inference tensors have no version; new tensors and what is only read keep theirs.
    with torch.inference_mode():
        x = a["x"].clone()
        assert torch.equal(client.dropout(x, draws(0.3), out=x), client.dropout(a["x"], draws(0.3)))
        client.join(**a, h=x)
    assert client.join(**a).h._version == 0 and all(t._version <= 1 for t in (a["x"], dh))
