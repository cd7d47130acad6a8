"""The join inside automatic differentiation, on the host: the gradient call gets the
addresses of the tensors that backward is handed, not those of the forward call's
(saved-tensor hooks and activation checkpointing hand back others).  CPU tensors
stand for CUDA ones and the library's calls record their argument structs."""

import ctypes

import pytest
import torch

from paper_1601_04033_gb300 import build


@pytest.fixture
def recorded(monkeypatch):
    """(client, the structs of the gradient calls): client.py's own marshalling, the
    library's calls recorded instead of made."""
    build.build()
    from paper_1601_04033_gb300 import client, fasgd
    calls = []

    def grad(at, stream):
        calls.append(fasgd.JoinArgs.from_buffer_copy(ctypes.string_at(at, ctypes.sizeof(fasgd.JoinArgs))))
        return 0

    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)      # what tensors say
    monkeypatch.setattr(client, "_fast", None)
    monkeypatch.setattr(client, "_stream", lambda t: 0)
    monkeypatch.setattr(fasgd, "fasgd_join", lambda at, stream: 0)
    monkeypatch.setattr(fasgd, "fasgd_join_workspace", lambda at: 64)
    monkeypatch.setattr(fasgd, "fasgd_join_grad", grad)
    return client, calls


NAMES = ("x", "y", "post", "post_bias", "gate", "pre", "pre_bias", "stats")


@pytest.mark.parametrize("gate", ["vector", "groups"])
def test_gradients_read_what_backward_is_handed(recorded, gate):
    client, calls = recorded
    R, D = 6, 24
    wide = torch.randn(R, 2 * D)

    def leaf(*size):
        return torch.randn(*size).requires_grad_(True)

    args = dict(x=wide[:, :D].requires_grad_(True), y=wide[:, D:].requires_grad_(True), post=leaf(D), post_bias=leaf(D),
                gate=leaf(D) if gate == "vector" else leaf(3, D), pre=leaf(D), pre_bias=leaf(D))
    handed = []

    def unpack(t):
        t = t.detach().clone(memory_format=torch.contiguous_format)
        handed.append(t)
        return t

    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
        h, z = client.joined(**args, norm="layer", carry=0.5, draws=client.Draws(0.25, 7, 3, 9))
    (h.sum() + z.sum()).backward()
    assert len(calls) == 1 and len(handed) == len(NAMES)
    a = calls[0]
    for name, t in zip(NAMES, handed):
        assert getattr(a, name) == t.data_ptr(), name
    # Rows that lay apart came back without gaps.
    assert a.ld_x == a.ld_y == D and (a.rows, a.cols, a.groups) == (R, D, 1 if gate == "vector" else 3)
    assert (a.norm, a.carry, a.rate, a.seed, a.client, a.n) == (1, 0.5, 0.25, 7, 3, 9)


def test_gradients_refuse_other_tensors(recorded):
    client, calls = recorded
    x, y, w = (torch.randn(*s) for s in ((6, 24), (6, 24), (24,)))
    j = client.join(x, y, post=w, pre=w)
    good = {n: getattr(j, n) for n in ("x", "y", "parameters", "stats")}
    for change in (dict(x=x[:4], y=y[:4]), dict(y=None), dict(parameters=(None, None, None, w, None)),
                   dict(parameters=(w, None, torch.randn(3, 24), w, None)), dict(stats=j.stats[:8]),
                   dict(stats=j.stats.double())):
        for n, t in {**good, **change}.items():
            setattr(j, n, t)
        with pytest.raises(ValueError):
            client.join_grad(j, x, x)
    assert not calls
