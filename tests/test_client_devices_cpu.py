"""Tensors of a client operator's call that are on another GPU than the first, or on
none, are refused before an address is taken or the library is called: tensors
without memory, which only say where they are, on a machine without a GPU."""

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_1601_04033_gb300 import build

NAMES = ("post", "post_bias", "gate", "pre", "pre_bias")


@pytest.fixture(params=["module", "python"])
def client(request, monkeypatch):
    build.build()
    from paper_1601_04033_gb300 import client as c, fasgd

    def reached(*_):
        raise AssertionError("the library was called")

    for name in ("fasgd_dropout", "fasgd_join", "fasgd_join_grad", "fasgd_balance", "fasgd_join_workspace",
                 "fasgd_balance_workspace"):
        monkeypatch.setattr(fasgd, name, reached)
    if request.param == "module":
        if c._fast is None:
            pytest.skip("built without torch's headers")
    else:
        monkeypatch.setattr(c, "_fast", None)
    return c


def calls(c):
    """(name, the call, its tensors by name)."""
    def new(*size, dtype=torch.float32):
        return torch.empty(*size, dtype=dtype, device="cuda:0")

    def record(v):
        j = c.Joined()
        j.x, j.y, j.stats = v["x"], v["y"], v["stats"]
        j.parameters = tuple(v[n] for n in NAMES)
        j.args = bytes(c._f.JoinArgs(rows=4, cols=8, groups=1, x=16, y=16, post=16, pre=16, norm=1, eps=1e-6))
        return j

    w, x = (8,), (4, 8)
    yield "dropout", lambda v: c.dropout(v["x"], c.Draws(0.5), residual=v["residual"], out=v["out"]), \
        {n: new(*x) for n in ("x", "residual", "out")}
    yield "join", lambda v: c.join(**v, norm="layer"), \
        {n: new(*(x if n in "xyhz" else w)) for n in ("x", "y", "h", "z", *NAMES)}
    into = {"into_" + n: new(*(x if n in "xy" else w)) for n in ("x", "y", *NAMES)}
    yield "join_grad", lambda v: c.join_grad(record(v), v["dh"], v["dz"], into=c.JoinGrads(
        **{n[5:]: t for n, t in v.items() if n.startswith("into_")})), \
        {**{n: new(*(x if n in ("x", "y", "dh", "dz") else w)) for n in ("x", "y", "dh", "dz", *NAMES)},
         "stats": new(16), **into}
    yield "balance", lambda v: c.balance(v["logits"], v["chosen"], valid=v["valid"], upstream=v["upstream"]), \
        {"logits": new(*x), "chosen": new(4, 2, dtype=torch.int32), "valid": new(4, dtype=torch.bool), "upstream": new(1)}


@pytest.mark.parametrize("where", ["cuda:1", "cpu"])
def test_tensors_of_another_device_are_refused(client, where):
    if where == "cuda:1" and torch.cuda.device_count() == 1:
        pytest.skip("torch looks for the second GPU where there is one")
    with FakeTensorMode(allow_non_fake_inputs=True):
        tried = 0
        for name, call, tensors in calls(client):
            for moved in tensors:
                v = {n: torch.empty_like(t, device=where) if n == moved else t for n, t in tensors.items()}
                with pytest.raises(ValueError, match="one device"):
                    call(v)
                tried += 1
    assert tried == 3 + 9 + 17 + 4
