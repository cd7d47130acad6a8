"""Arguments of a client operator's call that are refused: numbers beyond their fields, not cut
to another client's or another call's, and places for gradients of what is not there."""

import pytest

from test_gpu_client import _c

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


def test_draws_beyond_their_fields(client):
    import torch
    from paper_1601_04033_gb300 import fasgd
    x = torch.ones(4, 256, device="cuda")
    for who, n in (((1 << 32) + 5, 3), (1 << 31, 3), (1 << 30, 3), (1 << 64, 3), (-1, 3), (5 - (1 << 32), 3),
                   (5 - (1 << 64), 3), (5, 1 << 48), (5, 1 << 63), (5, (1 << 64) + 3), (5, -1), (5, 3 - (1 << 64)),
                   (5, 3 - (1 << 70))):
        d = client.Draws(0.5, 7, who, n)
        for call in (lambda: client.dropout(x, d), lambda: client.join(x, x.clone(), draws=d)):
            with pytest.raises(fasgd.FasgdError, match="client|n must") as e:
                call()
            assert e.value.code == fasgd.EINVAL
    for who, n in ((0, 0), ((1 << 30) - 1, (1 << 48) - 1)):
        assert torch.equal(client.dropout(x, client.Draws(0.5, 7 - (1 << 64), who, n)),
                           client.dropout(x, client.Draws(0.5, 7, who, n)))


def test_groups_beyond_their_field(client):
    import torch
    x, ids = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    for groups in ((1 << 64) + 1, 1 - (1 << 64), 1 << 63):
        with pytest.raises(OverflowError):
            client.balance(x, ids, groups=groups)


def test_gradients_of_absent_tensors_are_refused(client):
    """`into` for a tensor that the join does not have: no unwritten tensor is handed back."""
    import torch
    x, w = torch.ones(4, 8, device="cuda"), torch.ones(8, device="cuda")
    full = client.join(x, x.clone(), post=w, gate=w, pre=w)
    for j, absent in ((full, ("post_bias", "pre_bias")), (client.join(x, pre=w), ("y", "post", "post_bias", "gate", "pre_bias")),
                      (client.join(x, x.clone()), ("post", "post_bias", "gate", "pre", "pre_bias"))):
        dz = x if j.z is not None else None
        for name in absent:
            d = torch.full_like(x if name == "y" else w, 5.0)
            with pytest.raises(ValueError, match="not there"):
                client.join_grad(j, x, dz, into=client.JoinGrads(**{name: d}))
            assert (d == 5.0).all()
        g = client.join_grad(j, x, dz)
        assert all(getattr(g, name) is None for name in absent)
