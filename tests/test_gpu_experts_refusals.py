"""Tensors of the routed experts' and the score's calls that do not fit each other are
refused before the library is called, by the torch module and in Python."""

import pytest

from test_experts_cpu import calls, client, f  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_wrong_tensors_are_refused(client):  # noqa: F811
    def new(*size, dtype=torch.float32):
        return torch.empty(*size, dtype=dtype, device="cuda:0")

    other = {
        "chosen": [new(6, 2), new(6, 4, dtype=torch.int32)[:, ::2], new(6, 2, dtype=torch.int64)],
        "order": [new(11, dtype=torch.int32), new(12, dtype=torch.int64), new(24, dtype=torch.int32)[::2]],
        "place": [new(6, 3, dtype=torch.int32), new(6, 2), new(6, 4, dtype=torch.int32)[:, ::2]],
        "offsets": [new(5, dtype=torch.int32), new(4, dtype=torch.int64), new(3, dtype=torch.int32)],
        "labels": [new(5, dtype=torch.int64), new(6, dtype=torch.int32), new(6)],
        "weight": [new(6, 3), new(6, 2, dtype=torch.bfloat16), new(2, 6).t()],
        "dweight": [new(5, 2), new(6, 2, dtype=torch.float16)],
        "upstream": [new(2), new(1, dtype=torch.float64)],
        "lse": [new(5), new(6, dtype=torch.float64)],
        "rows": [new(7), new(12)[::2]],
    }
    tried = 0
    for call, tensors in calls(client):
        for name, t in tensors.items():
            wrong = other.get(name)
            if wrong is None:
                wrong = [t.half(), t.double(), new(*t.shape[:-1], t.shape[-1] + 1), new(*t.shape[:-2], t.shape[-2] + 1, t.shape[-1]),
                         new(*t.shape, 2)[..., 0]]
            for w in wrong:
                with pytest.raises(ValueError):
                    call({**tensors, name: w})
                tried += 1
    assert tried > 100
