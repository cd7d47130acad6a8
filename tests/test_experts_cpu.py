"""The routed experts' and the score's entry points on a machine without a GPU: the
binding's structs are the header's, and bad arguments are rejected on the host."""

import ctypes
import re
import subprocess

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from test_client_cpu import A, B, C, D, E, F, ROOT, f, refused  # noqa: F401

G = 7 << 20


def test_structs_are_the_headers(f, tmp_path):  # noqa: F811
    structs = {"fasgd_route_args": f.RouteArgs, "fasgd_exchange_args": f.ExchangeArgs, "fasgd_multiply_args": f.MultiplyArgs,
               "fasgd_score_args": f.ScoreArgs}
    lines = []
    for name, cls in structs.items():
        lines += [f'printf("%zu ", offsetof({name}, {n}));' for n, _ in cls._fields_] + [f'printf("%zu\\n", sizeof({name}));']
    src = tmp_path / "o.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "fasgd.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.run(["gcc", "-std=c11", f"-I{ROOT}/include", str(src), "-o", str(tmp_path / "o")], check=True)
    out = subprocess.run([str(tmp_path / "o")], capture_output=True, text=True, check=True).stdout.split("\n")
    for line, cls in zip(out, structs.values()):
        assert [int(v) for v in line.split()] == [getattr(cls, n).offset for n, _ in cls._fields_] + [ctypes.sizeof(cls)], cls
    header = open(f"{ROOT}/include/fasgd.h").read()
    for name, value in (("CLASSES_MAX", f.CLASSES_MAX), ("SCORE_PIECE", f.SCORE_PIECE)):
        assert 1 << int(re.search(rf"FASGD_{name} \(\(int64_t\)1 << (\d+)\)", header).group(1)) == value


def test_route_refusals(f):  # noqa: F811
    good = f.RouteArgs(rows=100, top=2, experts=8, chosen=A, offsets=B, order=C, place=D, workspace=E, workspace_bytes=1 << 16)
    shape = [dict(rows=-1), dict(top=0), dict(top=-2), dict(experts=0), dict(experts=f.EXPERTS_MAX + 1), dict(rows=1 << 30), dict(rows=1 << 62),
             dict(top=1 << 62)]
    refused(f, f.fasgd_route, good, shape + [
        dict(chosen=None), dict(offsets=None), dict(order=None), dict(place=None), dict(chosen=A + 2), dict(offsets=B + 1), dict(order=C + 2),
        dict(place=D + 3), dict(workspace=None), dict(workspace=E + 8), dict(workspace_bytes=0), dict(order=A), dict(place=A + 796),
        dict(offsets=D), dict(workspace=C), dict(place=C + 4)])
    refused(f, f.fasgd_route_workspace, good, shape)
    assert f.fasgd_route(None, None) == f.EINVAL and f.fasgd_route_workspace(None) == -1


def test_exchange_refusals(f):  # noqa: F811
    good = f.ExchangeArgs(rows=100, top=2, cols=40, row_values=A, ld_rows=40, places=B, ld_places=40, order=C, place=C + 4096, weight=D,
                          dplaces=E, ld_dplaces=40, dweight=F, dtype=f.BF16)
    every = [dict(rows=-1), dict(top=0), dict(cols=0), dict(cols=f.COLS_MAX + 1), dict(dtype=5), dict(rows=1 << 30), dict(row_values=None),
             dict(row_values=A + 1), dict(places=None), dict(places=B + 1), dict(ld_rows=39), dict(ld_places=-40), dict(place=None),
             dict(place=C + 4097)]
    refused(f, f.fasgd_gather, good, every + [dict(order=None), dict(order=C + 2), dict(places=A + 100), dict(place=B), dict(order=B + 400)])
    refused(f, f.fasgd_combine, good, every + [dict(weight=D + 2), dict(row_values=B), dict(place=A), dict(weight=A + 4)])
    refused(f, f.fasgd_combine_grad, good, every + [
        dict(order=None), dict(weight=None), dict(dplaces=None), dict(dplaces=E + 1), dict(ld_dplaces=12), dict(dweight=F + 2), dict(dplaces=B),
        dict(dplaces=A + 40), dict(dweight=D), dict(dweight=E), dict(place=E), dict(order=F)])
    for call in (f.fasgd_gather, f.fasgd_combine, f.fasgd_combine_grad):
        assert call(None, None) == f.EINVAL


def test_multiply_refusals(f):  # noqa: F811
    good = f.MultiplyArgs(rows=100, inputs=40, outputs=24, experts=4, offsets=A, x=B, ld_x=40, w=C, ld_w=24, step_w=960, y=D, ld_y=24,
                          workspace=G, workspace_bytes=1 << 20, dtype=f.BF16, w_dtype=f.BF16)
    every = [dict(rows=-1), dict(rows=1 << 31), dict(inputs=0), dict(inputs=f.COLS_MAX + 1), dict(outputs=0), dict(outputs=f.COLS_MAX + 1),
             dict(experts=0), dict(experts=f.EXPERTS_MAX + 1), dict(dtype=4), dict(w_dtype=f.F16), dict(w_dtype=9), dict(w_flip=2),
             dict(dw_flip=-1), dict(offsets=None), dict(offsets=A + 2)]
    forward = every + [dict(x=None), dict(x=B + 1), dict(ld_x=39), dict(w=None), dict(w=C + 1), dict(ld_w=23), dict(step_w=959),
                       dict(step_w=0), dict(step_w=1 << 61), dict(y=None), dict(y=D + 1), dict(ld_y=3), dict(w_flip=1)]
    refused(f, f.fasgd_multiply, good, forward + [dict(y=B + 80), dict(y=C), dict(y=A), dict(y=G), dict(w_dtype=f.F32, workspace=None),
                                                  dict(w_dtype=f.F32, workspace=G + 16), dict(w_dtype=f.F32, workspace_bytes=64)])
    refused(f, f.fasgd_multiply_workspace, good, forward)
    grad = f.MultiplyArgs.from_buffer_copy(good)
    grad.y, grad.dy, grad.ld_dy, grad.dx, grad.ld_dx, grad.dw, grad.ld_dw, grad.step_dw = None, D, 24, E, 40, F, 24, 960
    bad = every + [dict(x=None), dict(w=None), dict(dy=None), dict(dy=D + 1), dict(ld_dy=23), dict(dx=E + 1), dict(ld_dx=39), dict(dw=F + 1),
                   dict(ld_dw=23), dict(step_dw=900), dict(dw_flip=1)]
    refused(f, f.fasgd_multiply_grad, grad, bad + [dict(dx=None, dw=None), dict(dx=D), dict(dw=C), dict(dw=E + 400), dict(dx=A), dict(dw=G)])
    refused(f, f.fasgd_multiply_workspace, grad, bad)
    assert f.fasgd_multiply(None, None) == f.EINVAL and f.fasgd_multiply_grad(None, None) == f.EINVAL
    assert f.fasgd_multiply_workspace(None) == -1


def test_score_refusals(f):  # noqa: F811
    good = f.ScoreArgs(rows=100, cols=40, classes=24, z=A, ld_z=40, w=B, ld_w=24, labels=C, loss=D, row_loss=D + 4096, lse=D + 8192, dz=E, ld_dz=40,
                       dw=F, ld_dw=24, workspace=G, workspace_bytes=1 << 22, dtype=f.F16)
    every = [dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=f.COLS_MAX + 1), dict(classes=0), dict(classes=f.CLASSES_MAX + 1),
             dict(dtype=3), dict(z=None), dict(z=A + 1), dict(ld_z=39), dict(w=None), dict(w=B + 1), dict(ld_w=23), dict(w_flip=1), dict(w_flip=2),
             dict(dw_flip=1), dict(labels=None), dict(labels=C + 4), dict(loss=None), dict(row_loss=None), dict(loss=D + 2),
             dict(row_loss=D + 4097), dict(lse=D + 8193), dict(upstream=D + 1), dict(dz=E + 1), dict(ld_dz=1), dict(dw=F + 1), dict(ld_dw=23),
             dict(known=2), dict(known=1, lse=None), dict(known=1, row_loss=None), dict(known=1, dz=None, dw=None)]
    refused(f, f.fasgd_score, good, every + [
        dict(workspace=None), dict(workspace=G + 128), dict(workspace_bytes=512), dict(dz=A), dict(dw=B + 48), dict(row_loss=C), dict(loss=D + 4096),
        dict(lse=D + 4000), dict(upstream=D), dict(workspace=F), dict(dw=E + 8)])
    refused(f, f.fasgd_score_workspace, good, every)
    assert f.fasgd_score(None, None) == f.EINVAL and f.fasgd_score_workspace(None) == -1


def test_the_workspace_of_a_score_is_bounded(f):  # noqa: F811
    for rows, classes, dtype in ((1 << 20, 1 << 20, f.BF16), (1 << 14, 1 << 18, f.F32), (100, 1 << 24, f.F16)):
        a = f.ScoreArgs(rows=rows, cols=64, classes=classes, z=A, ld_z=64, w=A, ld_w=classes, labels=A, loss=A, row_loss=A, dz=A, ld_dz=64, dw=A,
                        ld_dw=classes, dtype=dtype)
        size = f.fasgd_score_workspace(ctypes.addressof(a))
        # g, the copies of z and w, dz's sums, and the statistics of tiles of 64 classes.
        most = f.SCORE_PIECE + 64 * 4 * (rows + 8) + rows * (64 * 8 + 64) + (classes + 64) * 64 * 4 + classes / 64 * rows * 8 + (1 << 20)
        assert 0 < size <= most


@pytest.fixture(params=["module", "python"])
def client(request, monkeypatch, f):  # noqa: F811
    from paper_1601_04033_gb300 import client as c

    def reached(*_):
        raise AssertionError("the library was called")

    for name in f.SIGNATURES:
        if name.split("_")[1] in ("route", "gather", "combine", "multiply", "score"):
            monkeypatch.setattr(f, name, reached)
    if request.param == "module":
        if c._fast is None:
            pytest.skip("built without torch's headers")
    else:
        monkeypatch.setattr(c, "_fast", None)
    return c


def calls(c):
    """(the call, its tensors by name)."""
    def new(*size, dtype=torch.float32):
        return torch.empty(*size, dtype=dtype, device="cuda:0")

    def ints(*size):
        return new(*size, dtype=torch.int32)

    def way(v):
        return c.Route(ints(4), v["order"], v["place"])

    yield lambda v: c.route(v["chosen"], 3), dict(chosen=ints(6, 2))
    way_of = dict(order=ints(12), place=ints(6, 2))
    yield lambda v: c.gather(v["x"], way(v), out=v["out"]), dict(x=new(6, 8), out=new(12, 8), **way_of)
    yield lambda v: c.combine(v["y"], way(v), v["weight"], out=v["out"]), dict(y=new(12, 8), weight=new(6, 2), out=new(6, 8), **way_of)
    yield lambda v: c.combine_grad(v["y"], way(v), v["weight"], v["dout"], into=c.CombineGrads(v["dy"], v["dweight"])), \
        dict(y=new(12, 8), weight=new(6, 2), dout=new(6, 8), dy=new(12, 8), dweight=new(6, 2), **way_of)
    yield lambda v: c.multiply(v["x"], v["w"], v["offsets"], out=v["out"]), dict(x=new(12, 8), w=new(3, 8, 16), offsets=ints(4), out=new(12, 16))
    yield lambda v: c.multiply_grad(v["x"], v["w"], v["offsets"], v["dy"], into=c.MultiplyGrads(v["dx"], v["dw"])), \
        dict(x=new(12, 8), w=new(3, 8, 16), offsets=ints(4), dy=new(12, 16), dx=new(12, 8), dw=new(3, 8, 16))
    yield lambda v: c.score(v["z"], v["w"], v["labels"], upstream=v["upstream"], known=c.Score(None, v["rows"], None, None, v["lse"]),
                            into=(v["dz"], v["dw"])), \
        dict(z=new(6, 8), w=new(8, 16), labels=new(6, dtype=torch.int64), upstream=new(1), rows=new(6), lse=new(6), dz=new(6, 8), dw=new(8, 16))


@pytest.mark.parametrize("where", ["cuda:1", "cpu"])
def test_tensors_of_another_device_are_refused(client, where):
    if where == "cuda:1" and torch.cuda.device_count() == 1:
        pytest.skip("torch looks for the second GPU where there is one")
    with FakeTensorMode(allow_non_fake_inputs=True):
        tried = 0
        for call, tensors in calls(client):
            for moved in tensors if len(tensors) > 1 else ["chosen"] if where == "cpu" else []:
                v = {n: torch.empty_like(t, device=where) if n == moved else t for n, t in tensors.items()}
                with pytest.raises(ValueError, match="one device"):
                    call(v)
                tried += 1
    assert tried == (where == "cpu") + 4 + 5 + 7 + 4 + 6 + 8
