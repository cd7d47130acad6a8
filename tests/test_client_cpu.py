"""The client operators on a machine without a GPU: the binding's structs are the
header's, and bad arguments are rejected on the host before the device is
touched."""

import ctypes
import os
import re
import subprocess

import pytest

from paper_1601_04033_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, B, C, D, E, F = (1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20, 6 << 20)   # addresses, never followed


@pytest.fixture(scope="module")
def f():
    build.build()
    from paper_1601_04033_gb300 import fasgd
    return fasgd


def test_structs_are_the_headers(f, tmp_path):
    lines = []
    for name, cls in (("fasgd_dropout_args", f.DropoutArgs), ("fasgd_join_args", f.JoinArgs),
                      ("fasgd_balance_args", f.BalanceArgs)):
        fields = [n for n, _ in cls._fields_]
        lines += [f'printf("%zu ", offsetof({name}, {n}));' for n in fields] + [f'printf("%zu\\n", sizeof({name}));']
    src = tmp_path / "o.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "fasgd.h"\nint main(void) {\n'
                   + "\n".join(lines) + "\nreturn 0; }\n")
    exe = tmp_path / "o"
    subprocess.run(["gcc", "-std=c11", f"-I{ROOT}/include", str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split("\n")
    for line, cls in zip(out, (f.DropoutArgs, f.JoinArgs, f.BalanceArgs)):
        want = [getattr(cls, n).offset for n, _ in cls._fields_] + [ctypes.sizeof(cls)]
        assert [int(v) for v in line.split()] == want, cls
    header = open(os.path.join(ROOT, "include", "fasgd.h")).read()
    for name in ("FASGD_F32 = 0", "FASGD_BF16 = 1", "FASGD_F16 = 2", "FASGD_RMS_NORM = 0", "FASGD_LAYER_NORM = 1"):
        assert name in header
    assert int(re.search(r"FASGD_EXPERTS_MAX (\d+)", header).group(1)) == f.EXPERTS_MAX and f.COLS_MAX == 1 << 20


def refused(f, call, good, changes, allowed=()):
    cls = type(good)
    for change in changes:
        a = cls.from_buffer_copy(good)
        for k, v in change.items():
            setattr(a, k, v)
        at = ctypes.addressof(a)
        rc = call(at, None) if call.__name__.find("workspace") < 0 else call(at)
        assert rc == (f.EINVAL if call.__name__.find("workspace") < 0 else -1), change
        assert f.fasgd_last_error(None).startswith(call.__name__), (change, f.fasgd_last_error(None))


def test_dropout_refusals(f):
    good = f.DropoutArgs(rows=10, cols=40, x=A, ld_x=40, out=B, ld_out=40, rate=0.5, dtype=f.BF16)
    refused(f, f.fasgd_dropout, good, [
        dict(rows=-1), dict(rows=(1 << 40) + 1), dict(cols=0), dict(cols=-4), dict(cols=(1 << 40) + 1), dict(dtype=3),
        dict(dtype=-1), dict(x=None), dict(x=A + 1), dict(out=None), dict(out=B + 1), dict(ld_x=39), dict(ld_out=0),
        dict(ld_x=-40), dict(ld_x=1 << 62), dict(residual=C, ld_residual=39), dict(residual=C + 1, ld_residual=40),
        dict(rate=-0.1), dict(rate=1.01), dict(rate=float("nan")), dict(client=-1), dict(client=1 << 30),
        dict(n=1 << 48), dict(rows=1 << 30, cols=1 << 21, ld_x=1 << 21, ld_out=1 << 21),
        dict(out=A + 2), dict(out=A - 78), dict(out=A, ld_out=48), dict(residual=B + 8, ld_residual=40),
        dict(dtype=f.F32, x=A + 2)])
    assert f.fasgd_dropout(None, None) == f.EINVAL


def join_args(f, **more):
    return f.JoinArgs(rows=10, cols=40, groups=1, x=A, ld_x=40, y=B, ld_y=40, h=C, ld_h=40, z=D, ld_z=40,
                      post=E, pre=E + 4096, gate=E + 8192, stats=F, eps=1e-6, carry=1.0, branch=1.0, dtype=f.BF16,
                      **more)


def test_join_refusals(f):
    refused(f, f.fasgd_join, join_args(f), [
        dict(rows=-1), dict(cols=0), dict(cols=f.COLS_MAX + 1, ld_x=f.COLS_MAX + 1), dict(groups=0), dict(groups=3), dict(groups=-1),
        dict(dtype=7), dict(norm=2), dict(norm=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
        dict(eps=float("inf")), dict(carry=float("nan")), dict(branch=float("inf")), dict(x=None), dict(x=A + 1),
        dict(ld_x=39), dict(y=None), dict(y=None, post=None, gate=None), dict(h=None), dict(z=None), dict(pre=None),
        dict(pre=None, z=None, pre_bias=E), dict(post=None, post_bias=E), dict(post=E + 2), dict(pre=E + 1),
        dict(gate=E + 2), dict(gate_dtype=f.F16), dict(stats=F + 8), dict(rate=2.0), dict(rate=float("nan")),
        dict(client=-2), dict(n=1 << 50), dict(h=A), dict(h=B + 4), dict(z=C), dict(z=E + 4096 - 8), dict(h=F),
        dict(y=None, h=None, post=None, gate=None, pre=None, z=None),
        dict(rows=1 << 40, cols=1 << 20, ld_x=1 << 20, ld_y=1 << 20, ld_h=1 << 20, ld_z=1 << 20)])
    assert f.fasgd_join(None, None) == f.EINVAL


def test_join_grad_refusals(f):
    good = join_args(f, dh=A + (1 << 16), ld_dh=40, dz=B + (1 << 16), ld_dz=40, dx=C, ld_dx=40, dy=D, ld_dy=40,
                     dpost=F + 4096, dgate=F + 8192, dpre=F + 12288, workspace=F + (1 << 16), workspace_bytes=1 << 19)
    bad = [dict(stats=None), dict(dz=None), dict(dy=None), dict(dx=None), dict(dx=C + 1), dict(ld_dh=3), dict(ld_dz=39),
           dict(ld_dx=39), dict(ld_dy=-1), dict(dpost=F + 4098), dict(dgate=F + 8194), dict(pre=None),
           dict(pre=None, dz=None), dict(post=None), dict(gate=None), dict(y=None), dict(groups=4), dict(rate=-1.0)]
    refused(f, f.fasgd_join_grad, good, bad + [
        dict(dx=A), dict(dy=A + (1 << 16)), dict(dx=D), dict(dpost=E), dict(dpre=F + 4096), dict(dgate=F),
        dict(workspace=A)])
    refused(f, f.fasgd_join_workspace, good, bad)
    assert f.fasgd_join_grad(None, None) == f.EINVAL and f.fasgd_join_workspace(None) == -1


def test_balance_refusals(f):
    good = f.BalanceArgs(rows=12, cols=40, groups=2, top=2, logits=A, ld_logits=40, chosen=B, dlogits=C, ld_dlogits=40,
                         counts=D, loss=E, workspace=F, workspace_bytes=1 << 20, balance_scale=1.0, dtype=f.BF16)
    shape = [dict(rows=-1), dict(cols=0), dict(cols=f.EXPERTS_MAX + 1), dict(groups=0), dict(groups=5), dict(top=0),
             dict(top=1 << 31), dict(rows=1 << 30, top=2), dict(dtype=9)]
    refused(f, f.fasgd_balance, good, shape + [
        dict(logits=None), dict(logits=A + 1), dict(ld_logits=39), dict(ld_dlogits=39), dict(dlogits=C + 1),
        dict(chosen=None), dict(chosen=B + 2), dict(counts=None), dict(counts=D + 1), dict(loss=E + 2),
        dict(upstream=E + 1), dict(workspace=None), dict(workspace=F + 8), dict(workspace_bytes=16),
        dict(balance_scale=float("nan")), dict(z_scale=float("inf")), dict(dlogits=A), dict(counts=B), dict(loss=D),
        dict(counts=F), dict(upstream=E + 8), dict(valid=C)])
    refused(f, f.fasgd_balance_workspace, good, shape)
    assert f.fasgd_balance(None, None) == f.EINVAL and f.fasgd_balance_workspace(None) == -1
    assert 0 < f.fasgd_balance_workspace(ctypes.addressof(good)) < 1 << 20
