"""A join of no rows may have any number of gates; one whose gates' bytes would not fit
64 bits is refused before the device is touched."""

import ctypes

import pytest

from paper_1601_04033_gb300 import build

A, B, C, D, E, F = (1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20, 6 << 20)   # addresses, never followed


@pytest.mark.parametrize("groups", [(1 << 40) + 1, 1 << 60, 1 << 61, (1 << 63) - 1])
def test_more_gates_than_rows_can_be(groups):
    build.build()
    from paper_1601_04033_gb300 import fasgd as f
    a = f.JoinArgs(rows=0, cols=40, groups=groups, x=A, ld_x=40, y=B, ld_y=40, h=C, ld_h=40, gate=E, dx=C, ld_dx=40,
                   dy=D, ld_dy=40, dgate=F, stats=F + 4096, workspace=A, workspace_bytes=64, eps=1e-6, dtype=f.BF16)
    at = ctypes.addressof(a)
    for name, call, want in (("join", lambda: f.fasgd_join(at, None), f.EINVAL),
                             ("grad", lambda: f.fasgd_join_grad(at, None), f.EINVAL),
                             ("workspace", lambda: f.fasgd_join_workspace(at), -1)):
        assert call() == want and "groups" in f.fasgd_last_error(None), name
