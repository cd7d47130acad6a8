"""build_client: a module of older sources is not left behind where a new one cannot be
built (it would fill argument structs of another layout), and one that is up to date
is kept."""

import os

import pytest

from paper_1601_04033_gb300 import build


@pytest.fixture
def module(tmp_path, monkeypatch):
    """A module's file, and sources that do not compile."""
    if build.torch_home() is None:
        pytest.skip("torch's headers are not installed")
    path, src = tmp_path / "_client.so", tmp_path / "client_torch.cpp"
    src.write_text("#error not this time\n")
    path.write_bytes(b"module")
    monkeypatch.setattr(build, "CLIENT", str(path))
    monkeypatch.setattr(build, "CLIENT_SRC", str(src))

    def age(seconds):                  # the module against the newest of what it is made of
        newest = max(os.path.getmtime(p) for p in (src, os.path.join(build.INCLUDE, "fasgd.h"),
                                                   os.path.join(build.torch_home(), "version.py")))
        os.utime(path, (newest - seconds, newest - seconds))
        return path

    return age


def test_an_old_module_goes_where_the_sources_do_not_compile(module):
    path = module(5)
    with pytest.warns(RuntimeWarning, match="was not built"):
        assert build.build_client() is None
    assert not path.exists()


def test_an_old_module_goes_where_headers_are_gone(module, monkeypatch):
    path = module(-5)
    monkeypatch.setattr(build, "torch_home", lambda: None)
    assert build.build_client() is None and path.exists()
    os.utime(path, (1, 1))
    assert build.build_client() is None and not path.exists()


def test_a_module_of_these_sources_is_kept(module):
    path = module(-5)
    assert build.build_client() == str(path) and path.read_bytes() == b"module"
    with pytest.warns(RuntimeWarning, match="was not built"):
        assert build.build_client(force=True) is None
    assert not path.exists()
