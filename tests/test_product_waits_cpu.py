"""The products' test hook on a machine without a GPU."""

from test_client_cpu import f  # noqa: F401


def test_limits_of_waits(f):  # noqa: F811
    for ns in (0, -1, 1, 999_999, 1_000_000_001, 1 << 62):
        assert f.fasgd_selftest_product_limit(ns) == f.EINVAL and "10^6" in f.fasgd_last_error(None)
        assert f.fasgd_selftest_product_wait(ns, None) == f.EINVAL
    for ns in (1_000_000, 1_000_000_000):
        assert f.fasgd_selftest_product_limit(ns) == 0


def test_sync_without_a_place_for_its_answer(f):  # noqa: F811
    assert f.fasgd_client_sync(None, None) == f.EINVAL and "NULL" in f.fasgd_last_error(None)
