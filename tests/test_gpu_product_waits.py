"""The bounded waits inside the products on the tensor cores."""

import pytest

from test_gpu_client import _c

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture
def limit():
    """Sets the time without a copy after which waits give up."""
    from paper_1601_04033_gb300 import fasgd

    def set_limit(ns):
        assert fasgd.fasgd_selftest_product_limit(ns) == 0

    yield set_limit
    set_limit(1_000_000_000)


@pytest.mark.parametrize("rows, width, dtype", [(1 << 16, 4096, torch.float32), (1 << 17, 8192, torch.bfloat16)])
def test_a_groups_last_rows_may_come_late(limit, rows, width, dtype):
    """Groups of whole copies (multiples of 64 rows), which keep the tensor cores for ten milliseconds, before
    one whose last copy is cut: the wait for that begins with the launch.  Copies go on all the while, so that
    it lasts longer than a limit of one millisecond."""
    c = _c()
    limit(1_000_000)
    g = torch.Generator(device="cuda").manual_seed(1)
    n = rows + 67
    x, dy = (torch.randn(n, width, generator=g, device="cuda", dtype=dtype) for _ in range(2))
    offsets = torch.tensor([0, rows, n], dtype=torch.int32, device="cuda")
    w = torch.empty(2, width, width, dtype=dtype, device="cuda")
    before, after = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    before.record()
    dw = c.multiply_grad(x, w, offsets, dy, grads=(False, True)).w
    after.record()
    assert dw.isfinite().all()
    assert before.elapsed_time(after) > 5.0
    cols = slice(width // 2, width // 2 + 32)
    for e, (a, b) in enumerate(((0, rows), (rows, n))):
        want = x[a:b, cols].double().t() @ dy[a:b].double()
        size = x[a:b, cols].double().abs().t() @ dy[a:b].double().abs()
        # (a sum of b - a products in fp32, as elsewhere; roundings to 16 bits)
        u = torch.finfo(dtype).eps / 2
        assert bool(((dw[e, cols].double() - want).abs() <= (b - a) * 2.0 ** -23 * size * 33 / 32 + u * want.abs() * (1 + 2.0 ** -8)).all())


def test_a_wait_that_runs_out_is_reported(limit):
    """Failure detection without a fault: a kernel whose barrier nobody arrives at gives up after the limit
    and returns; the next sync says so, once, and products are as before."""
    from paper_1601_04033_gb300 import fasgd
    c = _c()
    g = torch.Generator(device="cuda").manual_seed(2)
    x, w = torch.randn(300, 64, generator=g, device="cuda").bfloat16(), torch.randn(1, 64, 40, generator=g, device="cuda").bfloat16()
    offsets = torch.tensor([0, 300], dtype=torch.int32, device="cuda")
    y = c.multiply(x, w, offsets)
    c.sync()
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            assert fasgd.fasgd_selftest_product_wait(5_000_000, stream.cuda_stream) == 0
            with pytest.raises(fasgd.FasgdError, match="ran out") as e:
                c.sync()
            assert e.value.code == fasgd.EDEVICE
            c.sync()
            assert torch.equal(c.multiply(x, w, offsets), y)
            c.sync()


def test_sync_is_refused_in_a_capture():
    from paper_1601_04033_gb300 import fasgd
    c = _c()
    graph = torch.cuda.CUDAGraph()
    t = torch.zeros(4, device="cuda")
    with torch.cuda.graph(graph):
        t.add_(1.0)
        with pytest.raises(fasgd.FasgdError, match="captured"):
            c.sync()
    graph.replay()
    assert t.sum() == 4.0
    c.sync()
