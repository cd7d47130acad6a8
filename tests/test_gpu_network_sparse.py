"""The routed network with rows that go to their own experts only and the loss from the rows
before the last product: its gradient against the network in 64 bits, and runs that
repeat bit for bit."""

import pytest

from test_gpu_network import forward64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm, width, rows", [("rms", 96, 128), ("layer", 101, 37)])
def test_gradient_in_fp32(norm, width, rows):
    """The bounds of the network that runs every expert on every row: 2^-24 for each of some hundred
    roundings, and a thousandfold that would show at 1e-4."""
    import torch
    from paper_1601_04033_gb300 import network
    torch.backends.cuda.matmul.allow_tf32 = False
    net = network.RoutedNetwork(width=width, norm=norm, dtype=torch.float32, sparse=True)
    theta = net.theta0()
    x, labels = network.Classes(64, 10).batch(rows, 3, 5)
    loss, grad = net.gradient(theta, x, labels, (3, 5))
    leaf = theta.double().requires_grad_(True)
    want = forward64(net, leaf, x, labels, (3, 5))
    want.backward()
    assert abs(float(loss) - float(want.detach())) < 1e-5 * abs(float(want.detach()))
    off = (grad.double() - leaf.grad).norm() / leaf.grad.norm()
    assert off < 1e-4, float(off)


def test_training_runs_and_repeats():
    import torch
    from paper_1601_04033_gb300 import network
    losses, theta = network.train(network.RoutedNetwork(sparse=True), batches=20, log_every=10)
    again, theta2 = network.train(network.RoutedNetwork(sparse=True), batches=20, log_every=10)
    assert again == losses and torch.equal(theta, theta2) and torch.isfinite(theta).all()
