"""The routed network on the client operators: its gradient against the same network
out of elementary operations in 64 bits, training that learns, and runs that repeat
bit for bit."""

import numpy as np
import pytest

from client_util import factors, norm64

pytestmark = pytest.mark.gpu


def forward64(net, theta, x, labels, draws):
    """RoutedNetwork.forward's loss in 64 bits."""
    import torch
    p = {k: t.view(s) for (k, s), t in zip(net.shapes.items(), torch.split(theta, net.sizes))}

    def mask(place, shape):
        n = draws[1] * (net.blocks + 1) + place
        m = factors(np.arange(shape[0] * shape[1]), net.rate, net.seed, draws[0], n)
        return torch.from_numpy(m.reshape(shape)).cuda()

    h = x.double() @ p["in"]
    z = norm64(h, p["pre0"], None, net.norm == "layer", 1e-6)
    total = 0.0
    for b in range(net.blocks):
        s = z @ p[f"router{b}"]
        chosen = torch.topk(s.detach(), net.top, dim=1).indices
        sent = torch.nn.functional.one_hot(chosen, net.experts).sum(1).double()
        f = sent.sum(0) / (net.top * s.shape[0])
        total = total + 0.01 * net.experts * (f * torch.softmax(s, 1).mean(0)).sum() + \
            0.001 * torch.logsumexp(s, 1).square().mean()
        w = torch.softmax(s.masked_fill(sent == 0, float("-inf")), 1)
        y = torch.einsum("erh,ehd,re->rd", torch.relu(torch.einsum("rd,edh->erh", z, p[f"up{b}"])), p[f"down{b}"], w)
        u = norm64(y, p[f"post{b}"], None, net.norm == "layer", 1e-6) * mask(b, y.shape)
        h = h + p[f"gate{b}"] * u
        z = norm64(h, p[f"pre{b + 1}"], None, net.norm == "layer", 1e-6)
    z = z * mask(net.blocks, z.shape)
    return torch.nn.functional.cross_entropy(z @ p["out"], labels) + total


@pytest.mark.parametrize("norm, width", [("rms", 96), ("layer", 101)])
def test_gradient_in_fp32(norm, width):
    """fp32 throughout: 2^-24 for each of the some hundred roundings between the
    loss and a weight, of the gradient's norm; a thousandfold would show at 1e-4."""
    import torch
    from paper_1601_04033_gb300 import network
    torch.backends.cuda.matmul.allow_tf32 = False
    net = network.RoutedNetwork(width=width, norm=norm, dtype=torch.float32)
    theta = net.theta0()
    x, labels = network.Classes(64, 10).batch(128, 3, 5)
    loss, grad = net.gradient(theta, x, labels, (3, 5))
    leaf = theta.double().requires_grad_(True)
    want = forward64(net, leaf, x, labels, (3, 5))
    want.backward()
    want = float(want.detach())
    assert abs(float(loss) - want) < 1e-5 * abs(want)
    off = (grad.double() - leaf.grad).norm() / leaf.grad.norm()
    assert off < 1e-4, float(off)


def test_training_learns_and_repeats():
    import torch
    from paper_1601_04033_gb300 import network

    def run(norm):
        return network.train(network.RoutedNetwork(norm=norm), batches=120, log_every=60)

    for norm in ("rms", "layer"):
        losses, theta = run(norm)
        assert losses[-1] < 0.6 * losses[0], losses
    again, theta2 = run("layer")
    assert again == losses and torch.equal(theta, theta2)
