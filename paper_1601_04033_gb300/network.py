"""Asynchronous training of a routed residual network: clients that compute real
gradients in place of sim.py's quadratic, against the same server.

lambda clients hold copies of the flat parameter vector.  A dispatched client runs
one minibatch through the network on its (stale) copy -- residual blocks of routed
experts, with the client operators (``client.joined``, ``client.balanced``,
``client.dropped``) between the matrix products, which are torch's, or (``sparse``) with
rows that go to their experts alone (``client.route``, ``gathered``, ``multiplied``,
``combined``) and the loss from the rows before the last product (``scored``) -- and pushes
the gradient of the whole vector; the server applies the batch and the client
fetches fresh parameters (the protocol of the paper's Sec. 2.1 and 3).  Draws of
dropout are keyed by (seed, client, the client's count of gradients and the place
in the network), so a run can be repeated bit for bit.

``python -m paper_1601_04033_gb300.network`` trains on synthetic classes and
prints the losses.
"""

from __future__ import annotations

import argparse
import json

import torch

from . import client, fasgd, streams


class RoutedNetwork:
    """blocks x [norm, top-k routed experts, join], a last norm, dropout, classes.
    The parameters are views of one fp32 vector, in the order of `shapes`; each is
    a tensor of its own to the server's per-tensor rules (`sizes`).  sparse: every row
    goes through its own experts only, as fp32 parameters rounded to dtype, not through
    every expert with a weight."""

    def __init__(self, inputs=64, width=96, hidden=64, classes=10, blocks=3, experts=4, top=2, norm="rms",
                 rate=0.1, dtype=torch.bfloat16, seed=0, sparse=False):
        self.width, self.classes, self.blocks, self.experts, self.top = width, classes, blocks, experts, top
        self.norm, self.rate, self.dtype, self.seed, self.sparse = norm, rate, dtype, seed, sparse
        self.shapes = {"in": (inputs, width), "pre0": (width,)}
        for b in range(blocks):
            self.shapes.update({f"router{b}": (width, experts), f"up{b}": (experts, width, hidden),
                                f"down{b}": (experts, hidden, width), f"post{b}": (width,), f"gate{b}": (width,),
                                f"pre{b + 1}": (width,)})
        self.shapes["out"] = (width, classes)
        self.sizes = [torch.Size(s).numel() for s in self.shapes.values()]
        self.P = sum(self.sizes)

    def theta0(self):
        g = torch.Generator(device="cuda").manual_seed(self.seed)
        parts = []
        for name, shape in self.shapes.items():
            if name.startswith(("pre", "post")):
                parts.append(torch.ones(shape, device="cuda"))
            elif name.startswith("gate"):
                parts.append(torch.full(shape, 0.5, device="cuda"))
            else:
                parts.append(torch.randn(shape, generator=g, device="cuda") * shape[-2] ** -0.5)
        return torch.cat([p.reshape(-1) for p in parts])

    def forward(self, theta, x, draws=None):
        """Class scores, the sum of the blocks' balance losses, and each block's
        per-expert counts.  draws: (client, n) of a training pass; None: nothing
        is dropped."""
        z, out, balance, counts = self._rows(theta, x, draws)
        return z @ out, balance, counts

    def _rows(self, theta, x, draws):
        """forward's rows before the last product, fp32, and its matrix."""
        p = {k: t.view(s) for (k, s), t in zip(self.shapes.items(), torch.split(theta, self.sizes))}
        cast = self.dtype

        def at(place):
            return None if draws is None else \
                client.Draws(self.rate, self.seed, draws[0], draws[1] * (self.blocks + 1) + place)

        h = x.to(cast) @ p["in"].to(cast)
        _, z = client.joined(h, pre=p["pre0"], norm=self.norm)
        balance, counts = 0.0, []
        for b in range(self.blocks):
            scores = z.float() @ p[f"router{b}"]
            chosen = torch.topk(scores.detach(), self.top, dim=1).indices.to(torch.int32)
            loss, _, count = client.balanced(scores, chosen, balance=0.01, z=0.001)
            balance = balance + loss
            counts.append(count)
            open_ = (chosen[:, :, None] == torch.arange(self.experts, device="cuda")).any(1)
            weight = torch.softmax(scores.masked_fill(~open_, float("-inf")), 1).to(cast)
            if self.sparse:
                way = client.route(chosen, self.experts)
                u = torch.relu(client.multiplied(client.gathered(z, way), p[f"up{b}"], way.offsets))
                y = client.combined(client.multiplied(u, p[f"down{b}"], way.offsets), way,
                                    weight.float().gather(1, chosen.long()))
            else:
                # Every expert on every row, weighted: an example's way to route.
                u = torch.relu(torch.einsum("rd,edh->erh", z, p[f"up{b}"].to(cast)))
                y = torch.einsum("erh,ehd,re->rd", u, p[f"down{b}"].to(cast), weight)
            h, z = client.joined(h, y, post=p[f"post{b}"], gate=p[f"gate{b}"], pre=p[f"pre{b + 1}"], norm=self.norm,
                                 draws=at(b))
        if draws is not None:
            z = client.dropped(z, at(self.blocks))
        return z.float(), p["out"], balance, counts

    def gradient(self, theta, x, labels, draws):
        """(loss, its gradient as one vector) of a minibatch at theta."""
        leaf = theta.detach().requires_grad_(True)
        z, out, balance, _ = self._rows(leaf, x, draws)
        loss = client.scored(z, out, labels)[0] if self.sparse else torch.nn.functional.cross_entropy(z @ out, labels)
        loss = loss + balance
        loss.backward()
        return loss.detach(), leaf.grad


class Classes:
    """Minibatches of synthetic classes: a mean each, and noise as large."""

    def __init__(self, inputs, classes, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.means = torch.randn(classes, inputs, generator=g, device="cuda")
        self.seed = seed

    def batch(self, rows, client_, n):
        g = torch.Generator(device="cuda").manual_seed(self.seed * 1_000_003 + client_ * 65_537 + n + 1)
        labels = torch.randint(0, self.means.shape[0], (rows,), generator=g, device="cuda")
        return self.means[labels] + torch.randn(rows, self.means.shape[1], generator=g, device="cuda"), labels


def train(net: RoutedNetwork, *, lam=8, batches=200, K=2, alpha=2.0, variant=fasgd.FASGD, rows=128, inputs=64,
          exact=True, log_every=50):
    """Train `net` with lambda clients for `batches` dispatcher batches of K; the
    loss on a held-out minibatch (nothing dropped) before, during and after, and
    the server's parameters."""
    data = Classes(inputs, net.classes, net.seed)
    srv = fasgd.Server(net.P, lam, alpha, variant, seed=net.seed)
    srv.set_tensors(net.sizes)
    srv.set_exact(exact)
    theta = net.theta0()
    srv.set_params(theta)
    _copies, copies = fasgd.aligned_vectors(theta.repeat(lam, 1))
    _grads, grads = fasgd.aligned_vectors(torch.zeros(K, net.P))
    stamp, count = [0] * lam, [0] * lam
    held = data.batch(1024, lam, 0)

    def held_out():
        srv.pull(theta)
        with torch.no_grad():
            scores, balance, _ = net.forward(theta, held[0])
            loss = float(torch.nn.functional.cross_entropy(scores, held[1]) + balance)
        client.sync()       # no gradient since the last time is NaN for a wait that ran out
        return loss

    losses = [held_out()]
    for b, batch in enumerate(streams.dispatch_schedule(net.seed, lam, batches, K)):
        for k, c in enumerate(int(c) for c in batch):
            _, g = net.gradient(copies[c], *data.batch(rows, c, count[c]), (c, count[c]))
            grads[k].copy_(g)
            srv.push(c, stamp[c], grads[k])
            count[c] += 1
        srv.apply_pending(K)
        for c in (int(c) for c in batch):
            stamp[c] = srv.pull(copies[c])
        if (b + 1) % log_every == 0:
            losses.append(held_out())
    srv.pull(theta)
    srv.sync()
    srv.close()
    return losses, theta


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batches", type=int, default=400)
    ap.add_argument("--lam", type=int, default=8)
    ap.add_argument("--K", type=int, default=2)
    ap.add_argument("--norm", choices=["rms", "layer"], default="rms")
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--sparse", action="store_true", help="rows go to their own experts only")
    args = ap.parse_args()
    out = {}
    # Gradients' spreads are near 1e-3 here, so v nears its largest, eps^-1/2 = 100, and
    # FASGD's alpha / v is a fiftieth.
    for name, variant, alpha in (("sasgd", fasgd.SASGD, 0.04), ("fasgd", fasgd.FASGD, 2.0)):
        net = RoutedNetwork(norm=args.norm, seed=args.seed, sparse=args.sparse)
        losses, _ = train(net, lam=args.lam, batches=args.batches, K=args.K, alpha=alpha, variant=variant)
        out[name] = {"alpha": alpha, "held_out_losses": losses}
    print(json.dumps({"parameters": net.P, "lambda": args.lam, "batches": args.batches, "K": args.K, **out}))


if __name__ == "__main__":
    main()
