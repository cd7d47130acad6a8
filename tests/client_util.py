"""The client operators restated in 64 bits (torch on the CPU or GPU, gradients
by differentiating the definition), and the bounds their kernels are held to."""

from __future__ import annotations

import numpy as np
import torch

U32 = 2.0 ** -24                                       # unit roundoff of fp32
UNIT = {torch.float32: U32, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -24}   # subnormal spacing


def philox_words(c0, c1, c2, c3, seed):
    """Philox4x32-10 on arrays of counters (uint64 numpy arithmetic)."""
    m = np.uint64(0xFFFFFFFF)
    c = [np.broadcast_to(np.asarray(v, np.uint64) & m, np.shape(c0)).copy() for v in (c0, c1, c2, c3)]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    with np.errstate(over="ignore"):
        for _ in range(10):
            a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
            c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & m,
                 (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & m]
            k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def factors(index, rate, seed, client, n):
    """What elements of these indices are multiplied by (fp64, 0: dropped)."""
    index = np.asarray(index, np.uint64)
    q = index >> np.uint64(3)
    words = philox_words(q & np.uint64(0xFFFFFFFF), client + 3 * 2 ** 30, n & 0xFFFFFFFF,
                         np.uint64(n >> 32) + ((q >> np.uint64(32)) << np.uint64(16)), seed)
    i = (index & np.uint64(7)).astype(np.int64)
    word = np.choose(i >> 1, words)
    half = np.where(i & 1, word >> np.uint64(16), word & np.uint64(0xFFFF))
    cut = int(np.floor(rate * 65536 + 0.5))
    return np.where(half >= cut, 65536.0 / max(1, 65536 - cut), 0.0)


def norm64(t, w, b, layer, eps):
    mean = t.mean(-1, keepdim=True) if layer else 0.0
    out = (t - mean) / torch.sqrt(((t - mean) ** 2).mean(-1, keepdim=True) + eps) * w
    return out if b is None else out + b


class Join64:
    """fasgd_join in 64 bits on [rows, cols] tensors, with its gradients, and for
    every result the size of the terms that it is made of (the bounds' scale)."""

    def __init__(self, x, y, post, post_bias, gate, pre, pre_bias, layer, eps, carry, branch, draws, dh, dz):
        R, D = x.shape
        given = dict(x=x, y=y, post=post, post_bias=post_bias, gate=gate, pre=pre, pre_bias=pre_bias)
        v = {k: t.double().requires_grad_(True) for k, t in given.items() if t is not None}
        g = v.get
        m = torch.ones((), dtype=torch.float64, device=x.device)
        if draws is not None and draws[0]:
            m = torch.from_numpy(factors(np.arange(R * D), *draws).reshape(R, D)).to(x.device)
        G = 1 if gate is None or gate.dim() == 1 else gate.shape[0]
        gates = 1.0 if gate is None else \
            g("gate").reshape(G, 1, D).expand(G, R // G, D).reshape(R, D)
        u = None
        if y is not None:
            t = g("y") if post is None else norm64(g("y"), g("post"), g("post_bias"), layer, eps)
            u = torch.where(m > 0, t, 0.0) * m
            h = carry * g("x") + branch * gates * u
        else:
            h = g("x")
        z = None if pre is None else norm64(h, g("pre"), g("pre_bias"), layer, eps)
        self.h, self.z = h.detach(), None if z is None else z.detach()
        if dh is None and dz is None:
            return
        ends = [(e, d.double()) for e, d in ((h, dh), (z, dz)) if e is not None and d is not None]
        names = list(v)
        got = torch.autograd.grad([e for e, _ in ends], [v[k] for k in names], [d for _, d in ends],
                                  allow_unused=True)
        self.grads = {k: torch.zeros_like(v[k]) if t is None else t for k, t in zip(names, got)}

        # Sizes of the terms of the sums over rows.
        with torch.no_grad():
            d = self.grads["x"] / carry if y is not None else self.grads["x"]
            terms = {}

            def hat(t):
                mean = t.mean(1, keepdim=True) if layer else 0.0
                return (t - mean) / torch.sqrt(((t - mean) ** 2).mean(1, keepdim=True) + eps)

            self.row = d.abs().amax(1, keepdim=True) + \
                (dh.double().abs().amax(1, keepdim=True) if dh is not None else 0.0)
            if pre is not None:
                rstd = 1 / torch.sqrt(((h - (h.mean(1, keepdim=True) if layer else 0)) ** 2).mean(1, keepdim=True) + eps)
                qm = (dz.double() * pre.double()).abs().amax(1, keepdim=True)
                hm = hat(h).abs().amax(1, keepdim=True)
                self.row = self.row + rstd * qm * (1 + hm * hm)
                terms["pre"] = (dz.double().abs() * hm).sum(0)
                terms["pre_bias"] = dz.double().abs().sum(0)
            if y is not None:
                gm = gates.abs() if gate is not None else 1.0
                dt = (self.row * gm * m * abs(branch)).expand(R, D)
                if gate is not None:
                    # t's size, not its value: a norm's output is as exact as its row's largest terms.
                    tm = u.abs().amax(1, keepdim=True)
                    terms["gate"] = (abs(branch) * self.row * tm * (m > 0)).expand(R, D).reshape(G, R // G, D).sum(1)
                    if gate.dim() == 1:
                        terms["gate"] = terms["gate"][0]
                self.row_y = dt.abs().amax(1, keepdim=True)
                if post is not None:
                    ym = hat(g("y")).abs().amax(1, keepdim=True)
                    yr = 1 / torch.sqrt(((g("y") - (g("y").mean(1, keepdim=True) if layer else 0)) ** 2)
                                        .mean(1, keepdim=True) + eps)
                    terms["post"] = (dt * ym).sum(0)
                    terms["post_bias"] = dt.sum(0)
                    self.row_y = self.row_y * yr * post.double().abs().max() * (1 + ym * ym)
            self.terms = terms


def hold(got, want, scale, what, rows=0):
    """|got - want| <= the rounding of got's type + C 2^-24 scale, where scale is the
    size of the terms that meet in one value.  C counts the fp32 roundings that
    can pile up: 64 covers a row's statistic (tree sums of at most 13 levels, 32
    terms in a thread before that), the arithmetic before and after it; a sum
    over rows adds one for each row of a thread's chain, which is no longer than
    a hundredth of the rows (every part takes every 304th or so)."""
    got64 = got.double()
    over = want.to(got.dtype).isinf() & torch.isfinite(want)     # beyond the type: rounds to infinity
    got64, want = torch.where(over, got64.sign() * over, got64), torch.where(over, want.sign(), want)
    assert bool(torch.isinf(got[over]).all()), what
    C = 64 + rows / 100
    unit = UNIT[got.dtype]
    bound = unit * want.abs() * (1 + 2.0 ** -8) + C * U32 * scale + TINY[got.dtype]
    off = (got64 - want).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        i = int(torch.argmax(torch.where(bad, off / bound, torch.zeros_like(off)).reshape(-1)))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds; at {i}: "
                             f"{got64.reshape(-1)[i].item()!r} against {want.reshape(-1)[i].item()!r}, "
                             f"off {off.reshape(-1)[i].item():.3e}, bound {bound.expand_as(off).reshape(-1)[i].item():.3e}")
