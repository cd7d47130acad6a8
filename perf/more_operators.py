"""What is measured of a client's routed experts and of the loss at its network's end,
in four kinds of case:

* ``route``     a router's choices into the experts' order: places, order, offsets.
* ``exchange``  rows to their experts and back: the gather, the weighted combination,
                and (``train``) the gradients of both.
* ``multiply``  the experts' products on rows in their order, ragged sizes;
                ``train``: also the gradients of rows and weights.
* ``score``     softmax cross entropy of rows against a matrix of classes, from the
                rows before that matrix; ``train``: also the gradients of both.

Sizes are those of this package's networks (minibatches of 128; 784-200-10; the
routed network's 96, 64, 10 and 4 experts, 2 of them for a row) and generic ones:
powers of two, and odd and ragged sizes between them.
"""

from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _route(T, top, E):
    return {"kind": "route", "T": T, "top": top, "E": E}


def _exchange(T, top, E, D, dtype="bf16", train=True, pad=0):
    return {"kind": "exchange", "T": T, "top": top, "E": E, "D": D, "dtype": dtype, "train": train, "pad": pad}


def _multiply(T, top, E, K, N, dtype="bf16", weights="same", train=True, flip=False, pad=0):
    """weights: "same" type as the rows, or "f32" (parameters, which take part rounded to
    the rows' type and have fp32 gradients); flip: a weight's inputs are consecutive in
    memory, not its outputs."""
    return {"kind": "multiply", "T": T, "top": top, "E": E, "K": K, "N": N, "dtype": dtype, "weights": weights,
            "train": train, "flip": flip, "pad": pad}


def _score(R, D, V, dtype="bf16", train=True, flip=True, pad=0):
    return {"kind": "score", "R": R, "D": D, "V": V, "dtype": dtype, "train": train, "flip": flip, "pad": pad}


def listed():
    return [
        # The routed network's router on a minibatch.
        {"name": "route-128x2of4", **_route(128, 2, 4)},
        # A training step's token batch, many experts.
        {"name": "route-65536x8of256", **_route(65536, 8, 256)},
        # The routed network's rows on a minibatch.
        {"name": "exchange-128x2x96", **_exchange(128, 2, 4, 96, "f32")},
        # A token batch of a large model.
        {"name": "exchange-16384x8x2048", **_exchange(16384, 8, 64, 2048)},
        # One token of a served model: eight experts, a row each.
        {"name": "multiply-token-8of64x2048x1024", **_multiply(1, 8, 64, 2048, 1024, train=False)},
        # The routed network's products on a minibatch; weights are views of the flat fp32 parameters.
        {"name": "multiply-256x96x64", **_multiply(128, 2, 4, 96, 64, weights="f32")},
        # Odd widths and ragged experts, rows that lie in a wider buffer.
        {"name": "multiply-odd-4093x3x1021x509", **_multiply(4093, 3, 7, 1021, 509, "f16", pad=3)},
        # A training step's token batch of a large model.
        {"name": "multiply-32768x4096x2048", **_multiply(8192, 4, 32, 4096, 2048)},
        # The 784-200-10 network's last product and loss on a minibatch.
        {"name": "score-128x200x10", **_score(128, 200, 10, "f32", flip=False)},
        # How likely a served model's next token was.
        {"name": "score-token-4096x131072", **_score(1, 4096, 131072, train=False)},
        # Odd widths and an odd number of classes.
        {"name": "score-odd-1021x999x50021", **_score(1021, 999, 50021, "f16", flip=False)},
        # A training step's token batch, a large vocabulary.
        {"name": "score-8192x2048x131072", **_score(8192, 2048, 131072)},
    ]


def _size(rng, lo, hi):
    """Log-uniform; half of them whole multiples of 8 where that fits."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))
    if n >= 16 and rng.random() < 0.5:
        n = n // 8 * 8
    return max(lo, min(max(lo, hi), n))


def draw(rng):
    kind = rng.choice(["route", "exchange", "multiply", "multiply", "score", "score"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    pad = rng.choice([0, 0, 0, 16, 3])
    train = rng.random() < 0.75
    if kind == "score":
        V = _size(rng, 2, 262144)
        D = _size(rng, 16, min(4096, (1 << 29) // V))
        R = _size(rng, 1, min(16384, (1 << 41) // (V * D), (1 << 30) // V))
        return _score(R, D, V, dtype, train, rng.random() < 0.5, pad)
    E = _size(rng, 2, 256)
    top = rng.randint(1, min(8, E))
    if kind == "route":
        return _route(_size(rng, 1, 65536), top, E)
    if kind == "exchange":
        D = _size(rng, 8, 8192)
        return _exchange(_size(rng, 1, min(65536, (1 << 27) // (D * top))), top, E, D, dtype, train, pad)
    E = min(E, 128)
    top = min(top, E)
    K = _size(rng, 16, min(8192, (1 << 27) // E // 16))
    N = _size(rng, 16, min(8192, (1 << 27) // E // K))
    T = _size(rng, 1, min(8192, 32768 // top, (1 << 37) // (K * N * top)))
    return _multiply(T, top, E, K, N, dtype, rng.choice(["same", "same", "f32"]), train, rng.random() < 0.5, pad)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _rows(g, R, D, pad, dtype, scale):
    """R rows of D values that lie `pad` values apart."""
    wide = torch.randn(R, D + pad, generator=g, device="cuda", dtype=torch.float32) * scale
    return wide.to(dtype)[:, :D]


def _choices(g, T, top, E):
    """A router's choices, some experts well liked; one in fifty found its expert full."""
    scores = torch.randn(T, E, generator=g, device="cuda") + torch.randn(E, generator=g, device="cuda")
    chosen = torch.topk(scores, top, dim=1).indices.to(torch.int32)
    if T > 1:
        chosen[torch.rand(T, top, generator=g, device="cuda") < 0.02] = -1
    return chosen


def _weights(g, shape, flip, dtype, scale):
    if flip:
        shape = (*shape[:-2], shape[-1], shape[-2])
    w = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)
    return w.transpose(-1, -2) if flip else w


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "score":
        R, D, V, pad, dtype = case["R"], case["D"], case["V"], case["pad"], TYPES[case["dtype"]]
        s["w"] = _weights(g, (D, V), case["flip"], dtype, 2.0 * D ** -0.5)
        # Frequent and rare classes; rows between ignorant and certain of theirs; a tenth has no label.
        u = torch.rand(R, generator=g, device="cuda", dtype=torch.float64)
        s["labels"] = torch.exp(u * math.log(V)).floor().clamp(1, V).long() - 1
        z = _rows(g, R, D, pad, torch.float32, 1.0)
        push = torch.rand(R, 1, generator=g, device="cuda") * 5.0
        z = z + push * s["w"][:, s["labels"]].t().float()
        s["z"] = torch.nn.functional.pad(z.to(dtype), (0, pad))[:, :D]
        if R > 1:
            s["labels"][torch.rand(R, generator=g, device="cuda") < 0.1] = -1
        return s
    T, top, E = case["T"], case["top"], case["E"]
    s["chosen"] = _choices(g, T, top, E)
    if case["kind"] == "route":
        return s
    s["offsets"], s["order"], s["place"] = _plain_route(s["chosen"], E).values()
    dtype = TYPES[case["dtype"]]
    n, pad = T * top, case["pad"]
    if case["kind"] == "multiply":
        K, N = case["K"], case["N"]
        s["x"] = _rows(g, n, K, pad, dtype, 1.0)
        s["w"] = _weights(g, (E, K, N), case["flip"], dtype if case["weights"] == "same" else torch.float32, K ** -0.5)
        if case["train"]:
            s["dy"] = _rows(g, n, N, pad, dtype, 0.05)
        s["bounds"] = s["offsets"].tolist()     # what a loop over the experts takes
        return s
    D = case["D"]
    s["x"] = _rows(g, T, D, pad, dtype, 1.0)
    s["y"] = _rows(g, n, D, pad, dtype, 0.7)
    s["weight"] = torch.softmax(torch.randn(T, top, generator=g, device="cuda"), 1)
    if case["train"]:
        s["dout"] = _rows(g, T, D, pad, dtype, 0.05)
        s["dxs"] = _rows(g, n, D, pad, dtype, 0.05)
    return s


def work(case):
    kind = case["kind"]
    if kind == "score":
        R, D, V = case["R"], case["D"], case["V"]
        size = 4 if case["dtype"] == "f32" else 2
        sides = 2 if case["train"] else 1        # read, and written as gradients
        return {"bytes": sides * (R * D + D * V) * size + 12 * R + 4, "flops": (6 if case["train"] else 2) * R * D * V}
    n = case["T"] * case["top"]
    if kind == "route":
        return {"bytes": 4 * n + 8 * n + 4 * (case["E"] + 1), "flops": n}
    size = 4 if case["dtype"] == "f32" else 2
    if kind == "exchange":
        T, D = case["T"], case["D"]
        once = (2 * T + 2 * n) * D * size + 12 * n            # x, xs, y, out; order, place, weight
        if not case["train"]:
            return {"bytes": once, "flops": 2 * n * D}
        return {"bytes": once + (2 * T + 2 * n) * D * size + 4 * n, "flops": 6 * n * D}   # dout, dy, dxs, dx; dweight
    K, N, E = case["K"], case["N"], case["E"]
    wsize = size if case["weights"] == "same" else 4
    read = n * K * size + min(E, n) * K * N * wsize + 4 * (E + 1)
    if not case["train"]:
        return {"bytes": read + n * N * size, "flops": 2 * n * K * N}
    return {"bytes": read + 2 * n * N * size + n * K * size + E * K * N * wsize, "flops": 6 * n * K * N}


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"route": _own_route, "exchange": _own_exchange, "multiply": _own_multiply, "score": _own_score}[kind](s)
    if kind == "route":
        return _plain_route(s["chosen"], s["case"]["E"])
    return {"exchange": _plain_exchange, "multiply": _plain_multiply, "score": _plain_score}[kind](s)


def _own_route(s):
    from paper_1601_04033_gb300 import client
    r = client.route(s["chosen"], s["case"]["E"])
    return {"offsets": r.offsets, "order": r.order, "place": r.place}


def _own_exchange(s):
    from paper_1601_04033_gb300 import client
    route = client.Route(s["offsets"], s["order"], s["place"])
    out = {"xs": client.gather(s["x"], route), "out": client.combine(s["y"], route, s["weight"])}
    if s["case"]["train"]:
        out["dy"], out["dweight"] = client.combine_grad(s["y"], route, s["weight"], s["dout"])
        out["dx"] = client.combine(s["dxs"], route)
    return out


def _own_multiply(s):
    from paper_1601_04033_gb300 import client
    out = {"y": client.multiply(s["x"], s["w"], s["offsets"])}
    if s["case"]["train"]:
        out["dx"], out["dw"] = client.multiply_grad(s["x"], s["w"], s["offsets"], s["dy"])
    return out


def _own_score(s):
    from paper_1601_04033_gb300 import client
    r = client.score(s["z"], s["w"], s["labels"], grad=s["case"]["train"])
    out = {"loss": r.loss, "rows": r.rows}
    if s["case"]["train"]:
        out.update(dz=r.dz, dw=r.dw)
    return out


def _plain_route(chosen, E):
    T, top = chosen.shape
    flat = chosen.reshape(-1)
    kept = (flat >= 0) & (flat < E)
    key = torch.where(kept, flat, E)
    order = torch.argsort(key, stable=True)
    counts = torch.zeros(E + 1, dtype=torch.int64, device="cuda").index_add_(0, key.long(), torch.ones_like(order))
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(counts[:E], 0)
    i = torch.arange(T * top, device="cuda")
    place = torch.empty_like(i)
    place[order] = i
    place = torch.where(kept, place, -1)
    order = torch.where(i < offsets[E], order, -1)
    return {"offsets": offsets, "order": order.to(torch.int32), "place": place.to(torch.int32).reshape(T, top)}


def _plain_exchange(s):
    c = s["case"]
    top, dtype = c["top"], TYPES[c["dtype"]]
    order, place = s["order"].long(), s["place"].long()
    there, kept = (order >= 0)[:, None], (place >= 0)[:, :, None]
    token = torch.clamp(order, min=0) // top

    def back(rows, weight):
        taken = torch.where(kept, rows.float()[torch.clamp(place, min=0)], 0.0)
        return taken, (taken if weight is None else taken * weight[:, :, None]).sum(1).to(dtype)

    taken, out = back(s["y"], s["weight"])
    r = {"xs": torch.where(there, s["x"][token], 0.0).to(dtype), "out": out}
    if c["train"]:
        weight = s["weight"].reshape(-1)[torch.clamp(order, min=0)][:, None]
        r["dy"] = torch.where(there, weight * s["dout"].float()[token], 0.0).to(dtype)
        r["dweight"] = (taken * s["dout"].float()[:, None, :]).sum(2)
        r["dx"] = back(s["dxs"], None)[1]
    return r


def _plain_multiply(s):
    c, x, w = s["case"], s["x"], s["w"]
    train, bounds = c["train"], s["bounds"]
    y = torch.zeros(x.shape[0], c["N"], dtype=x.dtype, device="cuda")
    if train:
        dx, dw = torch.zeros(x.shape, dtype=x.dtype, device="cuda"), torch.zeros_like(w)
    for e in range(c["E"]):
        a, b = bounds[e], bounds[e + 1]
        if a == b:
            continue
        xe, we = x[a:b].float(), w[e].to(x.dtype).float()
        y[a:b] = (xe @ we).to(x.dtype)
        if train:
            d = s["dy"][a:b].float()
            dx[a:b] = (d @ we.t()).to(x.dtype)
            dw[e] = (xe.t() @ d).to(w.dtype)
    return {"y": y, "dx": dx, "dw": dw} if train else {"y": y}


def _plain_score(s):
    c, z, w, V = s["case"], s["z"].float(), s["w"].float(), s["case"]["V"]
    kept = (s["labels"] >= 0) & (s["labels"] < V)
    label = torch.where(kept, s["labels"], 0)[:, None]
    logits = z @ w
    top = logits.max(1, keepdim=True).values
    lse = top + torch.log(torch.exp(logits - top).sum(1, keepdim=True))
    rows = torch.where(kept, (lse - torch.gather(logits, 1, label))[:, 0], 0.0)
    share = 1.0 / torch.clamp(kept.sum().float(), min=1.0)
    out = {"loss": (rows.sum() * share).reshape(1), "rows": rows}
    if c["train"]:
        p = torch.exp(logits.sub_(lse))
        p.scatter_add_(1, label, torch.full_like(lse, -1.0))
        p.mul_(torch.where(kept, share, 0.0)[:, None])
        out["dz"] = (p @ w.t()).to(s["z"].dtype)
        out["dw"] = _like(z.t() @ p, s["w"])
    return out


def _like(t, w):
    """t in w's type and layout."""
    return torch.empty_like(w).copy_(t)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"route": _exact_route, "exchange": _exact_exchange, "multiply": _exact_multiply,
            "score": _exact_score}[case["kind"]](case, s)


def _exact_route(case, s):
    import numpy as np
    chosen, E = s["chosen"].cpu().numpy().reshape(-1), case["E"]
    by = [np.nonzero(chosen == e)[0] for e in range(E)]
    order = np.full(chosen.size, -1, np.int32)
    place = np.full(chosen.size, -1, np.int32)
    offsets = np.zeros(E + 1, np.int32)
    for e, a in enumerate(by):
        offsets[e + 1] = offsets[e] + a.size
        order[offsets[e]:offsets[e + 1]] = a
        place[a] = np.arange(offsets[e], offsets[e + 1])
    return {k: torch.from_numpy(v).cuda() for k, v in
            (("offsets", offsets), ("order", order), ("place", place.reshape(case["T"], case["top"])))}


def _exact_exchange(case, s):
    T, top, D = case["T"], case["top"], case["D"]
    n, chosen = T * top, s["chosen"].reshape(-1)
    kept = torch.nonzero(chosen >= 0)[:, 0]                       # assignments that have a place
    at = s["place"].reshape(-1)[kept].long()
    token = kept // top
    weight = s["weight"].double().reshape(-1)[kept]

    def zeros(*shape):
        return torch.zeros(shape, dtype=torch.float64, device="cuda")

    out = {"xs": zeros(n, D).index_copy_(0, at, s["x"].double()[token]),
           "out": zeros(T, D).index_add_(0, token, s["y"].double()[at] * weight[:, None])}
    if case["train"]:
        d = s["dout"].double()[token]
        out["dy"] = zeros(n, D).index_copy_(0, at, d * weight[:, None])
        out["dweight"] = zeros(n).index_copy_(0, kept, torch.einsum("ad,ad->a", d, s["y"].double()[at])).reshape(T, top)
        out["dx"] = zeros(T, D).index_add_(0, token, s["dxs"].double()[at])
    return out


def _exact_multiply(case, s):
    n, K, N, E = case["T"] * case["top"], case["K"], case["N"], case["E"]
    expert = torch.sort(s["chosen"].reshape(-1)).values           # of each place, the dropped ones first
    expert = expert[expert >= 0]
    y = torch.zeros(n, N, dtype=torch.float64, device="cuda")
    dx = torch.zeros(n, K, dtype=torch.float64, device="cuda")
    dw = torch.zeros(E, K, N, dtype=torch.float64, device="cuda") if case["train"] else None
    for e in expert.unique().tolist():
        i = torch.nonzero(expert == e)[:, 0]
        x, w = s["x"][i].double(), s["w"][e].to(s["x"].dtype).double()
        y[i] = x @ w
        if case["train"]:
            d = s["dy"][i].double()
            dx[i] = d @ w.t()
            dw[e] = x.t() @ d
    return {"y": y, "dx": dx, "dw": dw} if case["train"] else {"y": y}


def _exact_score(case, s):
    R, D, V = case["R"], case["D"], case["V"]
    w = s["w"].double()
    rows = torch.zeros(R, dtype=torch.float64, device="cuda")
    count = int((s["labels"] >= 0).sum())
    dz = torch.zeros(R, D, dtype=torch.float64, device="cuda")
    dw = torch.zeros(D, V, dtype=torch.float64, device="cuda") if case["train"] else None
    step = max(1, (1 << 28) // V)
    for a in range(0, R, step):
        i = a + torch.nonzero(s["labels"][a:a + step] >= 0)[:, 0]
        if i.numel() == 0:
            continue
        z, y = s["z"][i].double(), s["labels"][i]
        logp = torch.log_softmax(z @ w, 1)
        rows[i] = -logp[torch.arange(i.numel(), device="cuda"), y]
        if case["train"]:
            g = logp.exp_()
            g[torch.arange(i.numel(), device="cuda"), y] -= 1.0
            g /= count
            dz[i] = g @ w.t()
            dw.addmm_(z.t(), g)
    out = {"loss": (rows.sum() / max(count, 1)).reshape(1), "rows": rows}
    if case["train"]:
        out.update(dz=dz, dw=dw)
    return out
