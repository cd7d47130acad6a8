"""What is measured of the client's operators: what a client computes between a
fetch and a push besides its matrix products, in three kinds of case:

* ``join``     where a block's output meets the residual stream: the norm after
               the block, dropout, gate and residual scale, and the norm before
               the next block.  ``train``: the forward call, then the gradients of
               x, y and every parameter.
* ``dropout``  forward (plus the residual, where there is one), then the gradient.
* ``balance``  a router's balance and z losses, per-expert counts and the
               gradient of the logits.

Sizes are those of this package's workloads (minibatches of 128 and the hidden
widths 200 and 1,000 of its networks) and generic ones: powers of two, and odd
and ragged sizes between them.
"""

from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
CARRY, BRANCH = 0.95, 0.7
BALANCE, ZLOSS = 0.01, 0.001
CLIENT, COUNT = 5, (3 << 32) + 17       # whose draws, and how many it made before


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _join(R, D, dtype="bf16", norm="rms", groups=1, p=0.0, train=True, post=True, gate=True, pre=True, pad=0):
    return {"kind": "join", "R": R, "D": D, "dtype": dtype, "norm": norm, "groups": groups, "p": p,
            "train": train, "post": post, "gate": gate, "pre": pre, "pad": pad}


def _dropout(R, D, dtype="bf16", p=0.1, residual=False, pad=0):
    return {"kind": "dropout", "R": R, "D": D, "dtype": dtype, "p": p, "residual": residual, "pad": pad}


def _balance(T, E, k, dtype="f32", groups=1, ragged=False):
    return {"kind": "balance", "T": T, "E": E, "k": k, "dtype": dtype, "groups": groups, "ragged": ragged}


def listed():
    return [
        # One token through one join of a served model: what a call costs.
        {"name": "join-token", **_join(1, 4096, train=False)},
        # A batch of tokens being served, wide rows.
        {"name": "join-serve-64x8192", **_join(64, 8192, train=False)},
        # A minibatch of 128 at the hidden width of the 784-200-10 network.
        {"name": "join-128x200", **_join(128, 200, "f32", "layer", p=0.2)},
        # A ragged batch at an odd width: no row but the first starts on 16 bytes.
        {"name": "join-4093x1021", **_join(4093, 1021, p=0.1)},
        # Eight sequences of odd length, each with its own gate.
        {"name": "join-gates-8x1031x1024", **_join(8 * 1031, 1024, "f16", "layer", groups=8)},
        # A training step's token batch of a large model.
        {"name": "join-32768x4096", **_join(32768, 4096, p=0.1)},
        # The small network's hidden layer.
        {"name": "dropout-128x200", **_dropout(128, 200, "f32", 0.2)},
        # Rows that lie in a wider buffer, and a residual.
        {"name": "dropout-6007x1000-strided", **_dropout(6007, 1000, residual=True, pad=24)},
        # A large model's activations, and a residual.
        {"name": "dropout-65536x4096", **_dropout(65536, 4096, residual=True)},
        # A small router on a minibatch.
        {"name": "balance-128x8", **_balance(128, 8, 2)},
        # Sixteen padded sequences, an expert count that fills no vector evenly.
        {"name": "balance-16x2047x60", **_balance(16 * 2047, 60, 4, "bf16", groups=16, ragged=True)},
        # A training step's token batch, many experts.
        {"name": "balance-262144x256", **_balance(262144, 256, 8, "bf16")},
    ]


def _size(rng, lo, hi):
    """Log-uniform; half of them whole multiples of 8 where that fits."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n >= 16 and rng.random() < 0.5:
        n = n // 8 * 8
    return max(lo, min(hi, n))


def draw(rng):
    kind = rng.choice(["join", "join", "dropout", "balance"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    most = 1 << (25 if dtype == "f32" else 26)
    if kind == "balance":
        E = _size(rng, 4, 512)
        groups = rng.choice([1, 1, 2, 7, 32])
        L = _size(rng, 1, max(1, min(262144, most // E) // groups))
        return _balance(groups * L, E, rng.randint(1, min(8, E)), dtype, groups, rng.random() < 0.5)
    D = _size(rng, 8, 8192)
    p = rng.choice([0.0, 0.1, 0.25, 0.5])
    pad = rng.choice([0, 0, 0, 16, 3])
    if kind == "dropout":
        return _dropout(_size(rng, 1, max(1, most // D)), D, dtype, max(p, 0.1), rng.random() < 0.5, pad)
    groups = rng.choice([1, 1, 2, 13, 64])
    L = _size(rng, 1, max(1, min(32768, most // D) // groups))
    post, gate, pre = rng.choice([(True, True, True), (True, True, True), (False, True, True),
                                  (True, False, True), (True, True, False), (False, False, True)])
    return _join(groups * L, D, dtype, rng.choice(["rms", "layer"]), groups if gate else 1, p,
                 rng.random() < 0.75, post, gate, pre, pad)


def _rows(g, R, D, pad, dtype, scale):
    """R rows of D values that lie `pad` values apart."""
    wide = torch.randn(R, D + pad, generator=g, device="cuda", dtype=torch.float32) * scale
    return wide.to(dtype)[:, :D]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case, "draws": (seed * 0x9E3779B97F4A7C15 + 0x5851F42D4C957F2D) & ((1 << 64) - 1)}
    dtype = TYPES[case["dtype"]]
    if case["kind"] == "balance":
        T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
        liking = torch.randn(E, generator=g, device="cuda") * 0.7
        logits = torch.randn(T, E, generator=g, device="cuda") * 1.5 + liking
        s["chosen"] = torch.topk(logits, k, dim=1).indices.to(torch.int32)
        # One assignment in fifty found its expert full.
        s["chosen"][torch.rand(T, k, generator=g, device="cuda") < 0.02] = -1
        s["logits"] = logits.to(dtype)
        s["valid"] = None
        if case["ragged"]:
            length = torch.randint(0, T // G + 1, (G, 1), generator=g, device="cuda")
            s["valid"] = (torch.arange(T // G, device="cuda")[None] < length).reshape(T).to(torch.uint8)
        return s
    R, D, pad = case["R"], case["D"], case["pad"]
    if case["kind"] == "dropout":
        s["x"] = _rows(g, R, D, pad, dtype, 1.0)
        s["residual"] = _rows(g, R, D, pad, dtype, 2.0) if case["residual"] else None
        s["dout"] = _rows(g, R, D, pad, dtype, 0.05)
        return s
    layer = case["norm"] == "layer"
    # A residual stream with a few loud channels and an offset.
    loud = torch.exp(torch.randn(D, generator=g, device="cuda") * 0.5)
    s["x"] = (_rows(g, R, D, pad, torch.float32, 1.5) * loud + 0.1).to(dtype)
    if pad:
        s["x"] = torch.nn.functional.pad(s["x"], (0, pad))[:, :D]
    s["y"] = _rows(g, R, D, pad, dtype, 0.6)
    if case["train"]:
        s["dh"] = _rows(g, R, D, pad, dtype, 0.05)
        s["dz"] = _rows(g, R, D, pad, dtype, 0.05) if case["pre"] else None

    def vector(mean, spread):
        return torch.randn(D, generator=g, device="cuda") * spread + mean

    s["post"] = vector(1.0, 0.2) if case["post"] else None
    s["post_bias"] = vector(0.0, 0.1) if case["post"] and layer else None
    s["pre"] = vector(1.0, 0.2) if case["pre"] else None
    s["pre_bias"] = vector(0.0, 0.1) if case["pre"] and layer else None
    s["gate"] = None
    if case["gate"]:     # one learned vector, or one computed per group of rows
        G = case["groups"]
        s["gate"] = vector(0.4, 0.2) if G == 1 else \
            (torch.randn(G, D, generator=g, device="cuda") * 0.3 + 0.4).to(dtype)
    return s


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "balance":
        T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
        return {"bytes": 2 * T * E * size + 4 * T * k + (T if case["ragged"] else 0) + 4 * G * E, "flops": 12 * T * E}
    R, D = case["R"], case["D"]
    if case["kind"] == "dropout":    # x, dout, out, dx, and the residual
        return {"bytes": (5 if case["residual"] else 4) * R * D * size, "flops": 4 * R * D}
    vectors = (case["post"] + case["pre"]) * (2 if case["norm"] == "layer" else 1)
    gate = 0 if not case["gate"] else 4 * D if case["groups"] == 1 else case["groups"] * D * size
    once = 4 * vectors * D + gate
    forward = 3 + case["pre"]        # x, y, h and z
    if not case["train"]:
        return {"bytes": forward * R * D * size + once, "flops": 15 * R * D}
    grads = 3 + case["pre"]          # dh, dz, dx and dy
    return {"bytes": (forward + grads) * R * D * size + 2 * once, "flops": 50 * R * D}


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"join": _own_join, "dropout": _own_dropout, "balance": _own_balance}[kind](s)
    return {"join": _plain_join, "dropout": _plain_dropout, "balance": _plain_balance}[kind](s)


def _own_join(s):
    from paper_1601_04033_gb300 import client
    c = s["case"]
    draws = client.Draws(c["p"], s["draws"], CLIENT, COUNT) if c["p"] else None
    j = client.join(s["x"], s["y"], post=s["post"], post_bias=s["post_bias"], gate=s["gate"],
                    pre=s["pre"], pre_bias=s["pre_bias"], norm=c["norm"], eps=EPS, carry=CARRY,
                    branch=BRANCH, draws=draws)
    out = {"h": j.h, "z": j.z}
    if c["train"]:
        g = client.join_grad(j, s["dh"], s["dz"])
        out.update(dx=g.x, dy=g.y, dpost=g.post, dpost_bias=g.post_bias, dgate=g.gate, dpre=g.pre,
                   dpre_bias=g.pre_bias)
    return out


def _own_dropout(s):
    from paper_1601_04033_gb300 import client
    draws = client.Draws(s["case"]["p"], s["draws"], CLIENT, COUNT)
    return {"out": client.dropout(s["x"], draws, residual=s["residual"]), "dx": client.dropout(s["dout"], draws)}


def _own_balance(s):
    from paper_1601_04033_gb300 import client
    b = client.balance(s["logits"], s["chosen"], balance=BALANCE, z=ZLOSS, groups=s["case"]["groups"],
                       valid=s["valid"], grad=True)
    return {"loss": b.loss, "counts": b.counts, "dlogits": b.dlogits}


def _philox(q, seed):
    """The four words of Philox4x32-10 at counter (q, client + 3 * 2^30, count,
    count >> 32, with q's upper half above bit 16), key = seed: int64 tensors
    (a product of two 32-bit words keeps its low 64 bits)."""
    low = 0xFFFFFFFF
    c0, c1 = q & low, torch.full_like(q, CLIENT + (3 << 30))
    c2, c3 = torch.full_like(q, COUNT & low), (COUNT >> 32) | ((q >> 32) << 16)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _factors(s):
    """What each element is multiplied by, fp32[R, D]: 0 where dropped."""
    R, D = s["case"]["R"], s["case"]["D"]
    n = R * D
    cut = int(math.floor(s["case"]["p"] * 65536 + 0.5))
    words = torch.stack(_philox(torch.arange((n + 7) // 8, device="cuda"), s["draws"]), dim=1)
    halves = torch.stack((words & 0xFFFF, words >> 16), dim=2).reshape(-1)[:n].reshape(R, D)
    return torch.where(halves >= cut, 65536.0 / (65536 - cut), 0.0).to(torch.float32)


def _plain_norm(t, weight, bias, layer):
    D = t.shape[1]
    if layer:
        t = t - t.sum(1, keepdim=True) / D
    rstd = 1.0 / torch.sqrt((t * t).sum(1, keepdim=True) / D + EPS)
    hat = t * rstd
    out = hat * weight
    return (out if bias is None else out + bias), hat, rstd


def _plain_norm_grad(dout, weight, hat, rstd, layer):
    D = hat.shape[1]
    q = dout * weight
    dt = q - hat * ((q * hat).sum(1, keepdim=True) / D)
    if layer:
        dt = dt - q.sum(1, keepdim=True) / D
    return dt * rstd, (dout * hat).sum(0), dout.sum(0)


def _plain_join(s):
    c = s["case"]
    dtype, layer = TYPES[c["dtype"]], c["norm"] == "layer"
    R, D, G = c["R"], c["D"], c["groups"]
    x, t = s["x"].float(), s["y"].float()
    if s["post"] is not None:
        t, yhat, yr = _plain_norm(t, s["post"], s["post_bias"], layer)
    factors = _factors(s) if c["p"] else 1.0
    u = t * factors
    gate = 1.0
    if s["gate"] is not None:
        gate = s["gate"].float() if G == 1 else \
            s["gate"].float()[:, None, :].expand(G, R // G, D).reshape(R, D)
    h = CARRY * x + BRANCH * gate * u
    out = {"h": h.to(dtype), "z": None}
    if s["pre"] is not None:
        z, hhat, hr = _plain_norm(h, s["pre"], s["pre_bias"], layer)
        out["z"] = z.to(dtype)
    if not c["train"]:
        return out
    d = s["dh"].float()
    dpre = dpre_bias = dpost = dpost_bias = dgate = None
    if s["pre"] is not None:
        dn, dpre, dpre_bias = _plain_norm_grad(s["dz"].float(), s["pre"], hhat, hr, layer)
        d = d + dn
    if s["gate"] is not None:
        dgate = BRANCH * d * u
        dgate = dgate.sum(0) if G == 1 else dgate.reshape(G, R // G, D).sum(1).to(s["gate"].dtype)
    dy = BRANCH * gate * d * factors
    if s["post"] is not None:
        dy, dpost, dpost_bias = _plain_norm_grad(dy, s["post"], yhat, yr, layer)
    out.update(dx=(CARRY * d).to(dtype), dy=dy.to(dtype), dpost=dpost,
               dpost_bias=None if s["post_bias"] is None else dpost_bias, dgate=dgate, dpre=dpre,
               dpre_bias=None if s["pre_bias"] is None else dpre_bias)
    return out


def _plain_dropout(s):
    dtype, factors = TYPES[s["case"]["dtype"]], _factors(s)
    y = s["x"].float() * factors
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"out": y.to(dtype), "dx": (s["dout"].float() * factors).to(dtype)}


def _plain_balance(s):
    c = s["case"]
    T, E, k, G = c["T"], c["E"], c["k"], c["groups"]
    valid = torch.ones(T, device="cuda") if s["valid"] is None else s["valid"].float()
    group = torch.arange(T, device="cuda") // (T // G)
    chosen = s["chosen"].long()
    kept = (chosen >= 0) & (chosen < E) & (valid > 0)[:, None]
    counts = torch.zeros(G * E, dtype=torch.int32, device="cuda")
    counts.index_add_(0, (group[:, None] * E + chosen)[kept], torch.ones_like(chosen[kept], dtype=torch.int32))
    counts = counts.reshape(G, E)
    rows = valid.reshape(G, T // G).sum(1)                    # valid rows of each group
    some = rows > 0
    per_row = torch.where(some, 1.0 / torch.clamp(rows, min=1.0), 0.0)
    f = counts.float() * (per_row / k)[:, None]
    logits = torch.where(valid[:, None] > 0, s["logits"].float(), 0.0)
    top = logits.max(1, keepdim=True).values
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    p = e / total * valid[:, None]
    lse = (top + torch.log(total))[:, 0] * valid
    groups = torch.clamp(some.float().sum(), min=1.0)
    n = torch.clamp(rows.sum(), min=1.0)
    P = p.reshape(G, T // G, E).sum(1) * per_row[:, None]
    lb = E * (f * P).sum() / groups
    lz = (lse * lse).sum() / n
    fr = f[:, None, :].expand(G, T // G, E).reshape(T, E)
    pull = fr - (fr * p).sum(1, keepdim=True)
    scale = (BALANCE * E / groups * per_row)[group][:, None]
    dlogits = p * (scale * pull + (2.0 * ZLOSS / n) * lse[:, None])
    return {"loss": torch.stack((BALANCE * lb + ZLOSS * lz, lb, lz)), "counts": counts,
            "dlogits": dlogits.to(s["logits"].dtype)}


# ---------------------------------------------------------------------------
# the definitions in 64 bits; gradients by differentiating the definition
# ---------------------------------------------------------------------------
def _exact_factors(case, draws):
    """The draws again, with 16-bit halves in the products so that none wraps."""
    R, D = case["R"], case["D"]
    q = torch.arange(-(-R * D // 8), device="cuda", dtype=torch.int64)

    def product(v, m):               # (high, low) 32 bits of v * m
        lo, hi = v % 65536 * m, v // 65536 * m
        lo, hi = lo + hi % 65536 * 65536, hi // 65536
        return hi + lo // (1 << 32), lo % (1 << 32)

    word = [q % (1 << 32), torch.zeros_like(q) + (CLIENT + 3 * 2**30), torch.zeros_like(q) + COUNT % (1 << 32),
            q // (1 << 32) * 65536 + COUNT // (1 << 32)]
    key = [draws % (1 << 32), draws // (1 << 32)]
    for _ in range(10):
        h0, l0 = product(word[0], 0xD2511F53)
        h1, l1 = product(word[2], 0xCD9E8D57)
        word = [h1 ^ word[1] ^ key[0], l1, h0 ^ word[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    draw16 = torch.empty(q.numel(), 8, dtype=torch.int64, device="cuda")
    for i in range(4):
        draw16[:, 2 * i] = word[i] % 65536
        draw16[:, 2 * i + 1] = word[i] // 65536
    cut = round(case["p"] * 65536)
    return (draw16.reshape(-1)[:R * D].reshape(R, D) >= cut).double() * (65536.0 / (65536 - cut))


def _exact_norm(t, weight, bias, layer):
    mean = t.mean(1, keepdim=True) if layer else 0.0
    return (t - mean) / torch.sqrt((t - mean).square().mean(1, keepdim=True) + EPS) * weight + \
        (0.0 if bias is None else bias)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "dropout":
        m = _exact_factors(case, s["draws"])
        out = s["x"].double() * m + (0.0 if s["residual"] is None else s["residual"].double())
        return {"out": out, "dx": s["dout"].double() * m}
    if case["kind"] == "balance":
        return _exact_balance(case, s)
    names = ("x", "y", "post", "post_bias", "gate", "pre", "pre_bias")
    v = {n: None if s[n] is None else s[n].double().requires_grad_(case["train"]) for n in names}
    layer, G = case["norm"] == "layer", case["groups"]
    u = v["y"] if v["post"] is None else _exact_norm(v["y"], v["post"], v["post_bias"], layer)
    if case["p"]:
        u = u * _exact_factors(case, s["draws"])
    if v["gate"] is not None:
        u = u * v["gate"] if G == 1 else (u.reshape(G, -1, case["D"]) * v["gate"][:, None]).reshape(u.shape)
    h = CARRY * v["x"] + BRANCH * u
    z = None if v["pre"] is None else _exact_norm(h, v["pre"], v["pre_bias"], layer)
    out = {"h": h.detach(), "z": None if z is None else z.detach()}
    if not case["train"]:
        return out
    given = [n for n in names if v[n] is not None]
    ends, with_ = ([h], [s["dh"].double()]) if z is None else ([h, z], [s["dh"].double(), s["dz"].double()])
    got = dict(zip(given, torch.autograd.grad(ends, [v[n] for n in given], with_)))
    out.update({"d" + n: got.get(n) for n in names})
    return out


def _exact_balance(case, s):
    T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
    L = T // G
    ok = torch.ones(T, dtype=torch.bool, device="cuda") if s["valid"] is None else s["valid"] != 0
    logits = s["logits"].double().requires_grad_(True)
    counts = torch.zeros(G, E, dtype=torch.int32, device="cuda")
    balance, live = torch.zeros((), dtype=torch.float64, device="cuda"), 0
    for g in range(G):
        rows = ok[g * L:(g + 1) * L]
        n = int(rows.sum())
        if n == 0:
            continue
        live += 1
        ids = s["chosen"][g * L:(g + 1) * L][rows].reshape(-1)
        counts[g] = torch.bincount(ids[(ids >= 0) & (ids < E)].long(), minlength=E).to(torch.int32)
        mean = torch.softmax(logits[g * L:(g + 1) * L][rows], 1).mean(0)
        balance = balance + E * (counts[g].double() / (k * n) * mean).sum()
    if live:
        balance = balance / live
        z = torch.logsumexp(logits[ok], 1).square().mean()
    else:
        z = (logits * 0.0).sum()
        balance = balance + z
    total = BALANCE * balance + ZLOSS * z
    dlogits, = torch.autograd.grad(total, [logits])
    return {"loss": torch.stack((total, balance, z)).detach(), "counts": counts, "dlogits": dlogits}
