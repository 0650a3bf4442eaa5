"""The work of three operators: norm and rotation of queries and keys, the gated scan, and the orthogonalised update; one call per case.

They make and train a layer that mixes the frames of a dynamic series (or the tokens of any sequence):
    q, k = rotate(norm(q)), rotate(norm(k)) in front of the attention;   h_t = a_t h_(t-1) + sqrt(1 - a_t^2) u_t beside it;
    and the step that the layers' weight matrices take: momentum, Newton-Schulz products, update.
The listed cases are calls at the feature maps and layers of this repository's own configurations, and at generic sizes; `draw` spreads
sizes, types, layouts and directions between and around them.

A case is a dict:
  op       qk | scan | muon;   dir: fwd | bwd (gradients of the same call);   dtype: f32 | bf16, type of the activations
qk:   queries and keys [B][T][P][heads][d], each head normed (root mean square) and its first `rot` values rotated by their position
  B, T, P  sequences, tokens of each, pixels that interleave;   Hq, Hk: heads;   d, rot: width, and how much of it is rotated
  pairs    halves: value j turns with value j + rot/2;   neighbours: 2j with 2j + 1
  packed   q and k are parts of one projection's output;   ragged: sequences of different lengths, an empty one among them
  place    start: each sequence has a first position;   each: every token has a position of its own
scan: x, r, i [B][T][P][C]
  packed, ragged as above;   state: with a state in and the state after it out
muon: `count` matrices of rows x cols float32
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
WIDTH = {"f32": 4, "bf16": 2}
KAPPA = 8.0


def _qk(direction, dtype, B, T, P, Hq, Hk, d, rot, pairs="halves", packed=1, ragged=0, place="start", name=None):
    c = dict(op="qk", dir=direction, dtype=dtype, B=B, T=T, P=P, Hq=Hq, Hk=Hk, d=d, rot=rot, pairs=pairs, packed=packed, ragged=ragged, place=place)
    if name:
        c["name"] = name
    return c


def _scan(direction, dtype, B, T, P, C, packed=1, ragged=0, state=0, name=None):
    c = dict(op="scan", dir=direction, dtype=dtype, B=B, T=T, P=P, C=C, packed=packed, ragged=ragged, state=state)
    if name:
        c["name"] = name
    return c


def _muon(count, rows, cols, name=None):
    c = dict(op="muon", count=count, rows=rows, cols=cols)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # Queries and keys of a cine series' feature map, 20 frames of 192 x 160 pixels, 64 channels in four heads, out of one projection.
        _qk("fwd", "bf16", 1, 20, 192 * 160, 4, 4, 16, 16, name="qk-fwd-20x192x160-4x16-bf16"),
        # Gradients of one very long sequence whose keys serve four heads each; half of the width carries positions.
        _qk("bwd", "bf16", 1, 16384, 1, 16, 4, 128, 64, name="qk-bwd-16384-16x128-kv4-bf16"),
        # Gradients in float32: ragged lengths, an odd layout of heads and widths, tokens with positions of their own.
        _qk("bwd", "f32", 3, 1001, 1, 6, 6, 40, 32, pairs="neighbours", ragged=1, place="each", name="qk-bwd-3x1001-6x40-f32"),
        # The next token of 64 sequences at once, each at its own place.
        _qk("fwd", "bf16", 64, 1, 1, 16, 4, 128, 128, name="qk-step-64-16x128-kv4-bf16"),
        # The frames of a cine series at each pixel: many short scans.
        _scan("fwd", "bf16", 1, 20, 192 * 160, 64, name="scan-fwd-20x192x160-64ch-bf16"),
        # One very long sequence: the scan has to be split along its tokens.
        _scan("fwd", "bf16", 1, 16384, 1, 1024, name="scan-fwd-16384-1024ch-bf16"),
        # Gradients of four ordinary sequences.
        _scan("bwd", "bf16", 4, 2048, 1, 1024, name="scan-bwd-4x2048-1024ch-bf16"),
        # Gradients in float32: ragged lengths, an odd number of channels, a state carried over from the sequences' earlier parts.
        _scan("bwd", "f32", 3, 1001, 1, 301, packed=0, ragged=1, state=1, name="scan-bwd-3x1001-301ch-f32"),
        # The next token of 64 sequences: the smallest call of a server.
        _scan("fwd", "bf16", 64, 1, 1, 1024, state=1, name="scan-step-64-1024ch-bf16"),
        # The projection of a small temporal layer, 64 channels to queries, keys and values: latency alone.
        _muon(1, 192, 64, name="muon-1x192x64"),
        # The three hidden layers of the 100-channel network in each of eight modules: 3 x 3 taps of 100 channels.
        _muon(24, 100, 900, name="muon-24x100x900"),
        # A wide layer of a generic size: the largest products.
        _muon(1, 1024, 4096, name="muon-1x1024x4096"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    costs = [work(c) for c in listed()]
    most_bytes, most_flops = max(w["bytes"] for w in costs), max(w["flops"] for w in costs)
    while True:
        op = rng.choice(("qk", "scan", "muon"))
        dtype, direction = rng.choice(("f32", "bf16")), rng.choice(("fwd", "bwd"))
        kind = rng.choice(("sequence", "sequence", "pixels", "step"))
        B, T, P = rng.randint(1, 8), _log(rng, 2, 16384), 1
        if kind == "pixels":
            B, T, P = rng.randint(1, 2), rng.randint(2, 64), _log(rng, 100, 40000)
        elif kind == "step":
            B, T, direction = _log(rng, 1, 256), 1, "fwd"
        packed, ragged = int(rng.random() < 0.6), int(rng.random() < 0.4)
        if op == "qk":
            Hq = rng.choice((1, 2, 3, 4, 6, 8, 12, 16, 32))
            Hk = rng.choice([h for h in (1, 2, 3, 4, 6, 8, 12, 16, 32) if Hq % h == 0])
            d = rng.choice((16, 32, 64, 128, 256)) if rng.random() < 0.6 else rng.randint(8, 256)
            rot = 2 * (d // 2) if rng.random() < 0.5 else 2 * rng.randint(1, d // 2)
            c = _qk(direction, dtype, B, T, P, Hq, Hk, d, rot, rng.choice(("halves", "neighbours")), packed, ragged, rng.choice(("start", "each")))
        elif op == "scan":
            C = 8 * _log(rng, 1, 512) if rng.random() < 0.6 else _log(rng, 8, 4096)
            c = _scan(direction, dtype, B, T, P, C, packed, ragged, int(kind == "step" or rng.random() < 0.4))
        else:
            c = _muon(_log(rng, 1, 32), _log(rng, 16, 2048), _log(rng, 16, 4096))
        w = work(c)
        if 2e4 <= w["bytes"] <= 0.5 * most_bytes and w["flops"] <= 0.5 * most_flops:
            return c


# ------------------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    {"qk": _prepare_qk, "scan": _prepare_scan, "muon": _prepare_muon}[case["op"]](case, gen, s)
    return s


def _normal(gen, c, *shape, mean=0.0, std=1.0):
    return torch.empty(*shape, device="cuda").normal_(mean, std, generator=gen).to(TYPES[c["dtype"]])


def _empty(c, *shape):
    return torch.empty(*shape, device="cuda", dtype=TYPES[c["dtype"]])


def _lengths(c, gen):
    if not c["ragged"]:
        return None
    B, T = c["B"], c["T"]
    lengths = torch.randint(0, T + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
    lengths[0], lengths[B // 2] = T, 0 if B > 1 else T
    return lengths


def _prepare_qk(c, gen, s):
    B, T, P, d = c["B"], c["T"], c["P"], c["d"]
    heads = (c["Hq"], c["Hk"])

    def both(make):
        """Arrays for q and k: on their own, or parts of the output of a projection to queries, keys and values."""
        if c["packed"]:
            return [x.unflatten(3, (-1, d)) for x in make(B, T, P, (heads[0] + 2 * heads[1]) * d).split([h * d for h in (*heads, heads[1])], 3)[:2]]
        return [make(B, T, P, h, d) for h in heads]

    s["q"], s["k"] = both(lambda *n: _normal(gen, c, *n))
    s["gamma_q"], s["gamma_k"] = (1.0 + 0.1 * torch.randn(d, device="cuda", generator=gen) for _ in range(2))
    half = c["rot"] // 2
    s["freq"] = 10000.0 ** (-torch.arange(half, device="cuda") / half)                     # radians a position
    s["eps"] = 1e-6
    first = torch.randint(0, 100000, (B,), device="cuda", generator=gen, dtype=torch.int32)
    s["positions"] = first
    if c["place"] == "each":                                                               # two documents in each row
        t = torch.arange(T, device="cuda", dtype=torch.int32)
        s["positions"] = torch.where(t < T // 2, t + first[:, None], t - T // 2).contiguous()
    s["lengths"] = _lengths(c, gen)
    if c["dir"] == "fwd":
        s["q_out"], s["k_out"] = (_empty(c, B, T, P, h, d) for h in heads)
    else:
        s["gq_out"], s["gk_out"] = (_normal(gen, c, B, T, P, h, d) for h in heads)
        s["gq"], s["gk"] = both(lambda *n: _empty(c, *n))
        s["ggamma_q"], s["ggamma_k"] = torch.empty_like(s["gamma_q"]), torch.empty_like(s["gamma_k"])
    if own:
        from paper_2207_08393_amd import binding as gb
        fwd = c["dir"] == "fwd"
        s["plan"] = gb.make_qknorm(s["q"], s["k"], s["q_out"] if fwd else s["gq_out"], s["k_out"] if fwd else s["gk_out"], c["rot"], s["eps"],
                                   pairs=c["pairs"], positions=c["place"])
        s["ws"] = torch.empty(0 if fwd else gb.gleam_qknorm_workspace_bytes(s["plan"]), dtype=torch.uint8, device="cuda")


def _prepare_scan(c, gen, s):
    B, T, P, C = c["B"], c["T"], c["P"], c["C"]
    three = (lambda make: make(B, T, P, 3 * C).split(C, 3)) if c["packed"] else (lambda make: [make(B, T, P, C) for _ in range(3)])
    s["x"], s["r"], s["i"] = three(lambda *n: _normal(gen, c, *n))
    # memories of 2 to 1000 tokens where the gate is half open
    memory = 2.0 * 500.0 ** torch.rand(C, device="cuda", generator=gen)
    s["lam"] = torch.log(torch.expm1(2.0 / (KAPPA * memory)))
    s["lengths"] = _lengths(c, gen)
    s["state"] = torch.randn(B, P, C, device="cuda", generator=gen) if c["state"] else None
    if c["dir"] == "fwd":
        s["h"] = _empty(c, B, T, P, C)
        s["state_out"] = torch.empty_like(s["state"]) if c["state"] else None
    else:
        s["g"] = _normal(gen, c, B, T, P, C)
        s["g_state_out"] = torch.randn(B, P, C, device="cuda", generator=gen) if c["state"] else None
        s["gx"], s["gr"], s["gi"] = three(lambda *n: _empty(c, *n))
        s["glam"] = torch.empty_like(s["lam"])
        s["g_state"] = torch.empty_like(s["state"]) if c["state"] else None
    if own:
        from paper_2207_08393_amd import binding as gb
        s["plan"] = gb.make_gatedscan(s["x"], s["r"], s["i"], s["h"] if c["dir"] == "fwd" else s["g"], kappa=KAPPA)
        fwd, bwd = gb.gleam_gatedscan_workspace_bytes(s["plan"])
        s["ws"] = torch.empty(fwd if c["dir"] == "fwd" else bwd, dtype=torch.uint8, device="cuda")


def _prepare_muon(c, gen, s):
    n, rows, cols = c["count"], c["rows"], c["cols"]
    few = max(1, min(rows, cols) // 8)

    def gradient():
        """A few strong directions and a floor of noise, as a mini-batch leaves them."""
        a, b = (torch.randn(n, k, few, device="cuda", generator=gen) for k in (rows, cols))
        a = a * torch.logspace(0, -2, few, device="cuda")
        return 1e-3 * (torch.matmul(a, b.transpose(1, 2).contiguous()) + 0.3 * torch.randn(n, rows, cols, device="cuda", generator=gen))

    s["theta"] = torch.randn(n, rows, cols, device="cuda", generator=gen) / math.sqrt(cols)
    s["grad"], s["m"] = gradient(), 5.0 * gradient()
    s["hyper"] = dict(lr=0.02, momentum=0.95, weight_decay=0.01, eps=1e-7, nesterov=1, steps=5, a=3.4445, b=-4.7750, c=2.0315)
    if own:
        from paper_2207_08393_amd import binding as gb
        s["plan"] = gb.make_muon(**s["hyper"])
        s["ws"] = torch.empty(gb.gleam_muon_workspace_bytes(n, rows, cols), dtype=torch.uint8, device="cuda")


def work(case):
    c = case
    if c["op"] == "muon":
        size, m, n = c["count"] * c["rows"] * c["cols"], min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
        # a step: half of X X^T, half of its square, and one full product; the rest is element by element
        return {"bytes": 20 * size, "flops": c["count"] * 5 * (3 * m * m * n + m * m * m)}
    tokens, w = c["B"] * c["T"] * c["P"], WIDTH[c["dtype"]]
    if c["op"] == "qk":
        size = tokens * (c["Hq"] + c["Hk"]) * c["d"]
        return {"bytes": size * w * (2 if c["dir"] == "fwd" else 3) + 8 * c["d"], "flops": size * (8 if c["dir"] == "fwd" else 16)}
    size, states = tokens * c["C"], 4 * c["B"] * c["P"] * c["C"] * c["state"]
    if c["dir"] == "fwd":
        return {"bytes": 4 * size * w + 2 * states, "flops": 25 * size}
    return {"bytes": 7 * size * w + 3 * states, "flops": 50 * size}


# -------------------------------------------------------------------------------------------------------- one pass
def run(state):
    s, c = state, state["case"]
    if own:
        return {"qk": _own_qk, "scan": _own_scan, "muon": _own_muon}[c["op"]](s, c)
    return {"qk": _plain_qk, "scan": _plain_scan, "muon": _plain_muon}[c["op"]](s, c)


def _own_qk(s, c):
    from paper_2207_08393_amd import binding as gb
    if c["dir"] == "fwd":
        gb.gleam_qknorm_fwd(s["plan"], s["q"], s["k"], s["gamma_q"], s["gamma_k"], s["freq"], s["positions"], s["lengths"], s["q_out"], s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    gb.gleam_qknorm_bwd(s["plan"], s["q"], s["k"], s["gamma_q"], s["gamma_k"], s["freq"], s["positions"], s["lengths"], s["gq_out"], s["gk_out"],
                        s["gq"], s["gk"], s["ggamma_q"], s["ggamma_k"], s["ws"])
    return {n: s[n] for n in ("gq", "gk", "ggamma_q", "ggamma_k")}


def _own_scan(s, c):
    from paper_2207_08393_amd import binding as gb
    if c["dir"] == "fwd":
        gb.gleam_gatedscan_fwd(s["plan"], s["x"], s["r"], s["i"], s["lam"], s["lengths"], s["state"], s["h"], s["state_out"], s["ws"])
        return {"h": s["h"], "state": s["state_out"]} if c["state"] else {"h": s["h"]}
    gb.gleam_gatedscan_bwd(s["plan"], s["x"], s["r"], s["i"], s["lam"], s["lengths"], s["state"], s["g"], s["g_state_out"], s["gx"], s["gr"], s["gi"],
                           s["glam"], s["g_state"], s["ws"])
    return {n: s[n] for n in ("gx", "gr", "gi", "glam") + (("g_state",) if c["state"] else ())}


def _own_muon(s, c):
    from paper_2207_08393_amd import binding as gb
    gb.gleam_muon_step(s["plan"], s["theta"], s["grad"], s["m"], s["ws"])
    return {"theta": s["theta"], "m": s["m"]}


def _live(c, s):
    """[B][T] of whether a token is there, or None: all are."""
    return None if s["lengths"] is None else torch.arange(c["T"], device="cuda") < s["lengths"][:, None]


def _turn(x, rot, pairs, cos, sin):
    """The first `rot` values of each head turned by the angle whose cosine and sine are given."""
    y, rest = x[..., :rot], x[..., rot:]
    a, b = (y[..., :rot // 2], y[..., rot // 2:]) if pairs == "halves" else (y[..., 0::2], y[..., 1::2])
    u, v = a * cos - b * sin, b * cos + a * sin
    return torch.cat((u, v, rest) if pairs == "halves" else (torch.stack((u, v), -1).flatten(-2), rest), -1)


def _plain_qk(s, c):
    where = s["positions"] if c["place"] == "each" else s["positions"][:, None] + torch.arange(c["T"], device="cuda")
    angle = (where.double()[..., None] * s["freq"].double())[:, :, None, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    live = _live(c, s)
    keep = (lambda x: x) if live is None else (lambda x: torch.where(live[:, :, None, None, None], x, torch.zeros((), device="cuda")))
    out = {}
    for name in ("q", "k"):
        x, gamma = s[name].float(), s["gamma_" + name]
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"])
        if c["dir"] == "fwd":
            out[name] = keep(_turn(x * r * gamma, c["rot"], c["pairs"], cos, sin)).to(s[name].dtype)
            continue
        g = _turn(keep(s["g" + name + "_out"].float()), c["rot"], c["pairs"], cos, -sin)
        gg = g * gamma
        out["g" + name] = keep(r * (gg - x * r * r * (gg * x).mean(-1, keepdim=True))).to(s[name].dtype)
        out["ggamma_" + name] = (g * keep(x * r)).sum((0, 1, 2, 3))
    return out


def _along(log_a, b):
    """h_t = exp(log_a_t) h_(t-1) + b_t from zero, along dimension 1, and the sums of log_a: stretches of twice the length, again and again."""
    k, T = 1, b.shape[1]
    while k < T:
        b = torch.cat((b[:, :k], b[:, k:] + torch.exp(log_a[:, k:]) * b[:, :-k]), 1)
        log_a = torch.cat((log_a[:, :k], log_a[:, k:] + log_a[:, :-k]), 1)
        k *= 2
    return b, log_a


def _plain_scan(s, c):
    live = _live(c, s)
    keep = (lambda x: x) if live is None else (lambda x: torch.where(live[:, :, None, None], x, torch.zeros((), device="cuda")))
    x, r, i = (keep(s[n].float()) for n in ("x", "r", "i"))
    rate = KAPPA * torch.log1p(torch.exp(s["lam"]))
    gate, gate_x = torch.sigmoid(r), torch.sigmoid(i)
    log_a = keep(-rate * gate)
    level = torch.sqrt(-torch.expm1(2.0 * log_a))
    u = gate_x * x
    h, since = _along(log_a, keep(level * u))
    if c["state"]:
        h = h + torch.exp(since) * s["state"][:, None]
    if c["dir"] == "fwd":
        out = {"h": keep(h).to(s["x"].dtype)}
        return {**out, "state": h[:, -1]} if c["state"] else out
    first = torch.zeros_like(h[:, :1]) if s["state"] is None else s["state"][:, None]
    before = torch.cat((first, h[:, :-1]), 1)
    # backwards in time, token t hands exp(log_a_t) of what it has to the one before it
    after = torch.cat((log_a[:, 1:], torch.zeros_like(log_a[:, :1])), 1)
    g, until = _along(after.flip(1), keep(s["g"].float()).flip(1))
    g, until = g.flip(1), until.flip(1)
    if c["state"]:
        g = g + torch.exp(until) * s["g_state_out"][:, None]
    a = torch.exp(log_a)
    g_log_a = g * (a * before - torch.where(level > 0, a * a / level, torch.zeros((), device="cuda")) * u)
    gu = g * level
    out = {"gx": gu * gate_x, "gr": keep(-rate * g_log_a * gate * (1.0 - gate)), "gi": gu * x * gate_x * (1.0 - gate_x)}
    out = {n: keep(v).to(s["x"].dtype) for n, v in out.items()}
    out["glam"] = (-KAPPA * torch.sigmoid(s["lam"])) * keep(g_log_a * gate).sum((0, 1, 2))
    if c["state"]:
        out["g_state"] = a[:, 0] * g[:, 0]
    return out


def _plain_muon(s, c):
    p, theta, m, grad = s["hyper"], s["theta"], s["m"], s["grad"]
    m.mul_(p["momentum"]).add_(grad)
    x = grad + p["momentum"] * m if p["nesterov"] else m
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + p["eps"])
    tall = c["rows"] > c["cols"]
    if tall:
        x = x.transpose(1, 2).contiguous()
    for _ in range(p["steps"]):
        a = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = p["a"] * x + torch.matmul(p["b"] * a + p["c"] * torch.matmul(a, a), x)
    if tall:
        x = x.transpose(1, 2)
    theta.mul_(1.0 - p["lr"] * p["weight_decay"]).sub_(p["lr"] * math.sqrt(max(1.0, c["rows"] / c["cols"])) * x)
    return {"theta": theta, "m": m}


# ---------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s, c = prepare(case, seed), case
    return {"qk": _exact_qk, "scan": _exact_scan, "muon": _exact_muon}[c["op"]](s, c)


def _exact_qk(s, c):
    """Pairs as complex numbers; gradients by differentiating the forward formula."""
    B, T, rot = c["B"], c["T"], c["rot"]
    steps = torch.arange(T, device="cuda", dtype=torch.float64)
    where = s["positions"].double() if c["place"] == "each" else s["positions"].double()[:, None] + steps
    angle = (where[:, :, None] * s["freq"].double()).view(B, T, 1, 1, rot // 2)
    turn = torch.polar(torch.ones_like(angle), angle)
    there = torch.ones(B, T, dtype=torch.float64, device="cuda") if s["lengths"] is None else (steps < s["lengths"].double()[:, None]).double()
    there = there.view(B, T, 1, 1, 1)

    def forward(x, gamma):
        y = x * gamma / torch.sqrt((x * x).sum(-1, keepdim=True) / c["d"] + s["eps"])
        z = torch.stack((y[..., :rot // 2], y[..., rot // 2:rot]) if c["pairs"] == "halves" else (y[..., 0:rot:2], y[..., 1:rot:2]), -1)
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        head = torch.cat((z[..., 0], z[..., 1]), -1) if c["pairs"] == "halves" else z.flatten(-2)
        return torch.cat((head, y[..., rot:]), -1) * there

    out = {}
    for name in ("q", "k"):
        x, gamma = s[name].double(), s["gamma_" + name].double()
        if c["dir"] == "fwd":
            out[name] = forward(x, gamma)
            continue
        x.requires_grad_(), gamma.requires_grad_()
        out["g" + name], out["ggamma_" + name] = torch.autograd.grad(forward(x, gamma), (x, gamma), s["g" + name + "_out"].double())
    return out


def _exact_scan(s, c):
    """Token by token, and back again."""
    B, T, P, C = c["B"], c["T"], c["P"], c["C"]
    lam, lengths = s["lam"].double(), s["lengths"]
    rate = KAPPA * torch.nn.functional.softplus(lam, threshold=50.0)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    on = [None if lengths is None else (t < lengths).view(B, 1, 1) for t in range(T)]
    only = lambda t, x: x if on[t] is None else torch.where(on[t], x, zero)  # noqa: E731
    state = torch.zeros(B, P, C, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()

    def parts(t):
        x, r, i = (s[n][:, t].double() for n in ("x", "r", "i"))
        gate, into = 1.0 / (1.0 + torch.exp(-r)), 1.0 / (1.0 + torch.exp(-i))
        lost = -torch.expm1(-2.0 * rate * gate)                            # 1 - a^2
        return x, gate, into, torch.exp(-rate * gate), torch.sqrt(lost), lost

    states = [state]
    for t in range(T):
        x, gate, into, a, level, _ = parts(t)
        state = a * state + level * into * x if on[t] is None else torch.where(on[t], a * state + level * into * x, state)
        states.append(state)
    if c["dir"] == "fwd":
        out = {"h": torch.stack([only(t, states[t + 1]) for t in range(T)], 1)}
        return {**out, "state": state} if c["state"] else out
    g = torch.zeros_like(state) if s["g_state_out"] is None else s["g_state_out"].double()
    glam, got = torch.zeros(C, dtype=torch.float64, device="cuda"), {n: [] for n in ("gx", "gr", "gi")}
    for t in reversed(range(T)):
        x, gate, into, a, level, lost = parts(t)
        now = g + s["g"][:, t].double()
        # level^2 = 1 - a^2, so d level = -(a / level) da = (a^2 rate / level) d gate
        by_gate = now * rate * (a * a * into * x / level - a * states[t])
        got["gx"].append(only(t, now * level * into))
        got["gi"].append(only(t, now * level * x * into * (1.0 - into)))
        got["gr"].append(only(t, by_gate * gate * (1.0 - gate)))
        glam += only(t, by_gate * gate).sum((0, 1)) / rate * KAPPA * torch.sigmoid(lam)
        g = a * now if on[t] is None else torch.where(on[t], a * now, g)
    out = {n: torch.stack(v[::-1], 1) for n, v in got.items()}
    out["glam"] = glam
    return {**out, "g_state": g} if c["state"] else out


def _exact_muon(s, c):
    """The polynomial a + b z + c z^2 of z = sigma^2 applied to the singular values, by products with the smaller Gram matrix."""
    p = s["hyper"]
    theta, grad, m = s["theta"].double(), s["grad"].double(), s["m"].double()
    m = p["momentum"] * m + grad
    x = p["momentum"] * m + grad if p["nesterov"] else m
    x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + p["eps"])
    eye = torch.eye(min(c["rows"], c["cols"]), dtype=torch.float64, device="cuda")
    for _ in range(p["steps"]):
        y = x.transpose(1, 2).contiguous()
        z = torch.matmul(y, x) if c["rows"] > c["cols"] else torch.matmul(x, y)
        poly = p["a"] * eye + torch.matmul(z, p["b"] * eye + p["c"] * z)
        x = torch.matmul(x, poly) if c["rows"] > c["cols"] else torch.matmul(poly, x)
    scale = p["lr"] * max(1.0, c["rows"] / c["cols"]) ** 0.5
    return {"theta": theta - p["lr"] * p["weight_decay"] * theta - scale * x, "m": m}
