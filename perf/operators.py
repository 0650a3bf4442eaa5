"""The work the layer-norm, dropout and decaying linear-attention operators are timed on: one call per case.

Together they mix the frames of a dynamic series (or the tokens of any sequence) between convolution layers:
    y = layer_norm(x)        q, k, v = projections of y        h = x + dropout(projection of linear_attention(q, k, v))
The listed cases are calls of such a layer at the feature maps of this repository's own configurations, and at generic
sequence sizes; `draw` spreads sizes, types, head layouts and directions between and around them.

A case is a dict:
  op       norm | dropout | mix
  dir      fwd | bwd (gradients of the same call)
  dtype    f32 | bf16: type of the activations; scale, shift, statistics, decays and states are float32 throughout
norm, dropout:
  rows, n  rows x row length;  pad: elements between the end of a row and the start of the next one
  p, add   dropout rate, and whether a residual is added in the same pass
mix:
  B, T, P  sequences, tokens of each, and pixels that interleave: an activation is [B][T][P][heads][width]
  H, Hq, Hk, Hv   heads of the output, and of q, k, v (each shared by H / its own number of output heads)
  dk, dv   widths of q, k and of v
  layout   tokens: q, k, v on their own; packed: side by side in one array; heads: [B][heads][T][width] (P = 1)
  ragged   sequences of different lengths, an empty one among them;  state: with a state in and the state after it out
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
WIDTH = {"f32": 4, "bf16": 2}
WORD = 0xFFFFFFFF


def _rows(op, direction, dtype, rows, n, pad=0, p=0.0, add=0, name=None):
    c = dict(op=op, dir=direction, dtype=dtype, rows=rows, n=n, pad=pad)
    if op == "dropout":
        c.update(p=p, add=add)
    if name:
        c["name"] = name
    return c


def _mix(direction, dtype, B, T, P, H, Hq, Hk, Hv, dk, dv, layout="tokens", ragged=0, state=0, name=None):
    c = dict(op="mix", dir=direction, dtype=dtype, B=B, T=T, P=P, H=H, Hq=Hq, Hk=Hk, Hv=Hv, dk=dk, dv=dv, layout=layout,
             ragged=ragged, state=state)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One small frame on its way through a streaming reconstruction: 64 x 64 pixels of 16 channels, all latency.
        _rows("norm", "fwd", "f32", 64 * 64, 16, name="norm-fwd-64x64-16ch-f32"),
        # The feature map of the 100-channel network, four slices of 320 x 256, in float32: a width that no power of two divides.
        _rows("norm", "fwd", "f32", 4 * 320 * 256, 100, name="norm-fwd-4x320x256-100ch-f32"),
        # Gradients at the 128-channel bfloat16 feature map, four slices of 640 x 320: the largest reduction over rows.
        _rows("norm", "bwd", "bf16", 4 * 640 * 320, 128, name="norm-bwd-4x640x320-128ch-bf16"),
        # Long rows of an odd length with gaps between them, as a slice of a wider array has.
        _rows("norm", "bwd", "f32", 2000, 5001, pad=7, name="norm-bwd-2000x5001-f32"),
        # Dropout and residual of a cine series' feature map, 20 frames of 192 x 160, 64 channels.
        _rows("dropout", "fwd", "bf16", 20 * 192 * 160, 64, p=0.1, add=1, name="dropout-fwd-20x192x160-64ch-bf16"),
        # The gradient through dropout at the 100-channel network's feature map: the same mask, drawn again.
        _rows("dropout", "bwd", "f32", 4 * 320 * 256, 100, p=0.2, name="dropout-bwd-4x320x256-100ch-f32"),
        # The frames of a cine series mixed at each pixel: many short sequences, narrow heads.
        _mix("fwd", "bf16", 1, 20, 192 * 160, 4, 4, 4, 4, 16, 16, name="mix-fwd-20x192x160-4x16-bf16"),
        # Four ordinary sequences, q, k and v side by side as one projection leaves them.
        _mix("fwd", "bf16", 4, 2048, 1, 16, 16, 16, 16, 64, 64, layout="packed", name="mix-fwd-4x2048-16x64-bf16"),
        # Gradients of one very long sequence whose keys and values serve four heads each.
        _mix("bwd", "bf16", 1, 16384, 1, 16, 16, 4, 4, 128, 128, name="mix-bwd-16384-16x128-kv4-bf16"),
        # Gradients in float32: ragged lengths, odd widths, a state carried over from the sequences' earlier parts.
        _mix("bwd", "f32", 3, 1001, 1, 6, 6, 6, 6, 40, 72, layout="packed", ragged=1, state=1, name="mix-bwd-3x1001-6x40x72-f32"),
        # The next token of 64 sequences at once: the states are read and written once.
        _mix("fwd", "bf16", 64, 1, 1, 16, 16, 16, 16, 128, 128, state=1, name="mix-step-64-16x128-bf16"),
        # The next token of one sequence: the smallest call of a server.
        _mix("fwd", "bf16", 1, 1, 1, 8, 8, 8, 8, 64, 64, state=1, name="mix-step-1-8x64-bf16"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    costs = [work(c) for c in listed()]
    most_bytes, most_flops = max(w["bytes"] for w in costs), max(w["flops"] for w in costs)
    while True:
        op = rng.choice(("norm", "dropout", "mix", "mix"))
        dtype, direction = rng.choice(("f32", "bf16")), rng.choice(("fwd", "bwd"))
        if op == "norm" or op == "dropout":
            rows, n = _log(rng, 1, 1e6), _log(rng, 8, 16384) if rng.random() < 0.6 else 4 * _log(rng, 4, 512)
            c = _rows(op, direction, dtype, rows, n, pad=rng.choice((0, 0, 0, 8, rng.randint(1, 40))), p=round(rng.uniform(0.0, 0.6), 3),
                      add=int(direction == "fwd" and rng.random() < 0.7))
        else:
            kind = rng.choice(("sequence", "sequence", "pixels", "step"))
            H = rng.choice((1, 2, 3, 4, 6, 8, 12, 16, 32))
            Hq, Hk, Hv = rng.choice(((1, 1, 1), (1, 1, 1), (1, 0, 0), (0, 0, 1)))   # 1: a head of its own each, 0: shared
            few = rng.choice([h for h in (1, 2, 3, 4) if H % h == 0])
            dk, dv = (rng.choice((16, 32, 64, 128)) if rng.random() < 0.6 else rng.randint(8, 128) for _ in range(2))
            B, T, P = rng.randint(1, 8), _log(rng, 2, 16384), 1
            if kind == "pixels":
                B, T, P, dk = rng.randint(1, 2), rng.randint(2, 64), _log(rng, 100, 40000), rng.choice((8, 12, 16, 25, 32))
                dv = dk
            elif kind == "step":
                B, T, direction = _log(rng, 1, 256), 1, "fwd"
            c = _mix(direction, dtype, B, T, P, H, H if Hq else few, H if Hk else few, H if Hv else few, dk, dv,
                     rng.choice(("tokens", "packed") if P > 1 else ("tokens", "packed", "heads")),
                     int(rng.random() < 0.4), int(kind == "step" or rng.random() < 0.4))
        w = work(c)
        if 2e4 <= w["bytes"] <= 0.5 * most_bytes and w["flops"] <= 0.5 * most_flops:
            return c


# ------------------------------------------------------------------------------------------------------------- inputs
def _strided(gen, rows, n, pad, dtype, mean=0.0, std=1.0):
    """rows x n values with `pad` unused elements behind each row."""
    x = torch.empty(rows, n + pad, device="cuda").normal_(mean, std, generator=gen)
    return x.to(TYPES[dtype])[:, :n]


def _like(x):
    """An array of x's own layout for a result."""
    return torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device)


def prepare(case, seed):
    c, gen = case, torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": c}
    if c["op"] == "mix":
        _prepare_mix(c, gen, s)
        return s
    x = _strided(gen, c["rows"], c["n"], c["pad"], c["dtype"], *((0.3, 1.5) if c["op"] == "norm" else ()))
    s["x"] = x
    if c["op"] == "dropout":
        s["seed"] = 0x9E3779B97F4A7C15 * (seed + 1) & 0xFFFFFFFFFFFFFFFF
        s["offset"] = seed % 1000 + 5 * 2 ** 32
        s["add"] = _strided(gen, c["rows"], c["n"], c["pad"], c["dtype"]) if c["add"] else None
        s["out"] = _like(x)
        if own:
            from paper_2207_08393_amd import binding as gb
            s["plan"] = gb.make_dropout(x.dtype, c["rows"], c["n"], c["p"], s["seed"], s["offset"], ld=c["n"] + c["pad"])
        return s
    s["gamma"] = 1.0 + 0.1 * torch.randn(c["n"], device="cuda", generator=gen)
    s["beta"] = 0.1 * torch.randn(c["n"], device="cuda", generator=gen)
    s["eps"] = 1e-5
    xf = x.float()
    mean = xf.mean(1)
    s["mean"], s["rstd"] = mean, torch.rsqrt((xf - mean[:, None]).square().mean(1) + s["eps"])
    if c["dir"] == "fwd":
        s["y"], s["mean"], s["rstd"] = _like(x), torch.empty_like(mean), torch.empty_like(mean)
    else:
        s["g"] = _strided(gen, c["rows"], c["n"], c["pad"], c["dtype"], 0.0, 0.1)
        s["gx"], s["ggamma"], s["gbeta"] = _like(x), torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
    if own:
        from paper_2207_08393_amd import binding as gb
        s["plan"] = gb.make_layer_norm(x.dtype, c["rows"], c["n"], s["eps"], ld=c["n"] + c["pad"])
        s["ws"] = torch.empty(gb.gleam_layer_norm_workspace_bytes(s["plan"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_mix(c, gen, s):
    B, T, P, H = c["B"], c["T"], c["P"], c["H"]
    sizes = (c["Hq"] * c["dk"], c["Hk"] * c["dk"], c["Hv"] * c["dv"])

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(TYPES[c["dtype"]])

    def empty(*shape):
        return torch.empty(*shape, device="cuda", dtype=TYPES[c["dtype"]])

    def part(make, h, d):
        return make(B, h, T, 1, d).permute(0, 2, 3, 1, 4) if c["layout"] == "heads" else make(B, T, P, h, d)

    def three(make):
        """Arrays of the layout of q, k and v."""
        if c["layout"] == "packed":
            return [a.unflatten(3, (h, -1)) for a, h in zip(make(B, T, P, sum(sizes)).split(sizes, 3), (c["Hq"], c["Hk"], c["Hv"]))]
        return part(make, c["Hq"], c["dk"]), part(make, c["Hk"], c["dk"]), part(make, c["Hv"], c["dv"])

    s["q"], s["k"], s["v"] = three(normal)
    s["scale"] = c["dk"] ** -0.5
    s["log_decay"] = torch.log1p(-torch.exp2(torch.linspace(-3.0, -10.0, H, device="cuda")))
    s["lengths"] = None
    if c["ragged"]:
        lengths = torch.randint(0, T + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
        lengths[0], lengths[B // 2] = T, 0 if B > 1 else T
        s["lengths"] = lengths
    s["state"] = torch.randn(B, P, H, c["dk"], c["dv"], device="cuda", generator=gen) if c["state"] else None
    if c["dir"] == "fwd":
        s["o"] = part(empty, H, c["dv"])
        s["state_out"] = torch.empty_like(s["state"]) if c["state"] else None
    else:
        s["g"] = part(normal, H, c["dv"])
        s["g_state_out"] = torch.randn(B, P, H, c["dk"], c["dv"], device="cuda", generator=gen) if c["state"] else None
        s["gq"], s["gk"], s["gv"] = three(empty)
        s["g_state"] = torch.empty_like(s["state"]) if c["state"] else None
    if own:
        from paper_2207_08393_amd import binding as gb
        s["plan"] = gb.make_linattn(s["q"], s["k"], s["v"], s["o"] if c["dir"] == "fwd" else s["g"], scale=s["scale"])
        fwd, bwd = gb.gleam_linattn_workspace_bytes(s["plan"])
        s["ws"] = torch.empty(fwd if c["dir"] == "fwd" else bwd, dtype=torch.uint8, device="cuda")


def work(case):
    c = case
    w = WIDTH[c["dtype"]]
    if c["op"] == "norm":
        size = c["rows"] * c["n"]
        if c["dir"] == "fwd":
            return {"bytes": 2 * size * w + 8 * c["n"] + 8 * c["rows"], "flops": 7 * size}
        return {"bytes": 3 * size * w + 12 * c["n"] + 8 * c["rows"], "flops": 12 * size}
    if c["op"] == "dropout":
        size = c["rows"] * c["n"]
        return {"bytes": (3 if c["add"] else 2) * size * w, "flops": 2 * size}
    tokens, states = c["B"] * c["T"] * c["P"], c["B"] * c["P"] * c["H"] * c["dk"] * c["dv"] * 4 * c["state"]
    read = tokens * (c["Hq"] * c["dk"] + c["Hk"] * c["dk"] + c["Hv"] * c["dv"]) * w
    out = tokens * c["H"] * c["dv"] * w
    products = tokens * c["H"] * c["dk"] * c["dv"]
    if c["dir"] == "fwd":
        return {"bytes": read + out + 2 * states, "flops": 4 * products}
    return {"bytes": 2 * read + out + 3 * states, "flops": 10 * products}


# -------------------------------------------------------------------------------------------------------- one pass
def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(s, c)
    if c["op"] == "norm":
        return _plain_norm(s, c)
    if c["op"] == "dropout":
        return _plain_dropout(s, c)
    return _plain_mix(s, c)


def _run_own(s, c):
    from paper_2207_08393_amd import binding as gb
    if c["op"] == "norm":
        if c["dir"] == "fwd":
            gb.gleam_layer_norm_fwd(s["plan"], s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"])
            return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        gb.gleam_layer_norm_bwd(s["plan"], s["x"], s["gamma"], s["mean"], s["rstd"], s["g"], s["gx"], s["ggamma"], s["gbeta"], s["ws"])
        return {"gx": s["gx"], "ggamma": s["ggamma"], "gbeta": s["gbeta"]}
    if c["op"] == "dropout":
        if c["dir"] == "fwd":
            gb.gleam_dropout_fwd(s["plan"], s["x"], s["add"], s["out"])
        else:
            gb.gleam_dropout_bwd(s["plan"], s["x"], s["out"])
        return {"out": s["out"]}
    if c["dir"] == "fwd":
        gb.gleam_linattn_fwd(s["plan"], s["q"], s["k"], s["v"], s["log_decay"], s["lengths"], s["state"], s["o"], s["state_out"], s["ws"])
        return {"o": s["o"], "state": s["state_out"]} if c["state"] else {"o": s["o"]}
    gb.gleam_linattn_bwd(s["plan"], s["q"], s["k"], s["v"], s["log_decay"], s["lengths"], s["state"], s["g"], s["g_state_out"],
                         s["gq"], s["gk"], s["gv"], s["g_state"], s["ws"])
    out = {"gq": s["gq"], "gk": s["gk"], "gv": s["gv"]}
    return {**out, "g_state": s["g_state"]} if c["state"] else out


def _plain_norm(s, c):
    x = s["x"].float()
    if c["dir"] == "fwd":
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + s["eps"])
        return {"y": (d * rstd * s["gamma"] + s["beta"]).to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    g, rstd = s["g"].float(), s["rstd"][:, None]
    xhat = (x - s["mean"][:, None]) * rstd
    gg = g * s["gamma"]
    gx = rstd * (gg - gg.mean(1, keepdim=True) - xhat * (gg * xhat).mean(1, keepdim=True))
    return {"gx": gx.to(s["x"].dtype), "ggamma": (g * xhat).sum(0), "gbeta": g.sum(0)}


def _philox_round(c, k0, k1):
    """One round of Philox 4x32 (Salmon et al., Parallel random numbers: as easy as 1, 2, 3, 2011); words in 64-bit integers."""
    a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57          # products modulo 2^64: the low 64 bits are right whatever the sign
    return [(b >> 32 & WORD) ^ c[1] ^ k0, b & WORD, (a >> 32 & WORD) ^ c[3] ^ k1, a & WORD]


def _plain_dropout(s, c):
    rows, n = c["rows"], c["n"]
    block = torch.arange((rows * n + 7) // 8, device="cuda")
    ctr = [block & WORD, block >> 32, torch.full_like(block, s["offset"] & WORD), torch.full_like(block, s["offset"] >> 32)]
    k0, k1 = s["seed"] & WORD, s["seed"] >> 32
    for i in range(10):
        ctr = _philox_round(ctr, (k0 + i * 0x9E3779B9) & WORD, (k1 + i * 0xBB67AE85) & WORD)
    draws = torch.stack([h for w in ctr for h in (w & 0xFFFF, w >> 16)], 1).reshape(-1)[:rows * n].reshape(rows, n)
    kept = int(math.floor(65536 * (1 - c["p"]) + 0.5))   # of 65536 draws
    out = torch.where(draws < kept, s["x"].float() * (65536 / max(kept, 1)), torch.zeros((), device="cuda"))
    return {"out": (out if s["add"] is None else s["add"].float() + out).to(s["x"].dtype)}


def _causal(q, k, v, a):
    """sum over s <= t of exp(a (t - s)) (q_t . k_s) v_s for arrays [..., H, T, width]: products inside blocks of tokens, and
    products with the sums over the blocks before."""
    T = q.shape[-2]
    C = min(T, 64)
    n = -(-T // C)
    q, k, v = (torch.nn.functional.pad(x, (0, 0, 0, n * C - T)).unflatten(-2, (n, C)) for x in (q, k, v))
    i = torch.arange(C, device=q.device, dtype=torch.float32)
    j = torch.arange(n, device=q.device, dtype=torch.float32)
    a = a[:, None, None]
    inside = torch.tril(torch.exp(a * (i[:, None] - i).clamp(min=0)))[:, None]
    between = torch.tril(torch.exp(a * C * (j[:, None] - 1 - j).clamp(min=0)), -1)
    sums = torch.matmul((k * torch.exp(a[..., None] * (C - 1 - i)[:, None])).transpose(-1, -2), v)
    before = torch.matmul(between, sums.flatten(-2)).unflatten(-1, sums.shape[-2:])
    o = torch.matmul(torch.matmul(q, k.transpose(-1, -2)) * inside, v)
    o = o + torch.matmul(q * torch.exp(a[..., None] * (i + 1)[:, None]), before)
    return o.flatten(-3, -2)[..., :T, :]


def _gather(x, H, live):
    """[B][T][P][h][d] of any type as float32 [B][P][H][T][d], heads repeated, zero behind the ends of the sequences."""
    x = x.float().repeat_interleave(H // x.shape[3], 3).permute(0, 2, 3, 1, 4)
    return x if live is None else torch.where(live, x, torch.zeros((), device=x.device))


def _scatter(x, like):
    """The way back: the sum over the output heads that share a head."""
    h = like.shape[3]
    return x.unflatten(2, (h, x.shape[2] // h)).sum(3).permute(0, 3, 1, 2, 4).to(like.dtype)


def _plain_mix(s, c):
    H, T, a = c["H"], c["T"], s["log_decay"]
    t = torch.arange(T, device="cuda")
    live = None if s["lengths"] is None else (t < s["lengths"][:, None])[:, None, None, :, None]
    length = torch.full((c["B"],), T, device="cuda") if s["lengths"] is None else s["lengths"]
    q, k, v = (_gather(s[x], H, live) for x in ("q", "k", "v"))
    if c["state"]:
        since = torch.exp(a[:, None] * (t + 1))[None, None, :, :, None]                                  # decay since the start
        until = torch.exp(a[:, None] * (length[:, None, None] - 1 - t).clamp(min=0))[:, None, :, :, None]    # and to the end
        all_of_it = torch.exp(a * length[:, None])[:, None, :, None, None]
    if c["dir"] == "fwd":
        o = _causal(q, k, v, a)
        if c["state"]:
            o = o + torch.matmul(q * since, s["state"])
        out = {"o": _scatter(s["scale"] * o, s["o"])}
        if c["state"]:
            out["state"] = all_of_it * s["state"] + torch.matmul((k * until).transpose(-1, -2), v)
        return out
    g = s["scale"] * _gather(s["g"], H, live)
    gq = _causal(g, v, k, a)
    gk = _causal(v.flip(-2), g.flip(-2), q.flip(-2), a).flip(-2)
    gv = _causal(k.flip(-2), q.flip(-2), g.flip(-2), a).flip(-2)
    out = {}
    if c["state"]:
        gq = gq + torch.matmul(g * since, s["state"].transpose(-1, -2))
        gk = gk + torch.matmul(v * until, s["g_state_out"].transpose(-1, -2))
        gv = gv + torch.matmul(k * until, s["g_state_out"])
        out["g_state"] = all_of_it * s["g_state_out"] + torch.matmul((q * since).transpose(-1, -2), g)
    for name, x in (("q", gq), ("k", gk), ("v", gv)):
        out["g" + name] = _scatter(x if live is None else torch.where(live, x, torch.zeros((), device="cuda")), s[name])
    return out


# ---------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "norm":
        x = s["x"].double()
        if c["dir"] == "fwd":
            var, mean = torch.var_mean(x, 1, correction=0)
            rstd = 1.0 / torch.sqrt(var + s["eps"])
            return {"y": torch.addcmul(s["beta"].double(), (x - mean[:, None]) / torch.sqrt(var + s["eps"])[:, None], s["gamma"].double()),
                    "mean": mean, "rstd": rstd}
        g, gamma, mean, rstd = (s[n].double() for n in ("g", "gamma", "mean", "rstd"))
        x.sub_(mean[:, None]).mul_(rstd[:, None])
        ggamma, gbeta = (g * x).sum(0), g.sum(0)
        g.mul_(gamma)
        along = (g * x).sum(1, keepdim=True) / c["n"]
        g.sub_(g.sum(1, keepdim=True) / c["n"]).sub_(x.mul_(along)).mul_(rstd[:, None])
        return {"gx": g, "ggamma": ggamma, "gbeta": gbeta}
    if c["op"] == "dropout":
        return _exact_dropout(s, c)
    return _exact_mix(s, c)


def _exact_dropout(s, c):
    size = c["rows"] * c["n"]
    word = np.uint64(WORD)
    index = np.arange((size + 7) // 8, dtype=np.uint64)
    x0, x1 = index & word, index >> np.uint64(32)
    x2, x3 = np.full_like(x0, s["offset"] & WORD), np.full_like(x0, s["offset"] >> 32)
    key = [s["seed"] & WORD, s["seed"] >> 32]
    for _ in range(10):
        left, right = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        x0, x1, x2, x3 = (right >> np.uint64(32)) ^ x1 ^ np.uint64(key[0]), right & word, (left >> np.uint64(32)) ^ x3 ^ np.uint64(key[1]), left & word
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    draws = np.empty((len(index), 4), "<u4")
    draws[:, 0], draws[:, 1], draws[:, 2], draws[:, 3] = x0, x1, x2, x3
    kept = round(65536 * (1 - c["p"]))
    keep = torch.from_numpy((draws.view("<u2").reshape(-1)[:size] < kept).reshape(c["rows"], c["n"])).cuda()
    out = s["x"].double() * keep * (65536 / kept if kept else 0.0)
    return {"out": out if s["add"] is None else out + s["add"].double()}


def _exact_mix(s, c):
    """Token by token: S <- decay S + k v^T, o = scale S^T q; and back again for the gradients."""
    B, T, P, H, dk, dv = (c[n] for n in ("B", "T", "P", "H", "dk", "dv"))
    wide = {n: s[n].double().repeat_interleave(H // s[n].shape[3], 3) for n in ("q", "k", "v")}
    q, k, v = wide["q"], wide["k"], wide["v"]
    decay = torch.exp(s["log_decay"].double())[:, None, None]
    live = [None] * T if s["lengths"] is None else [(t < s["lengths"]).view(B, 1, 1, 1, 1) for t in range(T)]
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    choose = lambda on, x, y: x if on is None else torch.where(on, x, y)  # noqa: E731
    first = lambda x: torch.zeros(B, P, H, dk, dv, dtype=torch.float64, device="cuda") if x is None else x.double()  # noqa: E731
    S, rows = first(s["state"]), []
    g = None if c["dir"] == "fwd" else s["g"].double() * s["scale"]
    for t in range(T):
        S = choose(live[t], torch.addcmul(decay * S, k[:, t, :, :, :, None], v[:, t, :, :, None, :]), S)
        if g is None:
            row = torch.matmul(q[:, t, :, :, None, :], S).squeeze(3) * s["scale"]
        else:
            row = torch.matmul(S, g[:, t, :, :, :, None]).squeeze(4)
        rows.append(choose(None if live[t] is None else live[t][..., 0], row, zero))
    if g is None:
        out = {"o": torch.stack(rows, 1)}
        return {**out, "state": S} if c["state"] else out
    gq, gk, gv = torch.stack(rows, 1), [], []
    G = first(s["g_state_out"])                                  # of the state behind token t
    for t in reversed(range(T)):
        now = torch.addcmul(G, q[:, t, :, :, :, None], g[:, t, :, :, None, :])
        on = None if live[t] is None else live[t][..., 0]
        gk.append(choose(on, torch.matmul(now, v[:, t, :, :, :, None]).squeeze(4), zero))
        gv.append(choose(on, torch.matmul(k[:, t, :, :, None, :], now).squeeze(3), zero))
        G = choose(live[t], decay * now, G)
    out = {"gq": gq, "gk": torch.stack(gk[::-1], 1), "gv": torch.stack(gv[::-1], 1)}
    out = {"g" + n: out["g" + n].unflatten(3, (s[n].shape[3], -1)).sum(4) for n in ("q", "k", "v")}
    return {**out, "g_state": G} if c["state"] else out
