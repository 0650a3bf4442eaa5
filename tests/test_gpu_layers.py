"""Layer norm, dropout and linear attention through the C ABI against the float64 oracle, at the sizes and masks where they can go wrong.

Tolerances (relative L2, and element by element by assert_close).  float32: sums of at most a few hundred terms and a decay whose
exponent is rounded once, each within some 2^-24 of its terms' sum: 1e-5 (layer norm with a mean of m standard deviations: m + 8 of
2^-23).  bfloat16 has 8 significant bits: every rounding moves a value by 2^-8 of it at most, 2^-8 / sqrt 3 in the root mean square; an
output of linear attention passes four (scores, decayed values, state, the output itself), so 2 x 2^-8 / sqrt 3 = 4.5e-3 is the most that is
expected and 2^-7 = 7.8e-3 asked for; what is rounded once has 2^-8; states are
float32 in both.  Element by element the bound is the largest element's times sqrt(2 ln 2n) of that (elementwise_factor)."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from paper_2207_08393_amd import binding as gb
from tests.gpu_util import assert_close

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
F32, ONCE, BF16 = 1e-5, 2.0 ** -8, 2.0 ** -7
POISON = float("nan")


def dev(a, dtype):
    """numpy -> device, and the values that the device has."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(dtype)
    return t, t.double().cpu().numpy()


def host(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def rows_array(rows, n, ld, dtype, fill=POISON, offset=0):
    """rows x n view with ld elements from row to row, `offset` elements behind an aligned address; and the whole storage."""
    store = torch.full((offset + rows * ld,), fill, dtype=dtype, device="cuda")
    return store[offset:].as_strided((rows, n), (ld, 1)), store


# ------------------------------------------------------------------------------------------------------------ layer norm
NORM = [(1, 1, 0, 0), (3, 1, 2, 1), (1, 7, 0, 0), (5, 2, 0, 0), (9, 8, 0, 0), (4, 13, 0, 1), (70, 16, 0, 0), (65, 17, 3, 3), (33, 64, 0, 0), (130, 100, 0, 0),
        (17, 129, 0, 0), (16, 250, 6, 0), (7, 511, 0, 0), (9, 1001, 0, 2), (5, 2048, 0, 0), (3, 4100, 4, 0), (4, 5001, 7, 0), (3, 8192, 0, 0), (2, 16384, 0, 0), (700, 12000, 0, 0), (5, 9001, 0, 1),
        (3, 16391, 1, 0), (2, 40003, 0, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,pad,offset", NORM)
def test_layer_norm(rows, n, pad, offset, dtype):
    print("case norm", rows, n, pad, offset, dtype, flush=True)
    T, rng = TYPES[dtype], np.random.default_rng(n + rows)
    x, xs = rows_array(rows, n, n + pad, T, offset=offset)
    g, _ = rows_array(rows, n, n + 2 * pad, T, offset=offset)
    x.copy_(torch.from_numpy(rng.normal(0.7, 1.4, (rows, n)).astype(np.float32)))
    g.copy_(torch.from_numpy(rng.normal(0.0, 1.0, (rows, n)).astype(np.float32)))
    gamma, hgamma = dev(1 + 0.2 * rng.normal(size=n), torch.float32)
    beta, hbeta = dev(0.3 * rng.normal(size=n), torch.float32)
    hx, hg, eps = host(x), host(g), 1e-3
    d = gb.make_layer_norm(T, rows, n, eps, ld=n + pad, ld_out=n + 2 * pad)
    y, ys = rows_array(rows, n, n + 2 * pad, T, offset=offset)
    mean, rstd = torch.full((rows,), POISON, device="cuda"), torch.full((rows,), POISON, device="cuda")
    gb.gleam_layer_norm_fwd(d, x, gamma, beta, y, mean, rstd)
    ry, rmean, rrstd = lo.layer_norm(hx, hgamma, hbeta, np.float32(eps))
    assert_close(host(y), ry, F32 + (ONCE if dtype == "bf16" else 0), "y")
    assert_close(host(mean), rmean, F32, "mean")
    assert_close(host(rstd), rrstd, F32, "rstd")
    assert int(torch.isnan(ys).sum()) == ys.numel() - rows * n                     # nothing between the rows was written
    ws = torch.empty(gb.gleam_layer_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    gx, gxs = rows_array(rows, n, n + pad, T, offset=offset)
    gg, gbt = torch.full((n,), POISON, device="cuda"), torch.full((n,), POISON, device="cuda")
    gb.gleam_layer_norm_bwd(d, x, gamma, mean, rstd, g, gx, gg, gbt, ws)
    rx, rg, rb = lo.layer_norm_bwd(hx, hgamma, host(mean), host(rstd), hg)
    # g_x is what is left of terms of the size of r gg: the bound is on those
    scale = float(np.abs(host(rstd)[:, None] * hg * hgamma).max())
    assert np.abs(host(gx) - rx).max() <= scale * (8 * F32 + (ONCE if dtype == "bf16" else 0))
    if n > 2:
        assert_close(host(gx), rx, 4 * F32 + (ONCE if dtype == "bf16" else 0), "g_x")
    assert_close(host(gg), rg, F32, "g_gamma") if np.abs(rg).max() > 1e-3 else None
    assert_close(host(gbt), rb, F32, "g_beta")
    assert int(torch.isnan(gxs).sum()) == gxs.numel() - rows * n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [100, 1001, 4500, 20011])
def test_layer_norm_in_place_and_without_parameters(n, dtype):
    print("case norm in place", n, dtype, flush=True)
    T, rng, rows = TYPES[dtype], np.random.default_rng(n), 37
    x, hx = dev(rng.normal(0.2, 1.0, (rows, n)), T)
    g, hg = dev(rng.normal(size=(rows, n)), T)
    d = gb.make_layer_norm(T, rows, n, 1e-5)
    one = torch.ones(n, device="cuda")
    y, m, r = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    gb.gleam_layer_norm_fwd(d, x, one, None, y, m, r)
    gx, again, ws = torch.empty_like(x), g.clone(), torch.empty(gb.gleam_layer_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    gg = torch.empty(n, device="cuda")
    gb.gleam_layer_norm_bwd(d, x, None, m, r, g, gx, gg, None, ws)
    gb.gleam_layer_norm_bwd(d, x, one, m, r, again, again, None, None, None)
    assert torch.equal(gx, again)
    assert_close(host(gx), lo.layer_norm_bwd(hx, None, host(m), host(r), hg)[0], 4 * F32 + (ONCE if dtype == "bf16" else 0), "g_x")
    gb.gleam_layer_norm_fwd(d, x, None, None, x)                                   # y takes the place of x
    assert torch.equal(x, y)


def test_layer_norm_of_a_large_mean_and_of_constant_rows():
    rng = np.random.default_rng(5)
    x, hx = dev(rng.normal(1000.0, 1.0, (40, 300)), torch.float32)
    x[3] = 7.0
    hx[3] = 7.0
    d = gb.make_layer_norm(torch.float32, 40, 300, 1e-5)
    y = torch.empty_like(x)
    gb.gleam_layer_norm_fwd(d, x, None, None, y)
    assert not host(y)[3].any()                                                    # the mean of equal numbers is that number
    # the mean is good to a few 2^-24 of 1000 standard deviations
    assert np.abs(host(y) - lo.layer_norm(hx, None, None, 1e-5)[0]).max() <= (1000 + 8) * 2.0 ** -22


def test_layer_norm_gradients_against_differences():
    rng = np.random.default_rng(6)
    rows, n, eps = 6, 45, 1e-3
    x, hx = dev(rng.normal(0.5, 1.0, (rows, n)), torch.float32)
    g, hg = dev(rng.normal(size=(rows, n)), torch.float32)
    gamma, hgamma = dev(1 + 0.2 * rng.normal(size=n), torch.float32)
    d = gb.make_layer_norm(torch.float32, rows, n, eps)
    y, m, r = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    gb.gleam_layer_norm_fwd(d, x, gamma, None, y, m, r)
    gx, ga, be = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ws = torch.empty(gb.gleam_layer_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    gb.gleam_layer_norm_bwd(d, x, gamma, m, r, g, gx, ga, be, ws)
    loss = lambda a, b, c: (lo.layer_norm(a, b, c, np.float32(eps))[0] * hg).sum()  # noqa: E731
    at, h = [hx, hgamma, np.zeros(n)], 1e-4
    for i, grad in enumerate((gx, ga, be)):
        e = rng.normal(size=at[i].shape)
        f = lambda z: loss(*(z if j == i else at[j] for j in range(3)))  # noqa: E731,B023
        assert abs((f(at[i] + h * e) - f(at[i] - h * e)) / (2 * h) - (host(grad) * e).sum()) <= 1e-5 * np.abs(host(grad) * e).sum()


# --------------------------------------------------------------------------------------------------------------- dropout
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n,pad,offset,p", [(1, 1, 0, 0, 0.5), (1, 7, 0, 0, 0.1), (1, 8, 0, 0, 0.1), (3, 5, 0, 0, 0.3), (3, 5, 2, 1, 0.3), (17, 100, 0, 0, 0.2),
                                                 (9, 64, 8, 0, 0.5), (5, 64, 1, 3, 0.9), (4, 33, 0, 1, 0.0), (4, 33, 0, 0, 1.0), (2, 1025, 0, 0, 0.05)])
def test_dropout(rows, n, pad, offset, p, dtype):
    print("case dropout", rows, n, pad, offset, p, dtype, flush=True)
    T, rng = TYPES[dtype], np.random.default_rng(rows * n)
    seed, c = 0xDEADBEEF12345678, 2 ** 33 + 5
    x, _ = rows_array(rows, n, n + pad, T, offset=offset)
    res, _ = rows_array(rows, n, n + 2 * pad, T, offset=offset)
    out, store = rows_array(rows, n, n + 3 * pad, T, offset=offset)
    x.copy_(torch.from_numpy(rng.normal(size=(rows, n)).astype(np.float32)))
    res.copy_(torch.from_numpy(rng.normal(size=(rows, n)).astype(np.float32)))
    mask, factor = lo.dropout_mask(rows, n, p, seed, c)
    if not mask.all():
        r, k = np.argwhere(~mask)[0]
        x[r, k] = float("inf")                                                     # what is dropped is not read into the result
        x[tuple(np.argwhere(~mask)[-1])] = POISON
    d = gb.make_dropout(T, rows, n, p, seed, c, ld=n + pad, ld_res=n + 2 * pad, ld_out=n + 3 * pad)
    want = np.where(mask, np.nan_to_num(host(x)) * factor, 0.0)
    gb.gleam_dropout_fwd(d, x, res, out)
    assert_close(host(out), want + host(res), 1e-6 + (ONCE if dtype == "bf16" else 0), "out")
    assert int(torch.isnan(store).sum()) == store.numel() - rows * n
    gb.gleam_dropout_fwd(d, x, None, out)
    assert_close(host(out), want, 1e-6 + (ONCE if dtype == "bf16" else 0), "out without a residual")
    assert np.array_equal(host(out) != 0, mask & (np.nan_to_num(host(x)) != 0))
    g, _ = rows_array(rows, n, n + 3 * pad, T, fill=1.0, offset=offset)
    gx, _ = rows_array(rows, n, n + pad, T, offset=offset)
    gb.gleam_dropout_bwd(d, g, gx)
    assert_close(host(gx), np.where(mask, factor, 0.0), 1e-6 + (ONCE if dtype == "bf16" else 0), "g_x")


def test_dropout_mask_does_not_depend_on_layout_and_moves_with_the_step():
    rows, n, p, seed = 300, 40, 0.4, 99
    x = torch.randn(rows, n, device="cuda")
    wide = torch.zeros(rows, n + 3, device="cuda")[:, :n].copy_(x)
    a, b, low = torch.empty_like(x), torch.empty_like(wide), torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    assert b.is_contiguous()
    gb.gleam_dropout_fwd(gb.make_dropout(torch.float32, rows, n, p, seed, 7), x, None, a)
    gb.gleam_dropout_fwd(gb.make_dropout(torch.float32, rows, n, p, seed, 7, ld=n + 3, ld_out=n), wide, None, b)
    gb.gleam_dropout_fwd(gb.make_dropout(torch.bfloat16, rows, n, p, seed, 7), x.bfloat16(), None, low)
    assert torch.equal(a, b) and torch.equal(a != 0, low != 0)
    step = torch.tensor([3], device="cuda")
    gb.gleam_dropout_fwd(gb.make_dropout(torch.float32, rows, n, p, seed, 4), x, None, b, step)
    assert torch.equal(a, b)
    gb.gleam_dropout_fwd(gb.make_dropout(torch.float32, rows, n, p, seed, 8), x, None, b)
    assert not torch.equal(a, b)
    y = x.clone()
    gb.gleam_dropout_fwd(gb.make_dropout(torch.float32, rows, n, p, seed, 7), y, None, y)   # in place
    assert torch.equal(a, y)


def test_dropout_counts_elements_past_32_bits():
    """The last row of an array of more than 2^32 elements: bfloat16, 8.6 GB; only its rows' ends are looked at."""
    rows, n = 70000, 61440
    assert rows * n > 2 ** 32
    x = torch.ones(rows, n, dtype=torch.bfloat16, device="cuda")
    d = gb.make_dropout(torch.bfloat16, rows, n, 0.5, 11, 1)
    gb.gleam_dropout_fwd(d, x, None, x)
    first = rows - 1
    mask, factor = lo.dropout_mask(1, 64, 0.5, 11, 1)
    assert np.array_equal(host(x[0, :64]), np.where(mask, factor, 0.0)[0])
    e = first * n
    want = [[h for w in lo.philox(((e // 8 + i) & 0xFFFFFFFF, (e // 8 + i) >> 32, 1, 0), (11, 0)) for h in (w & 0xFFFF, w >> 16)] for i in range(8)]
    assert np.array_equal(host(x[first, :64]), np.where(np.array(want).ravel() < 32768, 2.0, 0.0))


# ------------------------------------------------------------------------------------------------------ linear attention
def strided(shape, layout, T, offset=0):
    """A poisoned [B][T][P][h][d] array: 'tokens' row-major, 'heads' [B][h][T][P][d], 'gaps' with unused elements around every axis."""
    B, t, P, h, d = shape
    if layout == "heads":
        return torch.full((B, h, t, P, d), POISON, dtype=T, device="cuda").permute(0, 2, 3, 1, 4)
    if layout == "gaps":
        store = torch.full((offset + B * (t + 1) * (P + 1) * (h + 1) * (d + 3),), POISON, dtype=T, device="cuda")
        return store[offset:].as_strided(shape, ((t + 1) * (P + 1) * (h + 1) * (d + 3), (P + 1) * (h + 1) * (d + 3), (h + 1) * (d + 3), d + 3, 1))
    return torch.full(shape, POISON, dtype=T, device="cuda")


class Mix:
    """One layer's arrays on the device and their values on the host; tokens behind the sequences' ends are NaN or infinite."""

    def __init__(self, B, T, P, heads, dk, dv, dtype, layout="tokens", lengths=None, state=True, seed=0, decays=None):
        H, Hq, Hk, Hv = heads
        self.T, rng = TYPES[dtype], np.random.default_rng(seed + T + 31 * dk)
        self.scale, self.layout = dk ** -0.5, layout
        a = decays if decays is not None else np.log1p(-np.exp2(-rng.uniform(0.3, 8.0, H)))
        self.log_decay, self.ha = dev(a, torch.float32)
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.hl = lengths
        live = np.arange(T)[None, :] < (np.full(B, T) if lengths is None else np.array(lengths))[:, None]
        self.arrays, self.host = {}, {}
        for name, h, d in (("q", Hq, dk), ("k", Hk, dk), ("v", Hv, dv), ("g", H, dv)):
            x = strided((B, T, P, h, d), layout, self.T, offset=1 if layout == "gaps" else 0)
            val = np.where(live[:, :, None, None, None], rng.normal(size=x.shape), rng.choice([np.nan, np.inf, -np.inf], size=x.shape))
            x.copy_(torch.from_numpy(val.astype(np.float32)))
            self.arrays[name], self.host[name] = x, host(x)
        shape = (B, P, H, dk, dv)
        self.state, self.hs = dev(rng.normal(size=shape), torch.float32) if state else (None, None)
        self.gstate, self.hgs = dev(rng.normal(size=shape), torch.float32) if state else (None, None)
        self.shape, self.state_shape = (B, T, P, H, dv), shape
        self.low = dtype == "bf16"

    def new(self, name):
        return strided(self.arrays[name].shape, self.layout, self.T, offset=1 if self.layout == "gaps" else 0)

    def fwd(self, state_out=True):
        o = self.new("g")
        d = gb.make_linattn(self.arrays["q"], self.arrays["k"], self.arrays["v"], o, self.scale)
        n = gb.gleam_linattn_workspace_bytes(d)[0]
        out = torch.full(self.state_shape, POISON, device="cuda") if state_out else None   # None: not wanted
        gb.gleam_linattn_fwd(d, self.arrays["q"], self.arrays["k"], self.arrays["v"], self.log_decay, self.lengths, self.state, o, out,
                             torch.full((n,), 255, dtype=torch.uint8, device="cuda"))
        return o, out

    def bwd(self, g_state=True):
        a = self.arrays
        d = gb.make_linattn(a["q"], a["k"], a["v"], a["g"], self.scale)
        n = gb.gleam_linattn_workspace_bytes(d)[1]
        grads = [self.new(x) for x in "qkv"]
        gs = torch.full(self.state_shape, POISON, device="cuda") if g_state else None
        gb.gleam_linattn_bwd(d, a["q"], a["k"], a["v"], self.log_decay, self.lengths, self.state, a["g"], self.gstate, *grads, gs,
                             torch.full((n,), 255, dtype=torch.uint8, device="cuda"))
        return grads, gs

    def check(self):
        tol = BF16 if self.low else F32
        h = self.host
        states = self.state is not None
        o, S = self.fwd(states)
        ro, rS = lo.linattn(h["q"], h["k"], h["v"], self.ha, self.scale, self.hl, self.hs)
        assert_close(host(o), ro, tol, "o")
        if states:
            assert_close(host(S), rS, F32, "state")
        grads, gS = self.bwd(states)
        ref = lo.linattn_bwd(h["q"], h["k"], h["v"], self.ha, self.scale, h["g"], self.hl, self.hs, self.hgs)
        for name, got, want in zip(("g_q", "g_k", "g_v"), grads, ref):
            assert_close(host(got), want, tol, name)
        if states:
            assert_close(host(gS), ref[3], F32, "g_state")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 129, 257])
def test_linattn_lengths(T, dtype):
    print("case linattn", T, dtype, flush=True)
    Mix(2, T, 1, (2, 2, 2, 2), 32, 32, dtype).check()
    Mix(1, T, 3, (1, 1, 1, 1), 64, 48, dtype, state=False).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(1, 1), (3, 2), (8, 8), (16, 16), (25, 25), (33, 7), (7, 33), (40, 72), (64, 64), (96, 80), (65, 128), (128, 64), (127, 127), (128, 128)])
def test_linattn_widths(dk, dv, dtype):
    print("case linattn widths", dk, dv, dtype, flush=True)
    Mix(1, 70, 2, (3, 3, 3, 3), dk, dv, dtype).check()
    Mix(2, 1, 2, (3, 3, 3, 3), dk, dv, dtype).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["tokens", "heads", "gaps"])
@pytest.mark.parametrize("heads", [(6, 6, 6, 6), (6, 6, 2, 2), (6, 1, 1, 6), (6, 3, 2, 1)])
def test_linattn_heads_and_layouts(heads, layout, dtype):
    print("case linattn heads", heads, layout, dtype, flush=True)
    Mix(2, 40, 2, heads, 20, 36, dtype, layout, lengths=[40, 13]).check()
    Mix(2, 1, 2, heads, 20, 36, dtype, layout, lengths=[0, 1]).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("state", [True, False])
@pytest.mark.parametrize("T,lengths", [(1, [0, 1, 1, 0, 1]), (70, [0, 1, 64, 65, 70]), (20, [20, 0, 0, 16, 17]), (700, [700, 0, 257, 513, 384])])
def test_linattn_ragged(T, lengths, state, dtype):
    """Empty sequences among others, ends on, before and behind the borders of chunks and segments; NaN and infinities behind the ends."""
    print("case linattn ragged", T, lengths, state, dtype, flush=True)
    Mix(5, T, 1, (2, 2, 2, 2), 32, 24, dtype, lengths=lengths, state=state).check()
    Mix(5, T, 1, (1, 1, 1, 1), 72, 40, dtype, lengths=lengths, state=state).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["tokens", "gaps"])
@pytest.mark.parametrize("dk,dv", [(16, 16), (8, 8), (5, 3), (25, 25), (24, 8), (12, 30), (32, 32)])
def test_linattn_short_sequences_of_narrow_heads(dk, dv, layout, dtype):
    """Few tokens at many pixels, no state: the tokens of one, two and four tiles, and their ends."""
    for T in (2, 7, 16, 17, 20, 32, 33, 50, 64):
        print("case linattn short", dk, dv, layout, T, dtype, flush=True)
        Mix(1, T, 5, (3, 3, 3, 3), dk, dv, dtype, layout, state=False).check()
        Mix(3, T, 3, (4, 2, 1, 4), dk, dv, dtype, layout, lengths=[T, 0, T // 2], state=False).check()
        Mix(3, T, 2, (8, 8, 8, 8), dk, dv, dtype, layout, lengths=[T, 0, T // 2], state=False).check()


def test_linattn_short_sequences_without_memory():
    Mix(1, 20, 2, (3, 3, 3, 3), 16, 16, "f32", state=False, decays=[-np.inf, -300.0, 0.0]).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_linattn_long(d, dtype):
    """Few problems of many chunks: the split into segments; a state in and out, heads shared, one sequence shorter."""
    print("case linattn long", d, dtype, flush=True)
    m = Mix(2, 1500, 1, (2, 2, 1, 1), d, d, dtype, lengths=[1500, 1111])
    desc = gb.make_linattn(m.arrays["q"], m.arrays["k"], m.arrays["v"], m.arrays["g"], m.scale)
    assert gb.gleam_linattn_workspace_bytes(desc)[0] > 0                           # there are segments
    m.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linattn_decays(dtype):
    """No decay, decays beyond the range of a float32 within a chunk, and none of the past at all."""
    print("case linattn decays", dtype, flush=True)
    Mix(1, 150, 1, (6, 6, 6, 6), 16, 16, dtype, decays=[0.0, -1e-6, -0.5, -5.0, -200.0, -np.inf]).check()
    Mix(1, 1, 1, (2, 2, 2, 2), 16, 16, dtype, decays=[-np.inf, 0.0]).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linattn_pieces_are_the_whole(dtype):
    """A sequence in one call, in two with the state handed over, and its last tokens one by one, the state updated in place."""
    print("case linattn pieces", dtype, flush=True)
    m = Mix(1, 90, 2, (2, 2, 2, 2), 48, 32, dtype)
    a, (o, S) = m.arrays, m.fwd()
    part, run = torch.full_like(o, POISON), m.state.clone()
    for lo_, hi in [(0, 50), (50, 85)] + [(t, t + 1) for t in range(85, 90)]:
        x = [a[n][:, lo_:hi] for n in "qkv"]
        d = gb.make_linattn(*x, part[:, lo_:hi], m.scale)
        gb.gleam_linattn_fwd(d, *x, m.log_decay, None, run, part[:, lo_:hi], run, torch.empty(gb.gleam_linattn_workspace_bytes(d)[0], dtype=torch.uint8, device="cuda"))
    assert_close(host(part), host(o), BF16 if m.low else F32, "o")
    assert_close(host(run), host(S), F32, "state")


@pytest.mark.parametrize("T", [1, 30, 400])
def test_linattn_lengths_out_of_range_count_as_the_nearest(T):
    for state in (True, False):
        Mix(3, T, 1, (2, 2, 2, 2), 24, 16, "f32", lengths=[T + 5, -3, 2 ** 31 - 1], state=state).check()


def test_linattn_description_that_changes():
    """A description whose fields are changed is compared with the arrays anew."""
    q = torch.randn(1, 6, 1, 2, 8, device="cuda")
    o, a = torch.empty_like(q), torch.zeros(2, device="cuda")
    d = gb.make_linattn(q, q, q, o, 1.0)
    gb.gleam_linattn_fwd(d, q, q, q, a, None, None, o, None, None)
    d.T = 60
    with pytest.raises(ValueError):
        gb.gleam_linattn_fwd(d, q, q, q, a, None, None, o, None, None)


def test_linattn_state_out_of_nothing():
    """A state behind the last token is wanted, none comes in."""
    for dtype in ("f32", "bf16"):
        m = Mix(2, 90, 1, (2, 2, 2, 2), 24, 16, dtype, lengths=[90, 0], state=False)
        _, S = m.fwd()
        assert_close(host(S), lo.linattn(m.host["q"], m.host["k"], m.host["v"], m.ha, m.scale, m.hl)[1], F32, "state")
        gS = m.bwd()[1]
        assert_close(host(gS), lo.linattn_bwd(m.host["q"], m.host["k"], m.host["v"], m.ha, m.scale, m.host["g"], m.hl)[3], F32, "g_state")


def test_linattn_gradients_against_differences():
    """Differences of the float64 forward pass at the library's inputs along a direction, against the library's gradients."""
    m = Mix(2, 40, 1, (2, 2, 1, 2), 12, 20, "f32", lengths=[40, 23])
    grads, gS = m.bwd()
    rng = np.random.default_rng(8)
    zero = {n: np.where(np.isfinite(x), x, 0.0) for n, x in m.host.items()}
    g = zero["g"]

    def loss(q, k, v, S0):
        o, S = lo.linattn(q, k, v, m.ha, m.scale, m.hl, S0)
        return (o * g).sum() + (S * m.hgs).sum()

    at, h = [zero["q"], zero["k"], zero["v"], m.hs], 1e-4
    for i, grad in enumerate((*grads, gS)):
        e = rng.normal(size=at[i].shape)
        f = lambda z: loss(*(z if j == i else at[j] for j in range(4)))  # noqa: E731,B023
        assert abs((f(at[i] + h * e) - f(at[i] - h * e)) / (2 * h) - (host(grad) * e).sum()) <= 1e-5 * np.abs(host(grad) * e).sum()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linattn_twice_is_the_same_bits_and_on_another_stream(dtype):
    m = Mix(1, 1200, 1, (4, 4, 2, 2), 64, 64, dtype)
    (o, S), (grads, gS) = m.fwd(), m.bwd()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        (o2, S2), (grads2, gS2) = m.fwd(), m.bwd()
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(S, S2) and torch.equal(gS, gS2) and all(torch.equal(x, y) for x, y in zip(grads, grads2))


def test_linattn_offsets_past_32_bits():
    """A stride that puts the last tokens more than 2^32 bytes behind the first ones, and more than 2^31 elements."""
    T, d, stride = 70, 16, 34_000_000
    store = torch.zeros(T * stride, dtype=torch.bfloat16, device="cuda")
    assert (T - 1) * stride > 2 ** 31
    rng = np.random.default_rng(9)
    q = store.as_strided((1, T, 1, 1, d), (0, stride, 0, 0, 1))
    k, v = (store[n * d:].as_strided((1, T, 1, 1, d), (0, stride, 0, 0, 1)) for n in (1, 2))
    for x in (q, k, v):
        x.copy_(torch.from_numpy(rng.normal(size=(1, T, 1, 1, d)).astype(np.float32)))
    o = torch.empty(1, T, 1, 1, d, dtype=torch.bfloat16, device="cuda")
    a = torch.tensor([-0.01], device="cuda")
    desc = gb.make_linattn(q, k, v, o, 1.0)
    gb.gleam_linattn_fwd(desc, q, k, v, a, None, None, o, None, None)
    assert_close(host(o), lo.linattn(host(q), host(k), host(v), host(a), 1.0)[0], BF16, "o")


def test_captured_calls_replay_as_the_eager_ones():
    """Layer norm, linear attention in segments, its gradients and dropout in one graph, replayed with other inputs and another step each
    time, eager work in between."""
    B, T, P, H, d = 1, 700, 1, 2, 32
    rows, C = B * T * P, H * d
    x = torch.randn(rows, C, device="cuda").bfloat16()
    gamma, beta, a = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda"), torch.tensor([-0.1, -0.01], device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    norm, drop = gb.make_layer_norm(torch.bfloat16, rows, C), gb.make_dropout(torch.bfloat16, rows, C, 0.3, 5)
    y, o, h = torch.empty_like(x), torch.empty_like(x).view(B, T, P, H, d), torch.empty_like(x)
    q = y.view(B, T, P, H, d)
    grads = [torch.empty_like(q) for _ in range(3)]
    mix = gb.make_linattn(q, q, q, o, 0.2)
    fwd, bwd = gb.gleam_linattn_workspace_bytes(mix)
    assert fwd > 0
    ws = torch.empty(max(fwd, bwd), dtype=torch.uint8, device="cuda")

    def calls():
        gb.gleam_layer_norm_fwd(norm, x, gamma, beta, y)
        gb.gleam_linattn_fwd(mix, q, q, q, a, None, None, o, None, ws)
        gb.gleam_linattn_bwd(mix, q, q, q, a, None, None, o, None, *grads, None, ws)
        gb.gleam_dropout_fwd(drop, o.view(rows, C), x, h, step)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    masks = []
    for k in range(4):
        x.copy_(torch.randn(rows, C, device="cuda"))
        step.fill_(k)
        graph.replay()
        got = [t.clone() for t in (y, o, h, *grads)]
        torch.cuda.synchronize()
        calls()
        assert all(torch.equal(g, t) for g, t in zip(got, (y, o, h, *grads)))
        masks.append((h - x == 0).sum().item())
    assert len(set(masks)) > 1                                                     # another mask at every step
