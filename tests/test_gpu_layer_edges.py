"""Rows, tokens and sizes at which the sequence-layer operators could go wrong: against the float64 oracle, or exactly.

Tolerances are those of the operators' other parity tests, derived the same way.  Layer norm: the mean is a sum of n terms x / n
and a second one of what that left over; with at most 38 additions in a row (16 a lane, 6 in a wave, 16 waves) each within 2^-24 of
the sum of magnitudes, itself at most twice the mean of |x| here, its error is below 38 x 2^-23 = 4.5e-6 of that; F32 = 1e-5."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from paper_2207_08393_amd import binding as gb
from tests.gpu_util import assert_close

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
F32, ONCE = 1e-5, 2.0 ** -8
POISON = float("nan")


def dev(a, dtype):
    """numpy -> device, and the values that the device has."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(dtype)
    return t, t.double().cpu().numpy()


def host(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


# ------------------------------------------------------------------------------------------------------------ layer norm
def norm_fwd(x, gamma=None, beta=None, eps=1e-5):
    rows, n = x.shape
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    gb.gleam_layer_norm_fwd(gb.make_layer_norm(x.dtype, rows, n, eps), x, gamma, beta, y, mean, rstd)
    return y, mean, rstd


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,size", [(13, 1e3), (100, 1e3), (129, 1e3), (1024, 1e3), (4096, 1e4), (5001, 1e4), (16384, 1e4), (20011, 1e4)])
def test_layer_norm_of_rows_whose_first_element_is_unlike_the_others(n, size, dtype):
    """One channel much larger than the others, the first one or the last: the others' outputs and the mean are as good as elsewhere."""
    print("case norm outlier", n, size, dtype, flush=True)
    rng = np.random.default_rng(n)
    a = rng.normal(0.3, 1.0, (6, n))
    a[:3, 0] = size * np.array([1.0, -1.0, 3.0])
    a[3:, -1] = size * np.array([1.0, -1.0, 3.0])
    x, hx = dev(a, TYPES[dtype])
    y, mean, rstd = norm_fwd(x)
    ry, rmean, rrstd = lo.layer_norm(hx, None, None, np.float32(1e-5))
    once = ONCE if dtype == "bf16" else 0.0
    for r in range(6):
        assert abs(host(mean)[r] - rmean[r]) <= F32 * np.abs(hx[r]).mean(), (r, host(mean)[r], rmean[r])
        others = slice(1, n) if r < 3 else slice(0, n - 1)
        assert_close(host(y)[r, others], ry[r, others], F32 + once, f"row {r}")
    assert_close(host(rstd), rrstd, F32, "rstd")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [2, 13, 100, 129, 1024, 5001, 9001, 20011])
def test_layer_norm_of_rows_that_begin_with_the_lowest_value(n, dtype):
    """The variance passes the range of a float32: r = 0 and outputs are beta, as 32-bit arithmetic has it, and not NaN."""
    print("case norm lowest", n, dtype, flush=True)
    rng = np.random.default_rng(n)
    x = torch.from_numpy(rng.normal(size=(5, n)).astype(np.float32)).cuda().to(TYPES[dtype])
    low = torch.finfo(TYPES[dtype]).min
    x[0, 0], x[1, -1], x[2, n // 2], x[3, 0] = low, low, low, -low
    beta, hbeta = dev(rng.normal(size=n), torch.float32)
    y, mean, rstd = norm_fwd(x, None, beta)
    want = hbeta if dtype == "f32" else host(beta.bfloat16())
    for r in range(4):
        assert np.array_equal(host(y)[r], want), r
    assert_close(host(mean)[:4], host(x)[:4].mean(1), F32, "mean")
    assert not host(rstd)[:4].any()
    assert_close(host(y)[4:], lo.layer_norm(host(x)[4:], None, hbeta, 1e-5)[0], F32 + (ONCE if dtype == "bf16" else 0.0), "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 13, 100, 300, 1001, 5001, 12000, 20011])
def test_layer_norm_of_constant_rows(n, dtype):
    """The mean of equal numbers is that number, bit by bit."""
    a = torch.tensor([7.0, 0.1, -3.3e4, 1e-20, 1e30, 0.0, -3e38], device="cuda")
    x = a[:, None].repeat(1, n).to(TYPES[dtype])
    y, mean, rstd = norm_fwd(x)
    assert not host(y).any()
    assert np.array_equal(host(mean), host(x)[:, 0])
    assert_close(host(rstd), np.full(len(a), 1e-5 ** -0.5), F32, "rstd")


@pytest.mark.parametrize("n", [13, 100, 5001, 20011])
def test_layer_norm_of_rows_with_infinities_and_nan(n):
    """A row that holds an infinity or NaN becomes NaN; its neighbours stay as they are."""
    x, hx = dev(np.random.default_rng(n).normal(size=(7, n)), torch.float32)
    y0 = norm_fwd(x)[0]
    x[1, 0], x[3, -1], x[5, n // 2] = float("inf"), POISON, -float("inf")
    y, mean, _ = norm_fwd(x)
    assert np.isnan(host(y)[1::2]).all() and torch.equal(y[::2], y0[::2])
    assert host(mean)[1] == np.inf and np.isnan(host(mean)[3]) and host(mean)[5] == -np.inf


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(1, 13), (5, 16), (37, 100), (3, 129), (1030, 64), (5, 5001), (3, 20011)])
def test_layer_norm_gradients_of_infinities(rows, n, dtype):
    """An infinite gradient, in the last row too (where lanes without a row of their own must not count): sums over rows are infinite in
    its column and as they were in the others; the gradients of other rows are what they were."""
    print("case norm gradient infinity", rows, n, dtype, flush=True)
    T, rng = TYPES[dtype], np.random.default_rng(rows + n)
    x, hx = dev(rng.normal(size=(rows, n)), T)
    g, hg = dev(rng.normal(size=(rows, n)), T)
    d = gb.make_layer_norm(T, rows, n, 1e-5)
    _, mean, rstd = norm_fwd(x)
    ws = torch.empty(gb.gleam_layer_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")

    def gradients(g):
        gx, gg, gbt = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        gb.gleam_layer_norm_bwd(d, x, None, mean, rstd, g, gx, gg, gbt, ws)
        return gx, gg, gbt

    gx0, gg0, gb0 = gradients(g)
    g[-1, n - 1] = float("inf")
    gx, gg, gbt = gradients(g)
    xh = (hx[-1, n - 1] - host(mean)[-1]) * host(rstd)[-1]
    assert host(gbt)[-1] == np.inf and host(gg)[-1] == np.sign(xh) * np.inf
    assert torch.equal(gbt[:-1], gb0[:-1]) and torch.equal(gg[:-1], gg0[:-1]) and torch.equal(gx[:-1], gx0[:-1])
    assert not np.isfinite(host(gx)[-1]).any()


# ------------------------------------------------------------------------------------------------------ linear attention
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(4, 4, 4, 4), (3, 3, 3, 3), (4, 2, 1, 4)])
@pytest.mark.parametrize("dk,dv", [(16, 16), (5, 3), (25, 25), (32, 24), (40, 40)])
@pytest.mark.parametrize("T", [1, 2, 17, 40, 64, 100])
def test_linattn_zeros_behind_the_ends_whatever_the_tokens_hold(T, dk, dv, heads, dtype):
    """Infinities and NaN in tokens that are there: outputs and gradients behind the sequences' ends are zeros all the same, with a state
    and without one."""
    print("case linattn dead tokens", T, dk, dv, heads, dtype, flush=True)
    H, Hq, Hk, Hv = heads
    B, P, rng = 4, 2, np.random.default_rng(T + dk)
    lengths = [T, T // 2, 0, max(T - 1, 0)]
    live = np.arange(T)[None, :] < np.array(lengths)[:, None]
    T_ = TYPES[dtype]
    arrays = {}
    for name, h, d in (("q", Hq, dk), ("k", Hk, dk), ("v", Hv, dv), ("g", H, dv)):
        a = rng.normal(size=(B, T, P, h, d))
        bad = rng.random(size=a.shape) < 0.2
        a[bad] = rng.choice([np.nan, np.inf, -np.inf], size=int(bad.sum()))
        arrays[name] = dev(a, T_)[0]
    log_decay = torch.full((H,), -0.1, device="cuda")
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    desc = gb.make_linattn(arrays["q"], arrays["k"], arrays["v"], arrays["g"], 1.0)
    ws = torch.empty(max(gb.gleam_linattn_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
    for state in (None, torch.zeros(B, P, H, dk, dv, device="cuda")):
        o = torch.full_like(arrays["g"], POISON)
        gb.gleam_linattn_fwd(desc, arrays["q"], arrays["k"], arrays["v"], log_decay, n, state, o, None, ws)
        grads = [torch.full_like(arrays[x], POISON) for x in "qkv"]
        gb.gleam_linattn_bwd(desc, arrays["q"], arrays["k"], arrays["v"], log_decay, n, state, arrays["g"], None, *grads, None, ws)
        for name, t in zip(("o", "g_q", "g_k", "g_v"), (o, *grads)):
            assert not host(t)[~live].any(), name


# ------------------------------------------------------------- calls of more work-items than a grid's dimension holds (2^32)
def room_for(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < (gigabytes + 8) * 2 ** 30:
        pytest.skip(f"{gigabytes} GiB of GPU memory are not free")


def test_dropout_of_more_than_2_35_elements():
    """Eight elements a work-item: 33 x 2^30 of them, bfloat16 in place; 64 elements are looked at where the mask's counters, the grid's
    dimensions and the array begin and end."""
    room_for(67)
    rows, n = 33, 2 ** 30
    x = torch.ones(rows, n, dtype=torch.bfloat16, device="cuda")
    gb.gleam_dropout_fwd(gb.make_dropout(torch.bfloat16, rows, n, 0.5, 11, 1), x, None, x)
    for e in (0, 2 ** 32 - 32, 2 ** 35 - 32, 2 ** 35, rows * n - 64):
        mask, factor = lo.dropout_mask(1, 64, 0.5, 11, 1, first_row=e // 64) if e % 64 == 0 else (None, None)
        if mask is None:                              # half of it before the border
            both = [lo.dropout_mask(1, 64, 0.5, 11, 1, first_row=(e - 32) // 64 + i) for i in range(2)]
            mask, factor = np.concatenate([both[0][0][:, 32:], both[1][0][:, :32]], 1), both[0][1]
        assert np.array_equal(host(x.view(-1)[e:e + 64]), np.where(mask, factor, 0.0)[0]), e
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,rows", [("bf16", 2 ** 22 + 5)])
def test_layer_norm_of_more_than_2_22_long_rows(dtype, rows):
    """A workgroup of 1024 for each row, in place; every row is the same, so every result has to be."""
    n = 16385
    room_for(rows * n * 2 / 2 ** 30)
    base = torch.randn(n, generator=torch.Generator().manual_seed(1)).cuda().to(TYPES[dtype])
    want = norm_fwd(base[None])[0][0]
    x = base.expand(rows, n).contiguous()
    gb.gleam_layer_norm_fwd(gb.make_layer_norm(x.dtype, rows, n, 1e-5), x, None, None, x)
    for r in (0, 2 ** 21 - 3, 2 ** 21, 2 ** 22 - 3, 2 ** 22, rows - 3, *np.random.default_rng(0).integers(0, rows - 3, 50).tolist()):
        assert bool((x[r:r + 3] == want).all()), r
    del x
    torch.cuda.empty_cache()


def test_layer_norm_gradients_of_more_than_2_21_long_rows():
    rows, n = 2 ** 21 + 5, 16385
    room_for(2 * rows * n * 2 / 2 ** 30)
    gen = torch.Generator().manual_seed(1)
    base, gbase = (torch.randn(n, generator=gen).cuda().bfloat16() for _ in range(2))
    _, m, r = norm_fwd(base[None])
    want = torch.empty(1, n, dtype=torch.bfloat16, device="cuda")
    gb.gleam_layer_norm_bwd(gb.make_layer_norm(torch.bfloat16, 1, n, 1e-5), base[None], None, m, r, gbase[None], want, None, None, None)
    x, g = base.expand(rows, n).contiguous(), gbase.expand(rows, n).contiguous()
    gb.gleam_layer_norm_bwd(gb.make_layer_norm(torch.bfloat16, rows, n, 1e-5), x, None, m.repeat(rows), r.repeat(rows), g, g, None, None, None)
    for k in (0, 2 ** 21 - 3, 2 ** 21, rows - 3, *np.random.default_rng(0).integers(0, rows - 3, 50).tolist()):
        assert bool((g[k:k + 3] == want).all()), k
    del x, g
    torch.cuda.empty_cache()


def test_layer_norm_parameter_gradients_of_rows_of_more_than_2_26():
    """The sum over rows, 1024 work-items for 32 columns of both gradients."""
    rows, n = 2, 2 ** 26 + 35
    room_for(8)
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, g = (torch.randn(rows, n, device="cuda", generator=gen) for _ in range(2))
    mean, rstd = torch.tensor([0.1, -0.2], device="cuda"), torch.tensor([1.3, 0.7], device="cuda")
    d = gb.make_layer_norm(torch.float32, rows, n, 1e-5)
    gx, gg, gbt = torch.empty_like(x), torch.full((n,), POISON, device="cuda"), torch.full((n,), POISON, device="cuda")
    gb.gleam_layer_norm_bwd(d, x, None, mean, rstd, g, gx, gg, gbt, torch.empty(gb.gleam_layer_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    assert torch.equal(gbt, g[0] + g[1])                                           # one rounding, and that is the same one
    for c in (slice(0, 4096), slice(2 ** 25 - 4096, 2 ** 25 + 4096), slice(n - 4096, n)):
        xh = (host(x[:, c]) - host(mean)[:, None]) * host(rstd)[:, None]
        assert_close(host(gg[c]), (host(g[:, c]) * xh).sum(0), F32, "g_gamma")


class ManyProblems:
    """B = 1 sequence of T tokens at P pixels; results are compared with the oracle at pixels where the grid's dimensions, and the arrays,
    begin and end, and everything has to be written."""

    def __init__(self, T, P, heads, dk, dv, dtype, state=False, most=0):
        print("case linattn many problems", T, P, heads, dk, dv, dtype, state, flush=True)
        H, Hq, Hk, Hv = heads
        assert P * H > most
        gen = torch.Generator(device="cuda").manual_seed(T + dk)
        make = lambda h, d: torch.empty(1, T, P, h, d, dtype=TYPES[dtype], device="cuda").normal_(generator=gen)  # noqa: E731
        self.a = {"q": make(Hq, dk), "k": make(Hk, dk), "v": make(Hv, dv), "g": make(H, dv)}
        self.log_decay = torch.linspace(-0.5, -0.1, H, device="cuda")
        self.state, self.g_state = (torch.empty(1, P, H, dk, dv, device="cuda").normal_(generator=gen) if state else None for _ in range(2))
        self.P, self.low = P, dtype == "bf16"
        self.desc = gb.make_linattn(*(self.a[n] for n in "qkvg"), 0.5)
        self.ws = gb.gleam_linattn_workspace_bytes(self.desc)

    def check(self, ref, got, names):
        edges = sorted({0, self.P - 40, *(min(e, self.P - 40) for e in (2 ** 20 - 20, 2 ** 21 - 20, 2 ** 22 - 20, 2 ** 23 - 20, 2 ** 24 - 20, 2 ** 27 - 20))})
        for e in edges:
            s = slice(e, e + 40)
            want = ref(*(host(self.a[n][:, :, s]) for n in "qkvg"), *(None if x is None else host(x[:, s]) for x in (self.state, self.g_state)))
            for name, t, w in zip(names, got, want):
                if t is not None:
                    states = name.endswith("state")
                    assert_close(host(t[:, s] if states else t[:, :, s]), w, F32 if states or not self.low else 2.0 ** -7, (name, e))
        assert not any(bool(torch.isnan(t).any()) for t in got if t is not None)

    def fwd(self):
        o = torch.full_like(self.a["g"], POISON)
        S = None if self.state is None else torch.full_like(self.state, POISON)
        gb.gleam_linattn_fwd(self.desc, *(self.a[n] for n in "qkv"), self.log_decay, None, self.state, o, S,
                             torch.empty(self.ws[0], dtype=torch.uint8, device="cuda"))
        self.check(lambda q, k, v, g, S0, gS: lo.linattn(q, k, v, host(self.log_decay), 0.5, None, S0), (o, S), ("o", "state"))

    def bwd(self):
        grads = [torch.full_like(self.a[n], POISON) for n in "qkv"]
        gS = None if self.state is None else torch.full_like(self.state, POISON)
        gb.gleam_linattn_bwd(self.desc, *(self.a[n] for n in "qkv"), self.log_decay, None, self.state, self.a["g"], self.g_state, *grads, gS,
                             torch.empty(self.ws[1], dtype=torch.uint8, device="cuda"))
        self.check(lambda q, k, v, g, S0, gS: lo.linattn_bwd(q, k, v, host(self.log_decay), 0.5, g, None, S0, gS), (*grads, gS), ("g_q", "g_k", "g_v", "g_state"))


def test_linattn_single_tokens_of_more_than_2_26_problems():
    """A wave each; and of 2^24, a workgroup each."""
    room_for(14)
    ManyProblems(1, 2 ** 24 + 50, (4, 4, 4, 4), 1, 1, "bf16", state=True, most=2 ** 26).fwd()
    ManyProblems(1, 2 ** 22 + 50, (4, 4, 4, 4), 128, 20, "bf16", most=2 ** 24).fwd()
    torch.cuda.empty_cache()


def test_linattn_short_sequences_of_more_than_2_26_problems():
    room_for(32)
    m = ManyProblems(2, 2 ** 24 + 50, (4, 4, 4, 4), 8, 8, "bf16", most=2 ** 26)       # four heads as whole rows
    m.fwd()
    m.bwd()
    del m
    m = ManyProblems(2, 2 ** 24 + 50, (4, 4, 4, 4), 1, 1, "f32", most=2 ** 26)
    m.fwd()
    m.bwd()
    torch.cuda.empty_cache()


def test_linattn_chunks_of_more_problems_than_one_launch_dimension_holds():
    """Four waves for four problems, three passes in the backward call: 2^32 work-items at 22.4 million problems."""
    room_for(8)
    m = ManyProblems(2, 2 ** 24 + 50, (4, 4, 4, 4), 1, 1, "bf16", state=True, most=2 ** 26)
    m.fwd()
    m.bwd()
    torch.cuda.empty_cache()


def test_linattn_gradients_of_more_than_2_29_shared_values():
    """The sum over shared heads, a value a work-item."""
    room_for(40)
    ManyProblems(4, 2 ** 27 + 50, (2, 2, 1, 2), 1, 1, "bf16", most=2 ** 28).bwd()
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------- walks over more rows than teams
def norm64(x, gamma, beta, eps):
    """The same in 64 bits on the device, row by row in blocks."""
    x = x.double()
    mean = x.mean(1)
    rstd = 1.0 / torch.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma.double() + beta.double(), mean, rstd


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(2 * 524288 + 37, 8), (524288 + 37, 16), (2 * 65536 + 5, 100), (65536 + 3, 250), (32768 + 3, 512), (2 * 32768 + 1, 700), (16384 + 7, 1000),
                                    (8192 + 3, 1500), (2 * 8192 + 1, 4000), (8192 + 5, 5001), (8192 + 1, 8000), (8192 + 3, 12000), (8192 + 1, 16001)])
def test_layer_norm_of_more_rows_than_teams(rows, n, dtype):
    """Rows behind the first of a team, with a remainder: the row on its way, the sums over rows, in place.  Sums over rows are of at most 80
    partial sums in a row, each rounded by 2^-24 of it: F32."""
    print("case norm rows", rows, n, dtype, flush=True)
    T, gen, eps = TYPES[dtype], torch.Generator(device="cuda").manual_seed(n), 1e-3
    make = lambda *s: torch.empty(*s, device="cuda").normal_(0.2, 1.3, generator=gen)  # noqa: E731
    x, g, gamma, beta = make(rows, n).to(T), make(rows, n).to(T), make(n), make(n)
    d = gb.make_layer_norm(T, rows, n, eps)
    y, mean, rstd = torch.full_like(x, POISON), torch.full((rows,), POISON, device="cuda"), torch.full((rows,), POISON, device="cuda")
    gb.gleam_layer_norm_fwd(d, x, gamma, beta, y, mean, rstd)
    ry, rmean, rrstd = norm64(x, gamma, beta, float(np.float32(eps)))
    once = ONCE if dtype == "bf16" else 0.0

    def close(got, want, tol, what):
        diff = (got.double() - want).abs_()
        assert float(diff.norm() / want.norm()) <= tol, what
        assert float(diff.max() / want.abs().max()) <= tol * (2 * np.log(2 * got.numel())) ** 0.5, what

    close(y, ry, F32 + once, "y")
    close(mean, rmean, F32, "mean")
    close(rstd, rrstd, F32, "rstd")
    del ry
    again = x.clone()
    gb.gleam_layer_norm_fwd(d, again, gamma, beta, again)
    assert torch.equal(again, y)
    del again, y
    gx, gg, gbt = torch.full_like(x, POISON), torch.full((n,), POISON, device="cuda"), torch.full((n,), POISON, device="cuda")
    ws = torch.empty(gb.gleam_layer_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    gb.gleam_layer_norm_bwd(d, x, gamma, mean, rstd, g, gx, gg, gbt, ws)
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    gd = g.double()
    close(gg, (gd * xh).sum(0), F32, "g_gamma")
    close(gbt, gd.sum(0), F32, "g_beta")
    gd *= gamma.double()
    want = rstd.double()[:, None] * (gd - gd.mean(1, keepdim=True) - xh * (gd * xh).mean(1, keepdim=True))
    close(gx, want, 4 * F32 + once, "g_x")
    gb.gleam_layer_norm_bwd(d, x, gamma, mean, rstd, g, g, None, None, None)
    assert torch.equal(g, gx)


# ------------------------------------------------------------------------------------- how far bfloat16 results are from exact ones
def relative(got, want):
    return float(np.linalg.norm((got - want).ravel()) / np.linalg.norm(want.ravel()))


def rounded(a):
    """An exact result as a bfloat16 array holds it."""
    return torch.from_numpy(a).bfloat16().double().numpy()


def bf16_mix(B, T, P, heads, dk, dv, log_decay, seed):
    """Outputs and gradients without a state, and the exact ones: [(name, result, exact)]."""
    H, Hq, Hk, Hv = heads
    rng = np.random.default_rng(seed)
    arrays, h = {}, {}
    for name, n, d in (("q", Hq, dk), ("k", Hk, dk), ("v", Hv, dv), ("g", H, dv)):
        arrays[name], h[name] = dev(rng.normal(size=(B, T, P, n, d)), torch.bfloat16)
    a, ha = dev(np.asarray(log_decay), torch.float32)
    desc = gb.make_linattn(*(arrays[n] for n in "qkvg"), dk ** -0.5)
    ws = torch.empty(max(gb.gleam_linattn_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
    o, grads = torch.full_like(arrays["g"], POISON), [torch.full_like(arrays[n], POISON) for n in "qkv"]
    gb.gleam_linattn_fwd(desc, *(arrays[n] for n in "qkv"), a, None, None, o, None, ws)
    gb.gleam_linattn_bwd(desc, *(arrays[n] for n in "qkv"), a, None, None, arrays["g"], None, *grads, None, ws)
    exact = [lo.linattn(h["q"], h["k"], h["v"], ha, dk ** -0.5)[0], *lo.linattn_bwd(h["q"], h["k"], h["v"], ha, dk ** -0.5, h["g"])[:3]]
    return [(name, host(t), e) for name, t, e in zip(("o", "g_q", "g_k", "g_v"), (o, *grads), exact)]


@pytest.mark.parametrize("T,P,heads,dk,dv", [(20, 50, (4, 4, 4, 4), 16, 16), (64, 20, (3, 3, 3, 3), 25, 25), (40, 20, (4, 4, 2, 2), 32, 24), (300, 2, (2, 2, 2, 2), 64, 64),
                                             (1500, 1, (2, 2, 2, 2), 128, 128), (200, 3, (4, 4, 1, 1), 40, 72)])
def test_linattn_bf16_error_is_that_of_one_rounding(T, P, heads, dk, dv):
    """Outputs are rounded to bfloat16, 8 bits, and what else is rounded has 16: it adds 2^-16 to the square of the error that the exact
    results rounded once have.  1.05 asked for; scores in 8 bits would make it 1.1 to sqrt 2."""
    print("case linattn bf16 error", T, P, heads, dk, dv, flush=True)
    for name, got, exact in bf16_mix(1, T, P, heads, dk, dv, np.linspace(-0.3, -0.01, heads[0]), T):
        assert relative(got, exact) <= 1.05 * relative(rounded(exact), exact), (name, relative(got, exact), relative(rounded(exact), exact))


def test_linattn_bf16_error_where_the_state_carries_the_result():
    """Hardly any decay: from the 1250th token on at most 64 of 1250 tokens reach an output by way of scores, and the rest by the state, in 16
    bits or more: 1.2 times the error of one rounding asked for.  One part less of the state, or of the values on their way into it, would
    make that sqrt 2."""
    T = 2500
    for d in (32, 64, 128):
        print("case linattn bf16 state", d, flush=True)
        for name, got, exact in bf16_mix(1, T, 1, (2, 2, 2, 2), d, d, [-1e-5, -1e-6], d):
            far = slice(T // 2, T) if name in ("o", "g_q") else slice(0, T // 2)
            got, exact = got[:, far], exact[:, far]
            assert relative(got, exact) <= 1.2 * relative(rounded(exact), exact), (name, relative(got, exact), relative(rounded(exact), exact))


# ------------------------------------------------------------------------------------------------------------- temporal layer
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [20, 100])
def test_temporal_layer_frames_behind_the_end_take_no_part(T, dtype):
    """Whatever finite numbers stand there: they come out as they went in, their gradient goes through, and nothing else changes."""
    from paper_2207_08393_amd.temporal import TemporalLayer
    B, P, C = 2, 5, 32
    layer = TemporalLayer(B, T, P, C, 4, dtype=dtype, dropout=0.2, seed=3)
    gen = torch.Generator().manual_seed(T)
    x, g = (torch.randn(B, T, P, C, generator=gen).cuda().to(dtype) for _ in range(2))
    lengths = torch.tensor([T, T // 3], dtype=torch.int32, device="cuda")
    live = torch.arange(T, device="cuda")[None] < lengths[:, None]
    results = []
    for filling in (0.0, 1e3):
        x[~live] = filling * torch.randn(int((~live).sum()), P, C, generator=gen).cuda().to(dtype)
        h = layer.forward(x, lengths).clone()
        gx = layer.backward(g)
        assert torch.equal(h[~live], x[~live]) and torch.equal(gx[~live], g[~live])
        results.append((h[live], gx[live], layer.grad.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*results))
