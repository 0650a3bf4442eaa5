"""The gated scan through the C ABI against the float64 oracle.

Tolerances.  c s is good to some 5 of 2^-24 and so a memory of any length to as much of its exponent; what a token adds to h to about 8; a scan's
roundings, 2^-24 of h a token over the length of the memory (1000 tokens and less, at random: 30 of 2^-24): 50 2^-24 = 3e-6, asked for 1e-5
relative to the largest values of a channel's kind, as for linear attention.  Gradients in r are differences of two such terms of one size.  Results in
bfloat16 are rounded once more: 2^-8.  Sums over tokens: 1e-5 of the sum of the terms' absolute values."""
import numpy as np
import pytest
import torch

from oracle import more_layer_oracle as mo
from paper_2207_08393_amd import binding as gb
from tests.gpu_util import assert_close
from tests.gpu_util import assert_close as close
from tests.test_gpu_layers import POISON, TYPES, dev, host

pytestmark = pytest.mark.gpu
F32, ONCE = 1e-5, 2.0 ** -8
# Where c s is below 2^-126, the smallest normal float32, its root counts as 0: sqrt(2 c s) < 1.6e-19 is what a unit gradient would have brought, and
# no G in the tests that go there passes 200 (140 tokens at most, whose normal gradients add up at random to some 12 of their 1, and each below 5)
TINY = 200 * 1.6e-19


def array(shape, layout, T):
    """A poisoned [B][T][P][C] array: 'tokens' row-major, 'pixels' [B][P][T][C], 'gaps' with unused elements around every axis."""
    B, t, P, C = shape
    if layout == "pixels":
        return torch.full((B, P, t, C), POISON, dtype=T, device="cuda").permute(0, 2, 1, 3)
    if layout == "gaps":
        store = torch.full((1 + B * (t + 1) * (P + 1) * (C + 3),), POISON, dtype=T, device="cuda")
        return store[1:].as_strided(shape, ((t + 1) * (P + 1) * (C + 3), (P + 1) * (C + 3), C + 3, 1))
    return torch.full(shape, POISON, dtype=T, device="cuda")


class Scan:
    """One call's arrays on the device and their values on the host; tokens behind the sequences' ends are NaN or infinite."""

    def __init__(self, B, T, P, C, dtype, layout="tokens", lengths=None, state=True, seed=0, kappa=8.0, memory=None, gate=(0.0, 1.0)):
        self.T, rng = TYPES[dtype], np.random.default_rng(seed + T + 31 * C)
        self.low, self.layout, self.kappa, self.shape = dtype == "bf16", layout, kappa, (B, T, P, C)
        live = np.arange(T)[None, :] < (np.full(B, T) if lengths is None else np.array(lengths))[:, None]
        self.x, self.h = {}, {}
        for name in "xrig":
            t = array(self.shape, layout, self.T)
            v = rng.normal(*gate, size=t.shape) if name == "r" else rng.normal(size=t.shape)
            t.copy_(torch.from_numpy(np.where(live[:, :, None, None], v, rng.choice([np.nan, np.inf, -np.inf], size=t.shape)).astype(np.float32)))
            self.x[name], self.h[name] = t, host(t)
        memory = 2.0 * 500.0 ** rng.random(C) if memory is None else np.full(C, memory)
        self.lam, self.hlam = dev(np.log(np.expm1(2.0 / (8.0 * memory))), torch.float32)
        self.state, self.hs = dev(rng.normal(size=(B, P, C)), torch.float32) if state else (None, None)
        self.gstate, self.hgs = dev(rng.normal(size=(B, P, C)), torch.float32) if state else (None, None)
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.hl = lengths

    def plan(self, out):
        return gb.make_gatedscan(self.x["x"], self.x["r"], self.x["i"], out, self.kappa)

    def new(self):
        return array(self.shape, self.layout, self.T)

    def new_state(self):
        return torch.full((self.shape[0], *self.shape[2:]), POISON, device="cuda")

    def fwd(self, state_out=True):
        h, S = self.new(), self.new_state() if state_out else None
        d = self.plan(h)
        ws = torch.full((gb.gleam_gatedscan_workspace_bytes(d)[0],), 255, dtype=torch.uint8, device="cuda")
        gb.gleam_gatedscan_fwd(d, self.x["x"], self.x["r"], self.x["i"], self.lam, self.lengths, self.state, h, S, ws)
        return h, S

    def bwd(self, g_state=True):
        d = self.plan(self.x["g"])
        ws = torch.full((gb.gleam_gatedscan_workspace_bytes(d)[1],), 255, dtype=torch.uint8, device="cuda")
        grads, gl, gS = [self.new() for _ in range(3)], torch.full((self.shape[3],), POISON, device="cuda"), self.new_state() if g_state else None
        gb.gleam_gatedscan_bwd(d, self.x["x"], self.x["r"], self.x["i"], self.lam, self.lengths, self.state, self.x["g"], self.gstate, *grads, gl, gS, ws)
        return grads, gl, gS

    def check(self, tiny=0.0):
        """tiny: results that are all smaller than this in 64 bits may be as small as that in any way (float32 has no numbers for them)."""
        once, k, h = ONCE if self.low else 0.0, self.kappa, self.h

        def assert_close(got, ref, tol, what):
            if np.abs(ref).max() < tiny:
                assert np.abs(got).max() <= tiny, what
            else:
                close(got, ref, tol, what)

        y, S = self.fwd()
        ry, rS = mo.gatedscan(h["x"], h["r"], h["i"], self.hlam, k, self.hl, self.hs)
        assert_close(host(y), ry, F32 + once, "h")
        assert_close(host(S), rS, F32, "state")
        grads, gl, gS = self.bwd()
        *ref, rgl, rgS, size = mo.gatedscan_bwd(h["x"], h["r"], h["i"], self.hlam, k, h["g"], self.hl, self.hs, self.hgs)
        for name, got, want in zip(("g_x", "g_r", "g_i"), grads, ref):
            assert_close(host(got), want, F32 + once, name)
        assert np.all(np.abs(host(gl) - rgl) <= F32 * size + 1e-30 + tiny), "g_lambda"
        assert_close(host(gS), rgS, F32, "g_state")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 15, 16, 17, 20, 31, 33, 64, 65, 127, 128, 129, 200, 256, 257, 1000])
def test_gatedscan_lengths(T, dtype):
    print("case scan", T, dtype, flush=True)
    Scan(2, T, 1, 40, dtype).check()
    Scan(1, T, 3, 7, dtype, state=False).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [1, 5])
@pytest.mark.parametrize("C", [1, 2, 3, 63, 64, 65, 127, 128, 129, 301])
def test_gatedscan_channels(C, P, dtype):
    print("case scan channels", C, P, dtype, flush=True)
    Scan(2, 21, P, C, dtype, lengths=[21, 10]).check()
    Scan(1, 150, P, C, dtype).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["tokens", "pixels", "gaps"])
@pytest.mark.parametrize("T,lengths", [(1, [0, 1, 1, 0, 1]), (20, [20, 0, 0, 16, 17]), (70, [0, 1, 64, 65, 70]), (700, [700, 0, 257, 513, 384]), (300, [305, -3, 2 ** 31 - 1, 128, 129])])
def test_gatedscan_ragged_and_strided(T, lengths, layout, dtype):
    """Empty sequences among others, ends on, before and behind the borders of waves and chunks, lengths out of range."""
    print("case scan ragged", T, lengths, layout, dtype, flush=True)
    Scan(5, T, 2, 9, dtype, layout, lengths).check()
    Scan(5, T, 1, 66, dtype, layout, lengths, state=False).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gatedscan_many_columns(dtype):
    print("case scan many columns", dtype, flush=True)
    Scan(1, 20, 2500, 16, dtype).check()
    Scan(3, 5, 1, 4099, dtype).check()
    Scan(1, 6000, 1, 5, dtype).check()


@pytest.mark.parametrize("B,P,C,dtype", [(1, 16641, 7, "f32"), (1, 16641, 300, "bf16"), (1, 30000, 64, "bf16"), (2, 150 * 150, 64, "f32"), (1, 200 * 200, 7, "bf16"),
                                         (1, 131073, 7, "f32"), (1, 368 * 368, 3, "f32")])
def test_gatedscan_gradients_of_many_pixels(B, P, C, dtype):
    """Numbers of pixels that the slabs of rows, which the sums over pixels are split into, do not divide; the workspace starts as NaN."""
    print("case scan pixels", B, P, C, dtype, flush=True)
    Scan(B, 2, P, C, dtype).check()


def test_gatedscan_of_long_memories_and_closed_gates():
    """Memories of 100 000 tokens, where a itself, rounded to float32, would be off by 0.3 % of 1 - a; gates that are shut or wide open, with
    decays from none to all."""
    Scan(1, 3000, 1, 16, "f32", memory=1e5, gate=(0.0, 0.0)).check()
    for mean in (-120.0, -60.0, -20.0, 20.0, 120.0):
        print("gate", mean, flush=True)
        Scan(1, 140, 1, 6, "f32", gate=(mean, 0.5), kappa=8.0).check(TINY)
        Scan(1, 10, 1, 6, "f32", gate=(mean, 0.5), kappa=2000.0).check(TINY)


@pytest.mark.parametrize("lam", [-200.0, -90.0, -30.0, 0.0, 30.0, 200.0])
def test_gatedscan_lambdas(lam):
    """From decays that float32 cannot tell from none to the loss of all memory."""
    m = Scan(1, 40, 1, 3, "f32")
    m.lam.fill_(lam)
    m.hlam = host(m.lam)
    m.check(TINY)


def test_gatedscan_without_decay():
    """kappa 0: nothing is lost and nothing enters."""
    m = Scan(1, 150, 1, 5, "f32", kappa=0.0)
    h, S = m.fwd()
    assert np.array_equal(host(S), host(m.state)) and np.array_equal(host(h), np.repeat(host(m.state)[:, None], 150, 1))
    grads, gl, gS = m.bwd()
    assert all(not host(g).any() for g in (*grads, gl))
    assert_close(host(gS), m.h["g"].sum(1) + m.hgs, F32, "g_state")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [7, 64, 129])
def test_gatedscan_pieces_are_the_whole(C, dtype):
    """A sequence in one call, in two with the state handed over, and its last tokens one by one, the state updated in place."""
    m = Scan(2, 300, 3, C, dtype)
    h, S = m.fwd()
    part, run = m.new(), m.state.clone()
    for a, b in [(0, 170), (170, 290)] + [(t, t + 1) for t in range(290, 300)]:
        x = [m.x[n][:, a:b] for n in "xri"]
        d = gb.make_gatedscan(*x, part[:, a:b], m.kappa)
        gb.gleam_gatedscan_fwd(d, *x, m.lam, None, run, part[:, a:b], run, torch.empty(gb.gleam_gatedscan_workspace_bytes(d)[0], dtype=torch.uint8, device="cuda"))
    assert_close(host(part), host(h), F32 + (ONCE if m.low else 0), "h")
    assert_close(host(run), host(S), F32, "state")


def test_gatedscan_writes_nothing_else():
    """Values between the rows of h and of the gradients stay what they were."""
    for dtype in ("f32", "bf16"):
        m = Scan(2, 20, 3, 9, dtype, layout="gaps", lengths=[20, 3])
        h = m.new()
        d, (ref, _) = m.plan(h), m.fwd()
        store = torch.full((h.untyped_storage().nbytes() // h.element_size(),), 7.0, dtype=m.T, device="cuda")
        h = store[1:].as_strided(h.shape, h.stride())
        gb.gleam_gatedscan_fwd(d, m.x["x"], m.x["r"], m.x["i"], m.lam, m.lengths, m.state, h, None, None)
        assert torch.equal(h, ref)
        h.fill_(7.0)
        assert bool((store == 7.0).all())


def test_gatedscan_infinities_stay_in_their_channel():
    m = Scan(2, 200, 1, 6, "f32")
    clean, _ = m.fwd()
    m.x["x"][0, 50, 0, 2], m.x["r"][1, 150, 0, 4] = float("inf"), POISON
    h, _ = m.fwd()
    touched = torch.zeros_like(h, dtype=torch.bool)
    touched[0, 50:, 0, 2], touched[1, 150:, 0, 4] = True, True
    assert torch.equal(torch.where(touched, clean, h), clean) and not bool(torch.isfinite(h[touched]).any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 50, 200])
@pytest.mark.parametrize("C", [6, 7])
def test_gatedscan_of_inputs_that_stand_for_many(C, T, dtype):
    """Forward inputs with strides of 0 give what their copies give, bit by bit."""
    B, P, type_ = 3, 4, TYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(T)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(type_)  # noqa: E731
    x, r, i = new(1, T, P, C).expand(B, T, P, C), new(B, T, 1, C).expand(B, T, P, C), new(B, 1, P, C).expand(B, T, P, C)
    lam = torch.randn(C, device="cuda", generator=gen)
    out = []
    for args in ((x, r, i), tuple(t.contiguous() for t in (x, r, i))):
        h = torch.full((B, T, P, C), POISON, dtype=type_, device="cuda")
        d = gb.make_gatedscan(*args, h)
        ws = torch.full((gb.gleam_gatedscan_workspace_bytes(d)[0],), 255, dtype=torch.uint8, device="cuda")
        gb.gleam_gatedscan_fwd(d, *args, lam, None, None, h, None, ws)
        out.append(h)
    assert torch.equal(out[0], out[1]) and bool(torch.isfinite(out[0]).all())


@pytest.mark.parametrize("T", [3, 200])
@pytest.mark.parametrize("strides", [(0, 0, 0, 1), (0, 9, 0, 1), (9, 0, 9, 1)])
def test_gatedscan_gradients_of_a_gradient_that_stands_for_many(strides, T):
    """Backwards g_h is only read: with strides of 0, as a sum's gradient has them, it gives what its copy gives, bit by bit."""
    B, P, C = 2, 3, 9
    m = Scan(B, T, P, C, "f32", lengths=[T, T - 1])
    g = torch.randn(T * C + B * P * 9 * T, device="cuda").as_strided((B, T, P, C), strides)
    out = []
    for m.x["g"] in (g, g.contiguous()):
        out.append(m.bwd())
    (a, al, aS), (b, bl, bS) = out
    assert all(torch.equal(x, y) for x, y in zip((*a, al, aS), (*b, bl, bS))) and bool(torch.isfinite(torch.cat([x.flatten() for x in (*a, al, aS)])).all())


def test_gatedscan_state_out_of_nothing_and_not_wanted():
    m = Scan(2, 140, 1, 6, "bf16", lengths=[140, 0], state=False)
    S = m.fwd()[1]
    assert_close(host(S), mo.gatedscan(m.h["x"], m.h["r"], m.h["i"], m.hlam, m.kappa, m.hl)[1], F32, "state")
    assert torch.equal(m.fwd(False)[0], m.fwd()[0])
    grads, gl, _ = m.bwd(False)
    again = m.bwd()
    assert all(torch.equal(a, b) for a, b in zip((*grads, gl), (*again[0], again[1])))


def test_gatedscan_gradients_against_differences():
    m = Scan(2, 150, 1, 5, "f32", lengths=[150, 93])
    (grads, gl, gS), rng, step = m.bwd(), np.random.default_rng(8), 1e-5
    zero = {n: np.where(np.isfinite(v), v, 0.0) for n, v in m.h.items()}

    def loss(x, r, i, lam, S0):
        h, S = mo.gatedscan(x, r, i, lam, m.kappa, m.hl, S0)
        return (h * zero["g"]).sum() + (S * m.hgs).sum()

    at = [zero["x"], zero["r"], zero["i"], m.hlam, m.hs]
    for k, grad in enumerate((*grads, gl, gS)):
        e = rng.normal(size=at[k].shape)
        f = lambda z: loss(*(z if j == k else at[j] for j in range(5)))  # noqa: E731,B023
        assert abs((f(at[k] + step * e) - f(at[k] - step * e)) / (2 * step) - (host(grad) * e).sum()) <= 1e-5 * np.abs(host(grad) * e).sum()


def test_gatedscan_offsets_past_32_bits():
    """Tokens more than 2^31 elements behind the first."""
    T, C, stride = 70, 8, 34_000_000
    store = torch.zeros(T * stride, dtype=torch.bfloat16, device="cuda")
    at = lambda n: store[n * C:].as_strided((1, T, 1, C), (0, stride, 0, 1))  # noqa: E731
    rng = np.random.default_rng(9)
    for n in range(3):
        at(n).copy_(torch.from_numpy(rng.normal(size=(1, T, 1, C)).astype(np.float32)))
    lam, hlam = dev(np.full(C, -3.0), torch.float32)
    d = gb.make_gatedscan(at(0), at(1), at(2), at(3), 8.0)
    ws = torch.empty(gb.gleam_gatedscan_workspace_bytes(d)[0], dtype=torch.uint8, device="cuda")
    gb.gleam_gatedscan_fwd(d, at(0), at(1), at(2), lam, None, None, at(3), None, ws)
    assert_close(host(at(3)), mo.gatedscan(host(at(0)), host(at(1)), host(at(2)), hlam, 8.0)[0], F32 + ONCE, "h")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gatedscan_twice_is_the_same_bits_on_another_stream_and_in_a_graph(dtype):
    m = Scan(2, 700, 1, 70, dtype, lengths=[700, 300])
    h, S = m.fwd()
    grads, gl, gS = m.bwd()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        h2, S2 = m.fwd()
        grads2, gl2, gS2 = m.bwd()
    side.synchronize()
    mine = (h, S, *grads, gl, gS)
    assert all(torch.equal(a, b) for a, b in zip(mine, (h2, S2, *grads2, gl2, gS2)))
    d = m.plan(h)
    ws = torch.empty(max(gb.gleam_gatedscan_workspace_bytes(d)), dtype=torch.uint8, device="cuda")   # both directions share it
    x, r, i, g = (m.x[n] for n in "xrig")
    state = m.state.clone()

    def calls():
        gb.gleam_gatedscan_fwd(d, x, r, i, m.lam, m.lengths, state, h, S, ws)
        gb.gleam_gatedscan_bwd(d, x, r, i, m.lam, m.lengths, state, g, m.gstate, *grads, gl, gS, ws)

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for k in range(4):
        for t in (x, r, i, g):
            t.copy_(torch.randn(t.shape, device="cuda"))
        m.lengths.copy_(torch.tensor([700 - k, 100 * k], dtype=torch.int32))
        state.fill_(float(k))
        graph.replay()
        got = [t.clone() for t in mine]
        torch.cuda.synchronize()
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, mine))
