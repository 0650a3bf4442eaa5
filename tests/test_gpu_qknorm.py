"""Norm and rotation of queries and keys through the C ABI against the float64 oracle.

Tolerances.  A row's sum of up to 256 squares is formed in at most 16 + 6 additions, 22 of 2^-24 in the worst case and half of that in its
root; mean, root and quotient, the products with r and gamma, an angle's fraction rounded to float32 (pi 2^-24), sine and cosine (2 of
2^-24 each) and the turn (3) add about 12: 25 2^-24 = 1.5e-6, asked for 2e-6.  A gradient is a difference of terms of the size of r g gamma that
have as much each: 4e-6 of the largest of those.  Results in bfloat16 are rounded once more: 2^-8.  Sums over rows: 4e-6 of the sum of the
absolute values."""
import numpy as np
import pytest
import torch

from oracle import more_layer_oracle as mo
from paper_2207_08393_amd import binding as gb
from tests.gpu_util import assert_close
from tests.test_gpu_layers import POISON, TYPES, dev, host, strided

pytestmark = pytest.mark.gpu
F32, ONCE = 2e-6, 2.0 ** -8


class Qk:
    """One call's arrays on the device and their values on the host; tokens behind the sequences' ends are NaN or infinite."""

    def __init__(self, B, T, P, Hq, Hk, d, rot, dtype, pairs="halves", layout="tokens", lengths=None, positions="start", gamma=True, eps=1e-3, seed=0, span=2 ** 31):
        self.T, rng = TYPES[dtype], np.random.default_rng(seed + 7 * T + d)
        self.low, self.pairs, self.rot, self.eps, self.layout, self.each = dtype == "bf16", pairs, rot, eps, layout, positions == "each"
        self.heads = [h for h in (Hq, Hk) if h]
        live = np.arange(T)[None, :] < (np.full(B, T) if lengths is None else np.array(lengths))[:, None]
        self.x, self.hx, self.g, self.hg = [], [], [], []
        for h in self.heads:
            for dst, hdst in ((self.x, self.hx), (self.g, self.hg)):
                t = strided((B, T, P, h, d), layout, self.T, offset=1 if layout == "gaps" else 0)
                v = np.where(live[:, :, None, None, None], rng.normal(size=t.shape), rng.choice([np.nan, np.inf, -np.inf], size=t.shape))
                t.copy_(torch.from_numpy(v.astype(np.float32)))
                dst.append(t)
                hdst.append(host(t))
        self.gamma, self.hgamma = zip(*(dev(1 + 0.2 * rng.normal(size=d), torch.float32) if gamma else (None, None) for _ in range(2)))
        self.freq, self.hfreq = dev(100.0 ** (-np.arange(rot // 2) / max(rot // 2, 1)), torch.float32) if rot else (None, None)
        self.hpos = None
        if positions:
            self.hpos = rng.integers(-span, span, (B, T) if self.each else (B,))
        self.pos = None if self.hpos is None else torch.from_numpy(self.hpos.astype(np.int32)).cuda()
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.hl = lengths

    def new(self, i):
        return strided(self.x[i].shape, self.layout, self.T, offset=1 if self.layout == "gaps" else 0)

    def both(self, arrays):
        return list(arrays) + [None] * (2 - len(self.heads))

    def plan(self, out):
        return gb.make_qknorm(*self.both(self.x), *self.both(out), self.rot, self.eps, self.pairs, "each" if self.each else "start")

    def fwd(self):
        out = [self.new(i) for i in range(len(self.heads))]
        gb.gleam_qknorm_fwd(self.plan(out), *self.both(self.x), *self.gamma, self.freq, self.pos, self.lengths, *self.both(out))
        return out

    def bwd(self, sums=True):
        out = [self.new(i) for i in range(len(self.heads))]
        d = self.x[0].shape[4]
        plan = self.plan(self.g)
        gg = [torch.full((d,), POISON, device="cuda") if sums else None for _ in range(2)]
        ws = torch.full((gb.gleam_qknorm_workspace_bytes(plan),), 255, dtype=torch.uint8, device="cuda") if sums else None
        gb.gleam_qknorm_bwd(plan, *self.both(self.x), *self.gamma, self.freq, self.pos, self.lengths, *self.both(self.g), *self.both(out), *self.both(gg[:len(self.heads)]), ws)
        return out, gg

    def check(self):
        once = ONCE if self.low else 0.0
        for i, y in enumerate(self.fwd()):
            assert_close(host(y), mo.qknorm(self.hx[i], self.hgamma[i], self.hfreq, np.float32(self.eps), self.rot, self.pairs, self.hpos, self.each, self.hl), F32 + once, f"out {i}")
        grads, gg = self.bwd()
        for i, gx in enumerate(grads):
            rx, rg, size = mo.qknorm_bwd(self.hx[i], self.hgamma[i], self.hfreq, np.float32(self.eps), self.rot, self.pairs, self.hg[i], self.hpos, self.each, self.hl)
            x, g = (np.nan_to_num(z, nan=0.0, posinf=0.0, neginf=0.0) for z in (self.hx[i], self.hg[i]))
            terms = np.sqrt(2.0) * np.abs(g).max() * (1.0 if self.hgamma[i] is None else np.abs(self.hgamma[i]).max()) / np.sqrt((x * x).mean(-1) + self.eps).min()
            got = host(gx)
            assert np.all(np.isfinite(got)) and np.abs(got - rx).max() <= 2 * F32 * terms + once * np.abs(rx).max(), f"g {i}"
            assert np.all(np.abs(host(gg[i]) - rg) <= 2 * F32 * size + 1e-30), f"g_gamma {i}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("d,rot", [(1, 0), (2, 2), (3, 2), (5, 4), (8, 8), (16, 16), (16, 4), (20, 12), (33, 32), (40, 32), (64, 64), (64, 0), (72, 8), (96, 48), (100, 100),
                                   (127, 126), (128, 128), (128, 64), (200, 6), (255, 254), (255, 2), (256, 256)])
def test_qknorm_widths(d, rot, pairs, dtype):
    print("case qk widths", d, rot, pairs, dtype, flush=True)
    Qk(2, 5, 1, 3, 2, d, rot, dtype, pairs).check()
    Qk(1, 3, 4, 2, 0, d, rot, dtype, pairs, positions="each", gamma=False).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["tokens", "heads", "gaps"])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (6, 2), (16, 1), (5, 0), (33, 11)])
def test_qknorm_heads_and_layouts(Hq, Hk, layout, dtype):
    print("case qk heads", Hq, Hk, layout, dtype, flush=True)
    Qk(2, 9, 2, Hq, Hk, 24, 16, dtype, "halves", layout, lengths=[9, 4]).check()
    Qk(3, 1, 1, Hq, Hk, 64, 64, dtype, "neighbours", layout, lengths=[0, 1, 1]).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("positions", [None, "start", "each"])
def test_qknorm_lengths_and_positions(positions, dtype):
    """Lengths out of range count as the nearest; empty sequences; positions over all of int32, and sums with a token's number beyond."""
    print("case qk lengths", positions, dtype, flush=True)
    Qk(5, 70, 1, 4, 4, 32, 32, dtype, lengths=[0, 75, -3, 1, 70], positions=positions).check()
    Qk(2, 70, 3, 2, 1, 16, 8, dtype, "neighbours", lengths=[69, 2], positions=positions, span=1000).check()
    m = Qk(1, 4, 1, 1, 1, 8, 8, dtype, positions="start")
    m.hpos[:] = 2 ** 31 - 2
    m.pos.fill_(2 ** 31 - 2)
    m.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_qknorm_many_rows(dtype):
    """Pixels of few frames, long sequences, more units of work than a launch has waves, and the longest rows of heads."""
    print("case qk many rows", dtype, flush=True)
    Qk(1, 3, 3001, 4, 4, 16, 16, dtype).check()
    Qk(2, 5000, 1, 3, 1, 64, 32, dtype, lengths=[5000, 4321]).check()
    Qk(1, 2, 1, 700, 41, 128, 128, dtype, "neighbours").check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_qknorm_in_place_and_without_sums(dtype):
    m = Qk(2, 40, 2, 4, 2, 48, 32, dtype, layout="gaps")
    out, (grads, _) = m.fwd(), m.bwd()
    same, _ = m.bwd(sums=False)
    assert all(torch.equal(a, b) for a, b in zip(grads, same))
    g = [strided(t.shape, "gaps", m.T, offset=1).copy_(t) for t in m.g]
    gb.gleam_qknorm_bwd(m.plan(g), *m.x, *m.gamma, m.freq, m.pos, m.lengths, *g, *g, None, None, None)
    assert all(torch.equal(a, b) for a, b in zip(grads, g))
    one = torch.empty(48, device="cuda")
    plan = m.plan(m.g)
    two = torch.empty_like(one)
    ws = torch.empty(gb.gleam_qknorm_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    gb.gleam_qknorm_bwd(plan, *m.x, *m.gamma, m.freq, m.pos, m.lengths, *m.g, *same, None, one, ws)   # the keys' alone
    gb.gleam_qknorm_bwd(plan, *m.x, *m.gamma, m.freq, m.pos, m.lengths, *m.g, *same, two, None, ws)
    both = m.bwd()[1]
    assert torch.equal(one, both[1]) and torch.equal(two, both[0])
    x = m.x
    gb.gleam_qknorm_fwd(m.plan(x), *x, *m.gamma, m.freq, m.pos, m.lengths, *x)                         # results in the place of q and k
    assert all(torch.equal(a, b) for a, b in zip(out, x))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,rot", [(16, 8), (5, 4)])
def test_qknorm_of_inputs_that_stand_for_many(d, rot, dtype):
    """Inputs with strides of 0 (a head for all heads, a token for all tokens) give what their copies give, bit by bit."""
    B, T, P, H, type_ = 2, 7, 3, 4, TYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(d)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(type_)  # noqa: E731
    q, k = new(B, T, P, 1, d).expand(B, T, P, H, d), new(1, 1, P, 2, d).expand(B, T, P, 2, d)
    freq, gamma, out = torch.rand(rot // 2, device="cuda", generator=gen), torch.rand(d, device="cuda", generator=gen), []
    for a, b in ((q, k), (q.contiguous(), k.contiguous())):
        to = [torch.full(t.shape, POISON, dtype=type_, device="cuda") for t in (a, b)]
        gb.gleam_qknorm_fwd(gb.make_qknorm(a, b, *to, rot), a, b, gamma, None, freq, None, None, *to)
        out.append(to)
    assert all(torch.equal(x, y) and bool(torch.isfinite(x).all()) for x, y in zip(*out))


def test_qknorm_writes_nothing_else():
    """Values between the heads, and rows of an array that the call does not name."""
    m = Qk(2, 3, 2, 3, 2, 20, 8, "bf16", layout="gaps")
    store = torch.full((2 * 4 * 3 * 4 * 23 + 64,), 7.0, dtype=m.T, device="cuda")
    q = store[1:].as_strided((2, 3, 2, 3, 20), (4 * 3 * 4 * 23, 3 * 4 * 23, 4 * 23, 23, 1))
    k = torch.empty(2, 3, 2, 2, 20, dtype=m.T, device="cuda")
    gb.gleam_qknorm_fwd(m.plan([q, k]), *m.x, *m.gamma, m.freq, m.pos, m.lengths, q, k)
    assert torch.equal(q, m.fwd()[0])
    q.fill_(7.0)
    assert bool((store == 7.0).all())


def test_qknorm_of_zeros_infinities_and_large_numbers():
    x = torch.zeros(1, 5, 1, 1, 8, device="cuda")
    x[0, 1], x[0, 2, 0, 0, 3], x[0, 3, 0, 0, 1], x[0, 4] = 3e19, float("inf"), float("nan"), 1e-30
    y, f = torch.full_like(x, POISON), torch.zeros(4, device="cuda")
    gb.gleam_qknorm_fwd(gb.make_qknorm(x, None, y, None, 8), x, None, None, None, f, None, None, y, None)
    y = host(y)[0, :, 0, 0]
    assert not y[0].any() and not y[1].any()                                       # the squares pass the range of a float32: r = 0
    assert np.isnan(y[2, 3]) and np.all(np.isnan(y[3]))
    assert np.allclose(y[4], 1e-30 / np.sqrt(1e-6), rtol=1e-6)


def test_qknorm_gradients_against_differences():
    m = Qk(2, 6, 1, 3, 2, 10, 8, "f32", lengths=[6, 4], span=100)
    (grads, gg), rng, h = m.bwd(), np.random.default_rng(8), 1e-4
    for i in range(2):
        at = [np.where(np.isfinite(m.hx[i]), m.hx[i], 0.0), m.hgamma[i]]
        g = np.where(np.isfinite(m.hg[i]), m.hg[i], 0.0)
        loss = lambda x, w: (mo.qknorm(x, w, m.hfreq, np.float32(m.eps), m.rot, m.pairs, m.hpos, m.each, m.hl) * g).sum()  # noqa: E731,B023
        for k, grad in enumerate((grads[i], gg[i])):
            e = rng.normal(size=at[k].shape)
            f = lambda z: loss(*(z if j == k else at[j] for j in range(2)))  # noqa: E731,B023
            assert abs((f(at[k] + h * e) - f(at[k] - h * e)) / (2 * h) - (host(grad) * e).sum()) <= 1e-5 * np.abs(host(grad) * e).sum()


def test_qknorm_offsets_past_32_bits():
    """Tokens more than 2^31 elements behind the first."""
    T, d, stride = 70, 16, 34_000_000
    store = torch.zeros(T * stride, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((1, T, 1, 1, d), (0, stride, 0, 0, 1))
    y = store[d:].as_strided((1, T, 1, 1, d), (0, stride, 0, 0, 1))
    x.copy_(torch.randn(1, T, 1, 1, d, generator=torch.Generator().manual_seed(1)))
    freq, hf = dev(0.5 ** np.arange(8), torch.float32)
    gb.gleam_qknorm_fwd(gb.make_qknorm(x, None, y, None, d), x, None, None, None, freq, None, None, y, None)
    assert_close(host(y), mo.qknorm(host(x), None, hf, np.float32(1e-6), d, "halves"), F32 + ONCE, "out")


def test_qknorm_twice_is_the_same_bits_on_another_stream_and_in_a_graph():
    m = Qk(2, 700, 1, 6, 2, 64, 32, "bf16", lengths=[700, 300])
    out, (grads, gg) = m.fwd(), m.bwd()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        out2, (grads2, gg2) = m.fwd(), m.bwd()
    side.synchronize()
    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))  # noqa: E731
    assert same(out, out2) and same(grads, grads2) and same(gg, gg2)
    plan, plan_b = m.plan(out), m.plan(m.g)
    ws = torch.empty(gb.gleam_qknorm_workspace_bytes(plan_b), dtype=torch.uint8, device="cuda")

    def calls():
        gb.gleam_qknorm_fwd(plan, *m.x, *m.gamma, m.freq, m.pos, m.lengths, *out)
        gb.gleam_qknorm_bwd(plan_b, *m.x, *m.gamma, m.freq, m.pos, m.lengths, *m.g, *grads, *gg, ws)

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for k in range(4):                                                             # other inputs, positions and lengths at each replay
        for x in m.x:
            x.copy_(torch.randn(x.shape, device="cuda"))
        m.pos.fill_(1000 * k)
        m.lengths.copy_(torch.tensor([700 - k, 10 * k], dtype=torch.int32))
        graph.replay()
        got = [t.clone() for t in (*out, *grads, *gg)]
        torch.cuda.synchronize()
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(got, (*out, *grads, *gg)))
