"""Refusals of query/key norm with rotation, gated scan and orthogonalised update, on the host before anything could be launched (no GPU
needed)."""
import ctypes as C

import pytest
import torch

from paper_2207_08393_amd import binding as gb
from tests.test_layer_ops_host import FAKE, changed, refused

S, N = gb.gleam_seq_strides, gb.gleam_scan_strides


def qk(B=2, T=5, P=3, Hq=4, Hk=2, d=24, rot=16, dtype=torch.float32, **more):
    a = lambda h: torch.empty(B, T, P, h, d, dtype=dtype)  # noqa: E731
    return gb.make_qknorm(a(Hq), a(Hk) if Hk else None, a(Hq), a(Hk) if Hk else None, rot, **more)


def test_qknorm_refusals():
    L, d = gb.lib(), qk()
    need = gb.gleam_qknorm_workspace_bytes(d)
    assert need > 0 and need % 256 == 0
    bad = [(0, None, gb.GLEAM_E_NULL)]
    bad += [(0, changed(d, **{f: v}), gb.GLEAM_E_DESC) for f, v in (("dtype", 2), ("dtype", -1), ("pairs", 2), ("each", -1), ("eps", 0.0), ("eps", -1.0), ("eps", float("nan")),
                                                                  ("eps", float("inf")))]
    bad += [(0, changed(d, **{f: v}), gb.GLEAM_E_DIMS) for f, v in (("d", 0), ("d", 257), ("rot", -2), ("rot", 15), ("rot", 26), ("q_heads", 0), ("k_heads", -1), ("B", 0), ("T", 0),
                                                                  ("T", (1 << 30) + 1), ("P", 0), ("P", 1 << 30), ("B", 1 << 39), ("B", 1 << 62), ("q", S(-1, 1, 1, 1)),
                                                                  ("k_out", S(1 << 45, 1, 1, 1)))]
    q, o = d.q, d.q_out
    args = [C.byref(d), *FAKE[:9], None]
    refused(L.gleam_qknorm_fwd, args, bad + [(i, None, gb.GLEAM_E_NULL) for i in (1, 2, 5, 8, 9)] +
            [(8, FAKE[1], gb.GLEAM_E_DIMS), (9, FAKE[0], gb.GLEAM_E_DIMS), (9, FAKE[7], gb.GLEAM_E_DIMS),
             (0, changed(d, q_out=S(o.b, o.t, o.p, o.h - 1)), gb.GLEAM_E_DIMS), (0, changed(d, q_out=S(o.b, 0, o.p, o.h)), gb.GLEAM_E_DIMS)])
    apart = changed(d, q_out=S(o.b * 2, o.t * 2, o.p * 2, o.h * 2))                 # in place with other strides
    assert L.gleam_qknorm_fwd(apart, FAKE[0], *FAKE[1:7], FAKE[0], FAKE[8], None) == gb.GLEAM_E_DIMS
    args = [C.byref(d), *FAKE[:13], FAKE[13], need, None]
    refused(L.gleam_qknorm_bwd, args, bad + [(i, None, gb.GLEAM_E_NULL) for i in (1, 2, 5, 8, 9, 10, 11, 14)] +
            [(10, FAKE[0], gb.GLEAM_E_DIMS), (10, FAKE[1], gb.GLEAM_E_DIMS), (11, FAKE[1], gb.GLEAM_E_DIMS), (11, FAKE[9], gb.GLEAM_E_DIMS), (10, FAKE[8], gb.GLEAM_E_DIMS),
             (13, FAKE[11], gb.GLEAM_E_DIMS), (15, need - 256, gb.GLEAM_E_WORKSPACE), (14, FAKE[13] + 64, gb.GLEAM_E_WORKSPACE),
             (0, changed(d, q=S(q.b, 0, q.p, q.h)), gb.GLEAM_E_DIMS)])
    n = C.c_size_t(0)
    assert L.gleam_qknorm_workspace_bytes(C.byref(d), None) == gb.GLEAM_E_NULL
    assert L.gleam_qknorm_workspace_bytes(changed(d, d=0), C.byref(n)) == gb.GLEAM_E_DIMS


def test_qknorm_binding_compares_arrays():
    a = lambda *s: torch.empty(*s)  # noqa: E731
    x, y = a(1, 2, 1, 4, 8), a(1, 2, 1, 2, 8)
    for bad in (lambda: gb.make_qknorm(x, y, x, None, 4), lambda: gb.make_qknorm(x, y, y, y, 4), lambda: gb.make_qknorm(x, y, x, x, 4),
                lambda: gb.make_qknorm(x, a(1, 2, 1, 2, 6), x, a(1, 2, 1, 2, 6), 4), lambda: gb.make_qknorm(x, y.bfloat16(), x, y, 4),
                lambda: gb.make_qknorm(x.half(), None, x.half(), None, 4), lambda: gb.make_qknorm(x, y, x, y, 4, pairs="both"),
                lambda: gb.make_qknorm(x, y, x, y, 4, positions="none"), lambda: gb.make_qknorm(x.transpose(3, 4), None, x.transpose(3, 4), None, 2)):
        with pytest.raises(ValueError):
            bad()
    d = gb.make_qknorm(x, None, x, None, 4)
    assert d.k_heads == 0
    with pytest.raises(ValueError):                                                  # not on the GPU
        gb.gleam_qknorm_fwd(d, x, None, None, None, a(2), None, None, x, None)


def scan(B=2, T=300, P=1, C_=6, dtype=torch.float32, **more):
    return gb.make_gatedscan(*(torch.empty(B, T, P, C_, dtype=dtype) for _ in range(4)), **more)


def test_gatedscan_refusals():
    L, d = gb.lib(), scan()
    fwd, bwd = gb.gleam_gatedscan_workspace_bytes(d)
    assert fwd > 0 and bwd > 0 and fwd % 256 == 0 and bwd % 256 == 0
    bad = [(0, None, gb.GLEAM_E_NULL)]
    bad += [(0, changed(d, **{f: v}), gb.GLEAM_E_DESC) for f, v in (("dtype", 2), ("kappa", -1.0), ("kappa", float("nan")), ("kappa", float("inf")))]
    bad += [(0, changed(d, **{f: v}), gb.GLEAM_E_DIMS) for f, v in (("B", 0), ("T", 0), ("P", -1), ("C", 0), ("T", (1 << 30) + 1), ("B", 1 << 35), ("C", 1 << 31), ("P", 1 << 62),
                                                                  ("x", N(-1, 1, 1)), ("r", N(1, 1 << 45, 1)))]
    h, x = d.h, d.x
    args = [C.byref(d), *FAKE[:8], FAKE[8], fwd, None]
    refused(L.gleam_gatedscan_fwd, args, bad + [(i, None, gb.GLEAM_E_NULL) for i in (1, 2, 3, 4, 7, 9)] + [(7, FAKE[i], gb.GLEAM_E_DIMS) for i in range(3)] +
            [(10, fwd - 256, gb.GLEAM_E_WORKSPACE), (9, FAKE[8] + 8, gb.GLEAM_E_WORKSPACE), (0, changed(d, h=N(h.b, h.t - 1, h.p)), gb.GLEAM_E_DIMS),
             (0, changed(d, h=N(h.b, 0, h.p)), gb.GLEAM_E_DIMS)])
    args = [C.byref(d), *FAKE[:13], FAKE[13], bwd, None]
    refused(L.gleam_gatedscan_bwd, args, bad + [(i, None, gb.GLEAM_E_NULL) for i in (1, 2, 3, 4, 7, 9, 10, 11, 12, 14)] +
            [(9, FAKE[0], gb.GLEAM_E_DIMS), (10, FAKE[6], gb.GLEAM_E_DIMS), (11, FAKE[9], gb.GLEAM_E_DIMS), (12, FAKE[3], gb.GLEAM_E_DIMS), (13, FAKE[7], gb.GLEAM_E_DIMS),
             (13, FAKE[5], gb.GLEAM_E_DIMS), (15, bwd - 256, gb.GLEAM_E_WORKSPACE), (14, FAKE[13] + 64, gb.GLEAM_E_WORKSPACE), (0, changed(d, x=N(x.b, 0, x.p)), gb.GLEAM_E_DIMS)])
    n = C.c_size_t(0)
    assert L.gleam_gatedscan_workspace_bytes(C.byref(d), C.byref(n), None) == gb.GLEAM_E_NULL
    assert L.gleam_gatedscan_workspace_bytes(changed(d, T=0), C.byref(n), C.byref(n)) == gb.GLEAM_E_DIMS
    assert gb.gleam_gatedscan_workspace_bytes(scan(T=1))[0] == 0
    assert L.gleam_gatedscan_workspace_bytes(changed(d, x=N(x.b, 0, x.p)), C.byref(n), C.byref(n)) == gb.GLEAM_OK   # arrays that are only read may repeat


def test_gatedscan_workspace_of_either_direction():
    """Backwards h's strides are those of a gradient that is only read; a description that neither direction takes is refused."""
    L, d, n = gb.lib(), scan(), C.c_size_t(0)
    query = lambda **more: L.gleam_gatedscan_workspace_bytes(changed(d, **more), C.byref(n), C.byref(n))  # noqa: E731
    h, x = d.h, d.x
    for repeated in (N(0, 0, 0), N(h.b, 0, h.p), N(0, h.t, h.p)):
        assert query(h=repeated) == gb.GLEAM_OK and query(x=repeated, r=repeated, i=repeated) == gb.GLEAM_OK
        assert query(h=repeated, x=N(x.b, 0, x.p)) == gb.GLEAM_E_DIMS
        assert L.gleam_gatedscan_fwd(changed(d, h=repeated), *FAKE[:8], FAKE[8], 1 << 40, None) == gb.GLEAM_E_DIMS
    y = torch.empty(2, 300, 1, 6)
    e = gb.make_gatedscan(y, y, y, torch.empty(6).expand(2, 300, 1, 6))
    assert gb.gleam_gatedscan_workspace_bytes(e) == gb.gleam_gatedscan_workspace_bytes(d)


def test_gatedscan_binding_compares_arrays():
    x = torch.empty(1, 5, 2, 8)
    for bad in ((x, x, x, x[..., :4]), (x, x[:, :4], x, x), (x, x, x.bfloat16(), x), (x[0], x[0], x[0], x[0]), tuple(x.transpose(2, 3) for _ in range(4))):
        with pytest.raises(ValueError):
            gb.make_gatedscan(*bad)
    d = gb.make_gatedscan(x, x, x, x)
    with pytest.raises(ValueError):
        gb.gleam_gatedscan_fwd(d, x, x, x, torch.empty(8), None, None, x, None, None)


def test_muon_refusals():
    L, h = gb.lib(), gb.make_muon(0.02)
    need = gb.gleam_muon_workspace_bytes(3, 140, 170)
    assert need > 0 and need % 256 == 0
    assert gb.gleam_muon_workspace_bytes(3, 170, 140) == need
    assert gb.gleam_muon_workspace_bytes(3, 40, 70) == 0                              # in one workgroup each
    n = C.c_size_t(0)
    assert L.gleam_muon_workspace_bytes(3, 40, 70, None) == gb.GLEAM_E_NULL
    for sizes in ((0, 4, 4), (1, 0, 4), (1, 4, -1), (1, 65537, 4), (1, 4, 65537), (1 << 40, 40, 70), (1 << 62, 65536, 65536)):
        assert L.gleam_muon_workspace_bytes(*sizes, C.byref(n)) == gb.GLEAM_E_DIMS
    args = [C.byref(h), 3, 140, 170, 23800, *FAKE[:3], FAKE[3], need, None]
    nan, inf = float("nan"), float("inf")
    bad = [(0, changed(h, **{f: v}), gb.GLEAM_E_DESC) for f, v in (("lr", nan), ("momentum", -0.1), ("momentum", 1.0), ("momentum", nan), ("weight_decay", inf), ("eps", 0.0),
                                                                 ("eps", nan), ("a", inf), ("b", nan), ("c", inf), ("steps", 0), ("steps", 101), ("nesterov", 2), ("a", 200.0), ("c", 20000.0))]
    assert L.gleam_muon_step(changed(h, a=200.0, steps=1), *args[1:4], 5, *args[5:]) == gb.GLEAM_E_DIMS   # one step never passes 128 before the last
    refused(L.gleam_muon_step, args, bad + [(i, None, gb.GLEAM_E_NULL) for i in (0, 5, 6, 7, 8)] +
            [(1, 0, gb.GLEAM_E_DIMS), (2, 0, gb.GLEAM_E_DIMS), (3, 65537, gb.GLEAM_E_DIMS), (4, 23799, gb.GLEAM_E_DIMS), (4, -1, gb.GLEAM_E_DIMS), (4, 1 << 62, gb.GLEAM_E_DIMS),
             (6, FAKE[0], gb.GLEAM_E_DIMS), (7, FAKE[0], gb.GLEAM_E_DIMS), (7, FAKE[1], gb.GLEAM_E_DIMS), (9, need - 256, gb.GLEAM_E_WORKSPACE),
             (8, FAKE[3] + 4, gb.GLEAM_E_WORKSPACE)])


def test_muon_binding_compares_arrays():
    h, x = gb.make_muon(0.02), torch.empty(2, 6, 8)
    for bad in ((x, x, x), (x.double(), x, x), (x.transpose(1, 2), x, x)):            # not on the GPU, another type, other strides
        with pytest.raises(ValueError):
            gb.gleam_muon_step(h, *bad, None)
