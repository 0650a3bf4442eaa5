"""Refusals of the sequence-layer operators' entry points, on the host before anything could be launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2207_08393_amd import binding as gb

FAKE = [0x10000 * (i + 1) for i in range(16)]   # 256-byte aligned, never dereferenced: validation fails first


def refused(fn, args, changes):
    """Every (index, value, status): the call with that one argument changed returns that status."""
    for i, value, status in changes:
        a = list(args)
        a[i] = value
        assert fn(*a) == status, (fn, i, value)


def changed(desc, **fields):
    new = type(desc)()
    C.memmove(C.byref(new), C.byref(desc), C.sizeof(desc))
    for k, v in fields.items():
        setattr(new, k, v)
    return C.byref(new)


def test_layer_norm_refusals():
    L, d = gb.lib(), gb.make_layer_norm(0, 100, 33, 1e-5, ld=40)
    need = gb.gleam_layer_norm_workspace_bytes(d)
    assert need > 0 and need % 4 == 0
    bad = [(0, None, gb.GLEAM_E_NULL), (0, changed(d, dtype=2), gb.GLEAM_E_DESC), (0, changed(d, rows=0), gb.GLEAM_E_DIMS), (0, changed(d, n=0), gb.GLEAM_E_DIMS),
           (0, changed(d, n=-5), gb.GLEAM_E_DIMS), (0, changed(d, ld_in=32), gb.GLEAM_E_DIMS), (0, changed(d, ld_out=32), gb.GLEAM_E_DIMS),
           (0, changed(d, ld_in=1 << 50), gb.GLEAM_E_DIMS), (0, changed(d, rows=1 << 40), gb.GLEAM_E_DIMS), (0, changed(d, eps=0.0), gb.GLEAM_E_DESC),
           (0, changed(d, eps=-1.0), gb.GLEAM_E_DESC), (0, changed(d, eps=float("nan")), gb.GLEAM_E_DESC), (0, changed(d, eps=float("inf")), gb.GLEAM_E_DESC)]
    x, y = FAKE[0], FAKE[1]
    refused(L.gleam_layer_norm_fwd, [C.byref(d), x, FAKE[2], FAKE[3], y, FAKE[4], FAKE[5], None], bad + [(1, None, gb.GLEAM_E_NULL), (4, None, gb.GLEAM_E_NULL)])
    apart = gb.make_layer_norm(0, 100, 33, 1e-5, ld=40, ld_out=48)
    assert L.gleam_layer_norm_fwd(C.byref(apart), x, None, None, x, None, None, None) == gb.GLEAM_E_DIMS
    args = [C.byref(d), x, FAKE[2], FAKE[3], FAKE[4], y, FAKE[5], FAKE[6], FAKE[7], FAKE[8], need, None]
    refused(L.gleam_layer_norm_bwd, args, bad + [(i, None, gb.GLEAM_E_NULL) for i in (1, 3, 4, 5, 6, 9)] +
            [(6, x, gb.GLEAM_E_DIMS), (10, need - 1, gb.GLEAM_E_WORKSPACE), (9, FAKE[8] + 8, gb.GLEAM_E_WORKSPACE)])
    n = C.c_size_t(0)
    assert L.gleam_layer_norm_workspace_bytes(C.byref(d), None) == gb.GLEAM_E_NULL
    assert L.gleam_layer_norm_workspace_bytes(changed(d, n=0), C.byref(n)) == gb.GLEAM_E_DIMS


def test_dropout_refusals():
    L, d = gb.lib(), gb.make_dropout(1, 10, 12, 0.1, 1, 2, ld=16)
    bad = [(0, None, gb.GLEAM_E_NULL), (0, changed(d, dtype=-1), gb.GLEAM_E_DESC), (0, changed(d, rows=-1), gb.GLEAM_E_DIMS), (0, changed(d, n=0), gb.GLEAM_E_DIMS),
           (0, changed(d, ld_in=11), gb.GLEAM_E_DIMS), (0, changed(d, ld_out=11), gb.GLEAM_E_DIMS), (0, changed(d, p=-0.1), gb.GLEAM_E_DESC),
           (0, changed(d, p=1.1), gb.GLEAM_E_DESC), (0, changed(d, p=float("nan")), gb.GLEAM_E_DESC), (0, changed(d, rows=1 << 30, n=1 << 11, ld_in=1 << 11), gb.GLEAM_E_DIMS)]
    refused(L.gleam_dropout_fwd, [C.byref(d), FAKE[0], FAKE[1], FAKE[2], None, None],
            bad + [(0, changed(d, ld_res=11), gb.GLEAM_E_DIMS), (1, None, gb.GLEAM_E_NULL), (3, None, gb.GLEAM_E_NULL)])
    refused(L.gleam_dropout_bwd, [C.byref(d), FAKE[0], FAKE[1], None, None], bad + [(1, None, gb.GLEAM_E_NULL), (2, None, gb.GLEAM_E_NULL)])
    apart = gb.make_dropout(1, 10, 12, 0.1, 1, 2, ld=16, ld_res=20, ld_out=24)
    assert L.gleam_dropout_fwd(C.byref(apart), FAKE[0], FAKE[1], FAKE[0], None, None) == gb.GLEAM_E_DIMS
    assert L.gleam_dropout_fwd(C.byref(apart), FAKE[0], FAKE[1], FAKE[1], None, None) == gb.GLEAM_E_DIMS
    assert L.gleam_dropout_bwd(C.byref(apart), FAKE[0], FAKE[0], None, None) == gb.GLEAM_E_DIMS


def mix(B=2, T=300, P=1, H=4, heads=(4, 2, 1), dk=32, dv=48, dtype=torch.float32):
    q, k, v = (torch.empty(B, T, P, h, d, dtype=dtype) for h, d in zip(heads, (dk, dk, dv)))
    return gb.make_linattn(q, k, v, torch.empty(B, T, P, H, dv, dtype=dtype), 0.5)


def test_linattn_refusals():
    L, d = gb.lib(), mix()
    fwd, bwd = gb.gleam_linattn_workspace_bytes(d)
    assert bwd > 0 and fwd % 256 == 0 and bwd % 256 == 0
    S = gb.gleam_seq_strides
    bad = [(0, None, gb.GLEAM_E_NULL), (0, changed(d, dtype=2), gb.GLEAM_E_DESC), (0, changed(d, scale=float("inf")), gb.GLEAM_E_DESC)]
    bad += [(0, changed(d, **{f: v}), gb.GLEAM_E_DIMS) for f, v in (("dk", 0), ("dk", 129), ("dv", 0), ("dv", 129), ("heads", 0), ("q_heads", 3), ("k_heads", 0),
                                                                  ("v_heads", 8), ("B", 0), ("T", 0), ("P", -1), ("T", (1 << 30) + 1), ("B", 1 << 31), ("P", 1 << 28), ("P", 1 << 45),
                                                                  ("q", S(-1, 1, 1, 1)), ("k", S(1 << 45, 1, 1, 1)))]
    args = [C.byref(d), *FAKE[:3], FAKE[3], FAKE[4], FAKE[5], FAKE[6], FAKE[7], FAKE[8], 1 << 40, None]
    o = d.o
    refused(L.gleam_linattn_fwd, args, bad + [(i, None, gb.GLEAM_E_NULL) for i in (1, 2, 3, 4, 7)] + [(7, FAKE[0], gb.GLEAM_E_DIMS), (7, FAKE[2], gb.GLEAM_E_DIMS)] +
            [(0, changed(d, o=S(o.b, o.t, o.p, o.h - 1)), gb.GLEAM_E_DIMS),       # heads that overlap by an element
             (0, changed(d, o=S(o.b, 0, o.p, o.h)), gb.GLEAM_E_DIMS)])            # all tokens in one place
    args = [C.byref(d), *FAKE[:3], FAKE[3], FAKE[4], FAKE[5], FAKE[6], FAKE[7], *FAKE[8:11], FAKE[11], FAKE[12], bwd, None]
    q = d.q
    refused(L.gleam_linattn_bwd, args, bad + [(i, None, gb.GLEAM_E_NULL) for i in (1, 2, 3, 4, 7, 9, 10, 11, 13)] +
            [(9, FAKE[0], gb.GLEAM_E_DIMS), (10, FAKE[6], gb.GLEAM_E_DIMS), (11, FAKE[9], gb.GLEAM_E_DIMS), (14, bwd - 256, gb.GLEAM_E_WORKSPACE),
             (13, FAKE[12] + 64, gb.GLEAM_E_WORKSPACE), (12, FAKE[7], gb.GLEAM_E_DIMS), (12, FAKE[5], gb.GLEAM_E_DIMS), (0, changed(d, q=S(q.b, 0, q.p, q.h)), gb.GLEAM_E_DIMS)])
    n = C.c_size_t(0)
    assert L.gleam_linattn_workspace_bytes(C.byref(d), C.byref(n), None) == gb.GLEAM_E_NULL
    assert L.gleam_linattn_workspace_bytes(changed(d, T=0), C.byref(n), C.byref(n)) == gb.GLEAM_E_DIMS
    # arrays that are only read may repeat: one query for all tokens
    assert L.gleam_linattn_workspace_bytes(changed(d, q=S(q.b, 0, q.p, q.h)), C.byref(n), C.byref(n)) == gb.GLEAM_OK


def test_linattn_workspace_of_a_single_token_and_of_many_problems():
    assert gb.gleam_linattn_workspace_bytes(mix(T=1))[0] == 0
    assert gb.gleam_linattn_workspace_bytes(mix(T=64, P=500))[0] == 0
    short, long_ = mix(T=2048, heads=(4, 4, 4)), mix(T=4096, heads=(4, 4, 4))
    assert 0 < gb.gleam_linattn_workspace_bytes(short)[0] <= gb.gleam_linattn_workspace_bytes(long_)[0]


def test_binding_compares_arrays_with_the_description():
    d = gb.make_layer_norm(torch.float32, 4, 6)
    x = torch.empty(4, 6)
    with pytest.raises(ValueError):
        gb.gleam_layer_norm_fwd(d, x, None, None, x)                                  # not on the GPU
    with pytest.raises(ValueError):
        gb.gleam_layer_norm_fwd(d, torch.empty(4, 12)[:, :6], None, None, x)          # other strides
    with pytest.raises(ValueError):
        gb.make_layer_norm(torch.float16, 4, 6)
    q = torch.empty(1, 5, 1, 2, 8)
    with pytest.raises(ValueError):
        gb.make_linattn(q, q, q, torch.empty(1, 5, 1, 2, 9))
    with pytest.raises(ValueError):
        gb.make_linattn(q, q, q.bfloat16(), q)
    with pytest.raises(ValueError):
        gb.make_linattn(q[:, :4], q, q, q)
    with pytest.raises(ValueError):
        gb.make_linattn(q, q, q, torch.empty(1, 5, 1, 8, 2).transpose(3, 4))
    d = gb.make_linattn(q, q, q, q)
    a = torch.empty(2)
    with pytest.raises(ValueError):
        gb.gleam_linattn_fwd(d, q, torch.empty(1, 5, 1, 2, 16)[..., :8], q, a, None, None, q, None, None)
    with pytest.raises(ValueError):
        gb.gleam_linattn_fwd(d, q, q[..., :4], q, a, None, None, q, None, None)
