"""The temporal layer (layer norm, projections, linear attention, dropout and residual) against the same layer of the float64 oracle's
parts: output, gradients, frames one by one, lengths.  Tolerances: float32 products of 3 x 48 terms and the operators' own 1e-5; bfloat16
rounds q, k, v, o, z, h (forward) and as many gradients, each by 2^-8 / sqrt 3 in the root mean square at most, of which a result sees ten
or fewer in a row: sqrt(10) 2^-8 / sqrt 3 = 7.1e-3, asked for 2^-6 = 1.6e-2."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from paper_2207_08393_amd import binding as gb
from paper_2207_08393_amd.temporal import TemporalLayer
from tests.gpu_util import rel_l2

pytestmark = pytest.mark.gpu


def host(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def oracle(layer, x, g, lengths, mask, factor):
    """h, g_x and the parameters' gradients of the layer at these values."""
    B, T, P, C = layer.shape
    H, d, scale = layer.H, layer.d, layer.d ** -0.5
    low = (lambda w: host(w.to(layer.dtype)))
    gamma, beta, wq, wo, a = host(layer.gamma), host(layer.beta), low(layer.w_qkv), low(layer.w_o), host(layer.log_decay)
    rows = x.reshape(-1, C)
    y, mean, rstd = lo.layer_norm(rows, gamma, beta, 1e-5)
    qkv = (y @ wq.T).reshape(B, T, P, 3, H, d)
    q, k, v = (qkv[:, :, :, i] for i in range(3))
    o, _ = lo.linattn(q, k, v, a, scale, lengths)
    z = o.reshape(-1, C) @ wo.T
    h = rows + np.where(mask, factor * z, 0.0)
    g = g.reshape(-1, C)
    gz = np.where(mask, factor * g, 0.0)
    gq, gk, gv, _ = lo.linattn_bwd(q, k, v, a, scale, (gz @ wo).reshape(B, T, P, H, d), lengths)
    gqkv = np.stack([gq, gk, gv], 3).reshape(-1, 3 * C)
    gx, gg, gb_ = lo.layer_norm_bwd(rows, gamma, mean, rstd, gqkv @ wq)
    return h, g + gx, gg, gb_, gqkv.T @ y, gz.T @ o.reshape(-1, C)


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 2.0 ** -6)], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,lengths", [(9, None), (70, None), (20, [20, 11])])
def test_temporal_layer(T, lengths, dtype, tol):
    print("case temporal", T, lengths, dtype, flush=True)
    B, P, C, p = 2, 3, 48, 0.25
    layer = TemporalLayer(B, T, P, C, 4, dtype=dtype, dropout=p, seed=5)
    layer.step += 7
    gen = torch.Generator().manual_seed(T)
    x = torch.randn(B, T, P, C, generator=gen).cuda().to(dtype)
    g = torch.randn(B, T, P, C, generator=gen).cuda().to(dtype)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    h = host(layer.forward(x, n)).reshape(-1, C)
    gx = host(layer.backward(g)).reshape(-1, C)
    mask, factor = lo.dropout_mask(B * T * P, C, p, 5, 7)
    ref = oracle(layer, host(x), host(g), lengths, mask, factor)
    got = (h, gx, host(layer.g_gamma), host(layer.g_beta), host(layer.g_qkv_w), host(layer.g_o_w))
    for name, a, b in zip(("h", "g_x", "g_gamma", "g_beta", "g_w_qkv", "g_w_o"), got, ref):
        assert rel_l2(a, b) <= tol, (name, rel_l2(a, b))


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 2.0 ** -6)], ids=["f32", "bf16"])
def test_temporal_layer_frame_by_frame(dtype, tol):
    B, T, P, C = 1, 25, 7, 32
    layer = TemporalLayer(B, T, P, C, 2, dtype=dtype, dropout=0.5, seed=1)
    x = torch.randn(B, T, P, C, generator=torch.Generator().manual_seed(3)).cuda().to(dtype)
    whole = host(layer.forward(x, training=False))
    for _ in range(2):                                                 # a second series starts from nothing again
        layer.restart()
        frames = np.stack([host(layer.frame(x[:, t].contiguous())) for t in range(T)], 1)
        assert rel_l2(frames, whole) <= tol


def test_temporal_layer_learns():
    B, T, P, C = 1, 12, 64, 32
    layer, hyper = TemporalLayer(B, T, P, C, 2, dtype=torch.float32, dropout=0.0), gb.make_adam(5e-3)
    x = torch.randn(B, T, P, C, generator=torch.Generator().manual_seed(3)).cuda()
    target = torch.cumsum(x, 1) / torch.arange(1, T + 1, device="cuda")[None, :, None, None]
    losses = []
    for k in range(1, 41):
        d = layer.forward(x) - target
        losses.append(float((d * d).mean()))
        layer.backward(2.0 / d.numel() * d)
        layer.update(hyper, k)
    assert losses[-1] < 0.3 * losses[0], losses
