"""The layer of the example step by step, in 8-bit cells with a scale for K and another for V: what each call leaves is what the next one makes of it."""
import os
import sys
from types import SimpleNamespace

import pytest
import torch

import attention_ref as R
from test_gpu_attention import _check

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("e4m3", [True, False])
def test_cells_between_append_and_attention(e4m3):
    import attention_layer as E
    hidden, H, KH, D, page, T = 512, 4, 2, 128, 32, 75
    w, maps = E.make_weights(hidden, H, KH, D, 64, 0.5, seed=4)
    per = -(-T // page)
    layer = E.AttentionLayer(w, maps, H, KH, D, 64, per, page, T, T, e4m3=e4m3, scales=(0.02, 0.031))
    X = torch.randn(T, hidden, generator=torch.Generator().manual_seed(5)).cuda().to(torch.bfloat16)
    Y = torch.empty(T, hidden, device="cuda")
    table = torch.tensor([list(range(per))[::-1]], dtype=torch.int32, device="cuda")
    layer.forward(X, Y, E.batch([T], [T], table), T)
    torch.cuda.synchronize()
    rows, pages = {n: layer.rows[n][:T].cpu().double() for n in "qkv"}, table[0].long().cpu()
    scales = [s.cpu().double() if e4m3 else torch.ones(KH).double() for s in (layer.scales if e4m3 else (None, None))]
    k = (layer.k.cpu()[pages].double() * scales[0][:, None, None]).transpose(1, 2).reshape(-1, KH, D)[:T]
    v = (layer.v.cpu()[pages].double() * scales[1][:, None, None]).permute(0, 3, 1, 2).reshape(-1, KH, D)[:T]
    want_k, mag = R.rotated(rows["k"].view(T, KH, D), torch.ones(D), 1e-6, R.table_of(T, D), torch.arange(T), D, False)
    half, least = (R.E4M3_HALF, 2.0 ** -10) if e4m3 else (R.BF16_HALF, 0.0)          # half a step, and below the cells' normal range
    top = 448.0 if e4m3 else 3e38
    for got, want, size, scale in ((k, want_k, mag, scales[0]), (v, rows["v"].view(T, KH, D), rows["v"].view(T, KH, D).abs(), scales[1])):
        want = want.clamp(-top * scale[:, None], top * scale[:, None])
        assert ((got - want).abs() <= (half * want.abs()).clamp(min=least * scale.max()) + 60 * 2.0 ** -24 * size).all()
    Q, O = layer.Q[:T], layer.O[:T]
    _check(SimpleNamespace(T=T, D=D, KH=KH, n=[T], kv=[T], ks=[k], vs=[v]), Q.cpu(), H, O, None)
    # the output product: exact products, H D of them added in fp32
    o, wo = O.cpu().double(), w["o"].cpu().double()
    assert ((Y.cpu().double() - o @ wo.T).abs() <= H * D * 2.0 ** -24 * (o.abs() @ wo.abs().T) + 1e-30).all()
    # the test tells scales apart: with V's taken a fifth larger the same check fails
    with pytest.raises(AssertionError):
        _check(SimpleNamespace(T=T, D=D, KH=KH, n=[T], kv=[T], ks=[k], vs=[1.2 * v]), Q.cpu(), H, O, None)
