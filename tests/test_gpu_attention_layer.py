"""The example that runs products, append and attention together, against the same layer in 64 bits without a cache."""
import os
import sys

import pytest
import torch

import attention_ref as R

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("hidden,heads,kv_heads,head_dim,page,shared,own,e4m3", [
    (512, 8, 2, 64, 16, 100, (7, 1, 33, 20), False), (256, 4, 4, 128, 64, 64, (3, 70), False), (512, 4, 1, 128, 32, 45, (1, 9, 2), True)])
def test_layer(hidden, heads, kv_heads, head_dim, page, shared, own, e4m3):
    import attention_layer as E
    steps = 3
    X0, X, got, w = E.run(hidden, heads, kv_heads, head_dim, 64, 0.5, page, shared, own, steps, e4m3=e4m3, seed=3)
    got, w = got.cpu().double(), {n: x.cpu().double() for n, x in w.items()}
    want = []
    for x in X:
        x = torch.cat([X0, x]).cpu().double()
        T = x.shape[0]
        pos = torch.arange(T)
        table = R.table_of(T, head_dim)
        q, k, v = (x @ w[n].T for n in "qkv")
        q = R.rotated(q.view(T, heads, head_dim), torch.ones(head_dim), 1e-6, table, pos, head_dim, False)[0][-1:]
        k = R.rotated(k.view(T, kv_heads, head_dim), torch.ones(head_dim), 1e-6, table, pos, head_dim, False)[0]
        # the last row is all that is asked for: one token that sees every key
        o = R.attention(q, [k], [v.view(T, kv_heads, head_dim)], heads // kv_heads, head_dim ** -0.5, [1], [T])[0]
        want.append(o.view(-1) @ w["o"].T)
    want = torch.stack(want)
    # Roundings on the way, each of half a step: q and k (which turn a score, here at most about 3, by as much of itself), p, v and the attention's result.  The
    # products' sums are fp32.  In e4m3 k and v have half a step of that type.
    cell = R.E4M3_HALF if e4m3 else R.BF16_HALF
    bound = 3 * (R.BF16_HALF + cell) + R.BF16_HALF + cell + R.BF16_HALF
    rel = float((got - want).norm() / want.norm())
    print(f"layer hidden={hidden} heads={heads}/{kv_heads}x{head_dim} e4m3={e4m3}: relF={rel:.2e}, bound {bound:.2e}", flush=True)
    assert rel <= bound
