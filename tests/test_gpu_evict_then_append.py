"""A cache of bf16 or e4m3 cells that tokens were evicted from, and a new token behind them: patch_kv_append rotates by the slot, so patch_qk_rope turns Q and K by their
positions first, and the append has them without a rotation."""
import numpy as np
import pytest
import torch

import attention_ref as R
import cache4_ref as C
from paper_2509_23410_amd import binding as B
from test_gpu_cache4 import _check

pytestmark = pytest.mark.gpu


def _stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("cells", ["bf16", "e4m3"])
@pytest.mark.parametrize("H,KH,D,page", [(4, 2, 64, 16), (3, 1, 128, 32), (4, 2, 256, 16)])
def test_a_token_behind_an_eviction(H, KH, D, page, cells):
    kv, keep, n_pos, width = [90, 70], 40, 500, (H + 2 * KH) * D
    b = C.batch(cells, [1, 1], kv, KH, D, page, seed=3)
    cache, seqs = b.on_gpu(B)
    stride = 96
    w = torch.rand(2, KH, stride, generator=torch.Generator().manual_seed(1)).cuda()
    came, kv_len = torch.empty(2, KH, keep, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    slots = torch.full((2, KH, stride), -1, dtype=torch.int32, device="cuda")
    B.patch_kv_evict(seqs, cache, w, w, stride, keep, came, kv_len, _stream(), sinks=2, recent=8, positions_out=slots)
    kv_len.add_(1)
    qkv = torch.randn(2, width, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    positions, table = torch.tensor(kv, dtype=torch.int32), R.table_of(n_pos, D)
    dx, dtable, Q, K = qkv.cuda(), table.cuda(), torch.empty(2, H * D, device="cuda", dtype=torch.bfloat16), torch.empty(2, KH * D, device="cuda", dtype=torch.bfloat16)
    part = lambda first, heads, **kw: B.Heads(dx.data_ptr() + 2 * first * D, heads, width, **kw)  # noqa: E731
    one = torch.arange(3, dtype=torch.int32, device="cuda")
    seqs = B.Seqs(2, 2, kv_len, b.d[1], b.table.shape[1], 1, keep + 1, q_start=one)
    O, lse = torch.empty_like(Q), torch.empty(2, H, device="cuda")
    B.patch_qk_rope(part(0, H, out=Q, out_stride=H * D), part(H, KH, out=K, out_stride=KH * D), positions.cuda(), 2, D, B.Rope(dtable, n_pos, D), _stream())
    B.patch_kv_append(B.Heads(K, KH, KH * D), part(H + KH, KH), seqs, cache, _stream())
    B.patch_attention(Q, H, seqs, cache, O, _stream(), lse=lse)
    B.patch_attention_weights(Q, H, seqs, cache, lse, w, w, stride, _stream(), positions=positions.cuda(), slot_positions=slots)
    torch.cuda.synchronize()
    # the new cells: K turned by its position, not by its slot (rounded to bf16, then to the cell), V as it is
    x, mag = R.rotated(qkv[:, H * D:(H + KH) * D].reshape(2, KH, D), None, 0, table, positions, D, False)
    v = qkv[:, (H + KH) * D:].reshape(2, KH, D).double()
    scales = [torch.ones(KH).double() if s is None else s.double() for s in (b.k_scale, b.v_scale)]
    cut = lambda t, *shape: t.cpu()[:, : KH * page * D].view(-1, *shape)  # noqa: E731
    ks, vs = cut(b.dk, KH, page, D), cut(b.dv, KH, D, page)
    came = came.cpu().long()
    for s in range(2):
        p, slot = int(b.table[s, keep // page]), keep % page
        k_new, v_new = ks[p, :, slot].double() * scales[0][:, None], vs[p, :, :, slot].double() * scales[1][:, None]
        first = R.BF16_HALF * x[s].abs() + 40 * 2.0 ** -24 * mag[s] * (1 + R.BF16_HALF)
        cell = lambda y, scale: 0.0 if cells == "bf16" else R.E4M3_HALF * y.abs() * (1 + R.BF16_HALF) + 2.0 ** -10 * scale[:, None]  # noqa: E731  (below 2^-6 steps of 2^-9)
        assert ((k_new - x[s]).abs() <= first * (1 + R.E4M3_HALF) + cell(x[s].abs() + first, scales[0])).all()
        assert ((v_new - v[s]).abs() <= cell(v[s], scales[1])).all()
        rows = torch.arange(KH)
        b.ks[s] = torch.cat([b.ks[s][came[s].T, rows], k_new[None]])
        b.vs[s] = torch.cat([b.vs[s][came[s].T, rows], v_new[None]])
    b.kv = [keep + 1, keep + 1]
    _check(b, Q.cpu(), H, O, lse)
    at = slots.cpu()
    assert torch.equal(at[:, :, :keep].long(), came) and (at[:, :, keep] == positions[:, None]).all() and (at[:, :, keep + 1:] == -1).all()
    new = w.cpu()[:, :, keep]
    z = torch.einsum("thd,thd->th", Q.cpu().double().view(2, H, D), torch.stack([b.ks[s][-1].repeat_interleave(H // KH, 0) for s in range(2)])) * D ** -0.5
    want = torch.exp(z - lse.cpu().double()).view(2, KH, -1).sum(-1)
    assert ((new - want).abs() <= want * 2.0 ** -16).all()       # scores of up to some 2^4, their products' sums and exponents off by some 2^-21 of that
