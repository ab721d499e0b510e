"""patch_attention_weights and patch_attention_weights4: a row whose lse is minus infinity adds nothing, whatever its query is and whatever keys it would have met."""
import numpy as np
import pytest
import torch

import cache4_ref as C
import test_gpu_weights as W
from paper_2509_23410_amd import binding as B

pytestmark = pytest.mark.gpu

SHAPES = [
    # n, kv, H, KH, D, page, the sequence none of whose rows adds anything
    ([3, 1, 2, 1], [100, 40, 300, 70], 4, 2, 64, 16, 1), ([5, 4], [1200, 40], 6, 1, 128, 32, 1), ([2, 3], [90, 300], 8, 2, 256, 64, 0),       # few rows
    ([90, 40], [120, 40], 4, 2, 64, 16, 1), ([700, 33], [700, 333], 4, 2, 128, 32, 1), ([150, 20], [150, 200], 2, 1, 256, 64, 1),             # more over few keys
    ([40, 33, 70, 65] * 9, [40, 100, 200, 65] * 9, 8, 4, 64, 16, 5), ([40, 3, 70, 129] * 9, [140, 100, 200, 65] * 9, 12, 4, 128, 64, 3),       # rows through LDS
    ([33, 20] * 20, [330, 60] * 20, 4, 4, 256, 32, 7)]


def _poison_key(b, cells, s, j):
    """Key j of sequence s becomes NaN in the pages (not in what the plain form sees)."""
    p, slot, KH, D, page = int(b.table[s, j // b.page]), j % b.page, b.KH, b.D, b.page
    if cells == "e2m1":
        b.views(b.pk, b.pv, b.sk, b.sv)[2][p, :, slot] = 255
    else:
        b.k.view(torch.uint8 if cells == "e4m3" else torch.int16)[p, : KH * page * D].view(KH, page, D)[:, slot] = 0x7F if cells == "e4m3" else 0x7FC0


@pytest.mark.parametrize("cells", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("n,kv,H,KH,D,page,silent", SHAPES)
def test_rows_that_are_out(n, kv, H, KH, D, page, silent, cells):
    b = C.batch(cells, n, kv, KH, D, page, seed=sum(kv))
    Q, w, stride = W._inputs(b, H)
    lse = W._lse(b, Q, H, D ** -0.5)
    out = torch.rand(b.T, H, generator=torch.Generator().manual_seed(4)) < 0.2
    for s in range(len(n)):
        out[b.q_start[s + 1] - 1] = True                          # the only rows that see the last key
        _poison_key(b, cells, s, kv[s] - 1)
    out[b.q_start[silent]:b.q_start[silent + 1]] = True
    lse[out] = -np.inf
    bad = Q.view(b.T, H, D).clone()
    bad[out] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0]).to(torch.bfloat16).repeat(D // 4)
    good = b.table.copy()
    b.table[silent, 0] = -1                                       # nor does a page that is not there matter to rows that add nothing
    cache, seqs = b.on_gpu(B)
    b.table = good
    got = torch.full_like(w, 7.0).cuda()
    print(f"rows out n={n[:4]} kv={kv[:4]} H={H} KH={KH} D={D} {cells}", flush=True)
    W._weigh(b, cells, bad.view(b.T, H * D).cuda(), H, seqs, cache, lse.cuda(), w.cuda(), got, stride, decay=0.75)
    want, off = C.weights(b, Q, H, lse, w, 0.75, D ** -0.5)
    got = got.cpu().double()
    for s in range(len(n)):
        L = kv[s]
        assert (got[s, :, L:] == 7).all() and not got[s, :, :L].isnan().any(), s
        assert ((got[s, :, :L] - want[s, :, :L]).abs() <= off[s, :, :L]).all(), s
        assert (got[s, :, L - 1] == 0).all()
    old = max(kv[silent] - n[silent], 0)
    assert torch.equal(got[silent, :, :old], (w[silent, :, :old] * 0.75).double()) and (got[silent, :, old:kv[silent]] == 0).all()
