"""patch_kv_append4 with its rows in place (out is x: bf16, the same strides): the same pages and rows, bit for bit, as with rows of their own."""
import pytest
import torch

import attention_ref as R
import cache4_ref as C
from paper_2509_23410_amd import binding as B

pytestmark = pytest.mark.gpu


def _stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,kv,KH", [([1, 1, 3, 1], [90, 33, 2, 0], 2), ([70, 1, 130, 9], [100, 1, 90, 300], 3), ([300, 40, 0, 65], [411, 17, 5, 65], 2)])   # few; runs of tokens: tiles of V
def test_rows_in_place(n, kv, KH, D, interleaved):
    H, n_pos = 2 * KH, 700
    b = C.Batch4(n, kv, KH, D, 16, seed=5)
    g = torch.Generator().manual_seed(9)
    T = b.T + 2                                                   # and two rows behind the last sequence's, which nobody has
    x = (3 * torch.randn(T, (H + 2 * KH) * D, generator=g)).to(torch.bfloat16)
    gamma, table = (1 + 0.5 * torch.randn(D, generator=g)).cuda(), R.table_of(n_pos, D).cuda()
    rope, row = B.Rope(table, n_pos, D, interleaved=interleaved), x.shape[1]
    results = []
    for in_place in (False, True):
        cache, _ = b.on_gpu(B)
        seqs = B.Seqs(len(n), T, b.d[0], b.d[1], b.table.shape[1], b.max_q, b.max_kv, q_start=b.d[2])
        dx = x.cuda()
        y = dx if in_place else torch.full_like(dx, 7.0)
        part = lambda first, heads, gam=None: B.Heads(dx.data_ptr() + 2 * first * D, heads, row, f32=False, gamma=gam, out=y.data_ptr() + 2 * first * D, out_stride=row)  # noqa: E731
        B.patch_kv_append4(part(H, KH, gamma), part(H + KH, KH), seqs, cache, _stream(), rope=rope, q=part(0, H, gamma))
        torch.cuda.synchronize()
        results.append([y.cpu().view(torch.int16)] + [t.cpu() for t in (b.dk, b.dv, b.dsk, b.dsv)])
    for one, other, what in zip(*results, ("rows", "k", "v", "k_scale", "v_scale")):
        assert torch.equal(one, other), what
    # what came out is what went in, normed, rotated and in cells; rows without a place are zero
    place = torch.cat([torch.cat([torch.arange(L - m, L) for m, L in zip(n, kv)]), torch.tensor([-1, -1])])
    rows = results[1][0].view(torch.bfloat16).double()
    assert (rows[place < 0] == 0).all()
    value = C.encode(x[:, (H + KH) * D:].reshape(T, KH, D))[2].view(T, -1)
    assert torch.equal(rows[place >= 0, (H + KH) * D:], value[place >= 0])
