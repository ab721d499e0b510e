"""patch_attention_weights over pages beyond 4 GB, rows and weights that lie far apart, and one token each without q_start: the same bits as with everything near."""
import pytest
import torch

import cache4_ref as C
import test_gpu_weights as W
from paper_2509_23410_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cells", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("n,kv", [([1, 1], [200, 70]), ([90, 3], [200, 70]), ([150] * 20, [330] * 20)])       # few rows, more over few keys, rows through LDS
def test_pages_beyond_4_gb(n, kv, cells):
    H, KH, D, page = 8, 8, 128, 64
    b = C.batch(cells, n, kv, KH, D, page, seed=13)
    Q, w, stride = W._inputs(b, H)
    lse = W._lse(b, Q, H, D ** -0.5).cuda()
    cache, seqs = b.on_gpu(B)
    dQ, dw = Q.cuda(), w.cuda()
    near = torch.full_like(dw, 7.0)
    W._weigh(b, cells, dQ, H, seqs, cache, lse, dw, near, stride, decay=0.5)
    held = [b.dk] if cells != "e2m1" else [b.dk, b.dsk]
    row = held[0].shape[1] * held[0].element_size()
    n_pages = (9 << 30) // row
    far = [torch.empty(n_pages, x.shape[1], device="cuda", dtype=x.dtype) for x in held]
    where = [n_pages - 1 - 7 * i for i in range(b.n_pages)]
    for i, p in enumerate(where):
        for x, y in zip(far, held):
            x[p] = y[i]
    moved = torch.tensor([[where[p] if p >= 0 else -1 for p in r] for r in b.table.tolist()], dtype=torch.int32, device="cuda")
    seqs = B.Seqs(len(n), b.T, b.d[0], moved, b.table.shape[1], b.max_q, b.max_kv, q_start=b.d[2])
    if cells == "e2m1":
        cache = B.KVCache4(far[0], far[0], far[1], far[1], n_pages, page, KH, D)
    else:
        cache = B.KVCache(far[0], far[0], n_pages, page, KH, D, e4m3=cells == "e4m3", k_scale=b.d[3], v_scale=b.d[4])
    got = torch.full_like(dw, 7.0)
    W._weigh(b, cells, dQ, H, seqs, cache, lse, dw, got, stride, decay=0.5)
    assert torch.equal(got, near)


def test_one_token_each_without_q_start():
    b = C.batch("e2m1", [1] * 5, [100, 0, 300, 64, 1], 2, 64, 16, seed=2)
    Q, w, stride = W._inputs(b, 6)
    lse = W._lse(b, Q, 6, 0.125).cuda()
    outs = []
    for q_start in (True, False):
        cache, seqs = b.on_gpu(B, q_start=q_start)
        outs.append(torch.full_like(w, 7.0).cuda())
        W._weigh(b, "e2m1", Q.cuda(), 6, seqs, cache, lse, w.cuda(), outs[-1], stride)
    assert torch.equal(*outs) and (outs[0][1] == 7).all() and (outs[0][0, :, :100] != 7).all()


def test_rows_and_weights_far_apart():
    """Rows 2^20 values apart and weights 2^26 (both beyond 2^31 bytes): few rows and many."""
    for n, kv in (([1, 1, 1], [90, 33, 70]), ([1200], [1200])):
        b = C.batch("bf16", n, kv, 12, 64, 16, seed=2)
        Q, w, stride = W._inputs(b, 12)
        lse = W._lse(b, Q, 12, 0.125).cuda()
        cache, seqs = b.on_gpu(B)
        dw, gap, far = w.cuda(), 1 << 20, 1 << 26
        near = torch.full_like(dw, 7.0)
        W._weigh(b, "bf16", Q.cuda(), 12, seqs, cache, lse, dw, near, stride)
        wide = torch.empty(b.T, gap, device="cuda", dtype=torch.bfloat16)
        wide[:, : 12 * 64] = Q.cuda()
        held = torch.empty(len(n), 12, far, device="cuda")
        held[:, :, :stride] = dw
        W._weigh(b, "bf16", wide, 12, seqs, cache, lse, held, held, far, q_stride=gap)
        for s, L in enumerate(kv):
            assert torch.equal(held[s, :, :L], near[s, :, :L]) and torch.equal(held[s, :, L:stride], dw[s, :, L:stride])
        del wide, held
