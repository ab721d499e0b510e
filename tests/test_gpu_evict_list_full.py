"""Heads so long that the list of those near the border may run out: whichever way the border is found then, the same tokens stay."""
import numpy as np
import pytest
import torch

from paper_2509_23410_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("length,keep,positions", [(205000, 102500, False), (212992, 106496, False), (212989, 100000, True), (212993, 106496, False), (180000, 90001, True)])
def test_who_stays(length, keep, positions):
    KH, D, page, stride = 8, 64, 256, -(-length // 4) * 4
    g = torch.Generator().manual_seed(length)
    w = torch.exp(2 * torch.randn(1, KH, stride, generator=g) - 3)
    pos = torch.stack([torch.randperm(stride, generator=g).int() for _ in range(KH)])[None] if positions else None
    dw, dpos = w.cuda(), None if pos is None else pos.cuda()
    pages = -(-length // page)
    byte = lambda *shape: torch.zeros(*shape, device="cuda", dtype=torch.uint8)  # noqa: E731
    held = [byte(pages, KH, page, D // 2), byte(pages, KH, D // 2, page), byte(pages, KH, page, D // 32), byte(pages, KH, D // 32, page)]
    kv_len, table = torch.tensor([length], dtype=torch.int32, device="cuda"), torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    came, left = torch.empty(1, KH, keep, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    out = torch.full_like(dw, 7.0)
    B.patch_kv_evict4(B.Seqs(1, 1, kv_len, table, pages, 1, length), B.KVCache4(*held, pages, page, KH, D), dw, out, stride, keep, came, left,
                      torch.cuda.current_stream().cuda_stream, sinks=4, recent=1000, positions=dpos)
    torch.cuda.synchronize()
    assert left.item() == keep
    for h in range(KH):
        p = np.arange(length) if pos is None else pos[0, h, :length].numpy()
        always = (p < 4) | (p > p.max() - 1000)
        order = np.lexsort((np.arange(length), np.where(always, 0, -w[0, h, :length].numpy().astype(np.float64)), ~always))
        stays = np.zeros(length, bool)
        stays[order[:keep]] = True
        want = np.arange(keep)
        want[~stays[:keep]] = keep + np.flatnonzero(stays[keep:])
        assert np.array_equal(came[0, h].cpu().numpy(), want), h
        assert torch.equal(out[0, h, :keep].cpu(), w[0, h, want])
