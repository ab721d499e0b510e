"""Batches as a program with fixed sizes describes them: rows that no sequence has in front and behind, idle sequences, bounds that are not close."""
import numpy as np
import torch

import attention_ref as R
from paper_2509_23410_amd import binding as B
from test_gpu_attention import _check, _rope_bound

FILL = 7.0


class Padded:
    """A Batch of attention_ref, `lead` rows of nobody in front of its tokens and `trail` behind, a page table `wide` columns wider than it has to be."""

    def __init__(self, n, kv, KH, D, page, lead=0, trail=0, wide=0, max_q=None, max_kv=None, **kw):
        self.b = b = R.Batch(n, kv, KH, D, page, **kw)
        self.lead, self.rows = lead, lead + b.T + trail
        if wide:
            b.table = np.concatenate([b.table, np.full((len(n), wide), -7, np.int32)], 1)
        self.max_q, self.max_kv = max_q or b.max_q, b.max_kv if max_kv is None else max_kv

    def on_gpu(self):
        b = self.b
        cache, _ = b.on_gpu(B)
        self.start = torch.as_tensor(b.q_start + self.lead).cuda()
        return cache, B.Seqs(len(b.n), self.rows, b.d[0], b.d[1], b.table.shape[1], self.max_q, self.max_kv, q_start=self.start)

    def attend(self, H, prefix=None, workspace="all", seed=1):
        """(Q of the tokens, O and lse of all rows), the rows of nobody being NaN in Q.  workspace: all that the call would like, half of it, or none."""
        b = self.b
        Q = torch.randn(b.T, H * b.D, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)
        cache, seqs = self.on_gpu()
        dQ = torch.full((self.rows, H * b.D), float("nan"), device="cuda", dtype=torch.bfloat16)
        dQ[self.lead:self.lead + b.T] = Q.cuda()
        O, lse = torch.full((self.rows, H * b.D), FILL, device="cuda", dtype=torch.bfloat16), torch.full((self.rows, H), FILL, device="cuda")
        prefix = b.prefix if prefix is None else prefix
        need = B.patch_attention_workspace_bytes(H, seqs, cache, prefix_len=prefix)
        size = dict(all=need, half=need // 2, none=0)[workspace]
        ws = torch.full((size // 4 + 1024,), float("nan"), device="cuda")
        B.patch_attention(dQ, H, seqs, cache, O, torch.cuda.current_stream().cuda_stream, prefix_len=prefix, lse=lse, workspace=ws if size else None, workspace_bytes=size)
        torch.cuda.synchronize()
        assert ws[size // 4:].isnan().all()
        return Q, O, lse

    def check_attention(self, H, prefix=None, workspace="all", skip=()):
        b = self.b
        Q, O, lse = self.attend(H, prefix, workspace)
        mine = slice(self.lead, self.lead + b.T)
        nobody = torch.ones(self.rows, dtype=torch.bool)
        nobody[mine] = False
        assert (O.cpu()[nobody] == FILL).all() and (lse.cpu()[nobody] == FILL).all()      # left as they are
        if b.T > len(skip):
            _check(b, Q, H, O[mine], lse[mine], skip=skip)
        return O[mine], lse[mine]

    def check_append(self, H=0, rot=0, seed=9):
        """Every token's cells hold its K and V (in bf16), every other cell what it held; Q of rows without a place is zero."""
        b, kv, g = self.b, self.b.kv, torch.Generator().manual_seed(seed)
        KH, D, page = b.KH, b.D, b.page
        row = (H + 2 * KH) * D
        x = (3 * torch.randn(self.rows, row, generator=g)).to(torch.bfloat16)
        table = R.table_of(max(self.max_kv, 1), rot) if rot else None
        cache, seqs = self.on_gpu()
        dx, dtable = x.cuda(), None if table is None else table.cuda()
        q_out = torch.full((self.rows, max(H, 1) * D), FILL, device="cuda", dtype=torch.bfloat16)
        part = lambda first, heads, **kw: B.Heads(dx.data_ptr() + first * D * 2, heads, row, **kw)  # noqa: E731
        B.patch_kv_append(part(H, KH), part(H + KH, KH), seqs, cache, torch.cuda.current_stream().cuda_stream,
                          rope=B.Rope(dtable, table.shape[0], rot) if rot else None, q=part(0, H, out=q_out, out_stride=H * D) if H else None)
        torch.cuda.synchronize()
        cells = KH * page * D
        want_k, want_v = b.k.clone(), b.v.clone()
        got_k, got_v, q_out = b.dk.cpu(), b.dv.cpu(), q_out.cpu()
        t, placed = self.lead, torch.zeros(self.rows, dtype=torch.bool)
        for s in range(len(b.n)):
            for pos in range(kv[s] - b.n[s], kv[s]):
                if pos >= 0:
                    placed[t] = True
                    p, slot = b.table[s, pos // page], pos % page
                    y, mag = R.rotated(x[t:t + 1, H * D:(H + KH) * D].reshape(1, KH, D), None, 0, table, torch.tensor([pos]), rot, False)
                    k = got_k[p, :cells].view(KH, page, D)[:, slot]
                    assert ((k.double() - y[0]).abs() <= _rope_bound(y[0], mag[0])).all(), (s, pos)
                    want_k[p, :cells].view(KH, page, D)[:, slot] = k
                    want_v[p, :cells].view(KH, D, page)[:, :, slot] = x[t, (H + KH) * D:].view(KH, D)
                    if H:
                        y, mag = R.rotated(x[t:t + 1, : H * D].reshape(1, H, D), None, 0, table, torch.tensor([pos]), rot, False)
                        assert ((q_out[t].double().view(H, D) - y[0]).abs() <= _rope_bound(y[0], mag[0])).all(), (s, pos)
                t += 1
        bits = lambda a: a.view(torch.int16)  # noqa: E731
        assert torch.equal(bits(got_k), bits(want_k)) and torch.equal(bits(got_v), bits(want_v))
        assert not H or (q_out[~placed] == 0).all()
