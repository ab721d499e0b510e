"""patch_attention_weights and patch_attention_weights4 against plain 64-bit forms (tests/cache4_ref.py)."""
import numpy as np
import pytest
import torch

import cache4_ref as C
from paper_2509_23410_amd import binding as B

pytestmark = pytest.mark.gpu


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _weigh(b, cells, *a, **kw):
    (B.patch_attention_weights4 if cells == "e2m1" else B.patch_attention_weights)(*a, _stream(), **kw)


def _inputs(b, H, seed=1, stride=None, amplitude=1.0):
    g = torch.Generator().manual_seed(seed)
    Q = (amplitude * torch.randn(b.T, H * b.D, generator=g)).to(torch.bfloat16)
    stride = stride or -(-max(b.max_kv, 1) // 4) * 4
    W = torch.rand(len(b.n), b.KH, stride, generator=g)
    return Q, W, stride


def _lse(b, Q, H, scale):
    """What attention would say, rounded to fp32."""
    lse, t = torch.full((b.T, H), -np.inf), 0
    for s in range(len(b.n)):
        for i in range(b.n[s]):
            seen = b.kv[s] - b.n[s] + i + 1
            if seen > 0:
                z = Q[t].double().view(b.KH, -1, b.D) @ b.ks[s][:seen].double().permute(1, 2, 0) * scale
                lse[t] = torch.logsumexp(z, -1).flatten().float()
            t += 1
    return lse


CASES = [
    # n, kv, H, KH, D, page
    ([1], [1], 1, 1, 64, 16), ([1], [500], 14, 2, 64, 16), ([1, 1, 1, 1], [31, 32, 33, 0], 32, 8, 128, 64), ([1, 1, 1], [1000, 3, 257], 8, 8, 128, 32),
    ([1, 0, 1], [700, 50, 2100], 4, 2, 256, 128), ([1] * 9, [600, 601, 640, 700, 513, 514, 900, 1, 0], 40, 2, 128, 64), ([5] * 3, [300, 310, 205], 10, 2, 128, 16),
    ([4, 0, 7, 1], [40, 17, 300, 60], 16, 1, 128, 32), ([3, 2], [300, 299], 14, 2, 64, 256), ([8, 3], [3, 3], 4, 2, 128, 16), ([33, 1, 20], [33, 90, 100], 8, 2, 64, 16),
    ([130], [130], 2, 1, 128, 64), ([90, 150, 7], [200, 150, 500], 4, 1, 256, 64), ([270, 40], [600, 333], 3, 3, 128, 32), ([257], [1300], 2, 2, 256, 256),
    ([64, 300], [64, 20], 6, 2, 64, 16),
    # enough blocks of keys for rows through LDS
    ([40, 33, 70, 65] * 9, [40, 100, 200, 65] * 9, 8, 4, 64, 16), ([40, 0, 70, 129] * 9, [140, 100, 200, 65] * 9, 12, 4, 128, 64), ([33, 20] * 20, [330, 60] * 20, 4, 4, 256, 32)]


@pytest.mark.parametrize("cells", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("n,kv,H,KH,D,page", CASES)
def test_weights(n, kv, H, KH, D, page, cells):
    b = C.batch(cells, n, kv, KH, D, page, seed=sum(kv))
    scale = D ** -0.5
    Q, W, stride = _inputs(b, H)
    lse = _lse(b, Q, H, scale)
    cache, seqs = b.on_gpu(B)
    for decay, gap in ((1.0, 0), (0.9, 8)):
        dQ = torch.full((b.T, H * D + gap), 9.0, device="cuda", dtype=torch.bfloat16)
        dQ[:, : H * D] = Q.cuda()
        dW, out = W.cuda(), torch.full_like(W, 7.0).cuda()
        print(f"weights n={n[:4]} kv={kv[:4]} H={H} KH={KH} D={D} page={page} {cells}", flush=True)
        _weigh(b, cells, dQ, H, seqs, cache, lse.cuda(), dW, out, stride, decay=decay, q_stride=H * D + gap)
        want, off = C.weights(b, Q, H, lse, W, decay, scale)
        got = out.cpu().double()
        for s in range(len(n)):
            L = max(kv[s], 0) if n[s] else 0
            assert (got[s, :, L:] == 7).all()
            over = (got[s, :, :L] - want[s, :, :L]).abs() - off[s, :, :L]
            assert L == 0 or (not got[s, :, :L].isnan().any() and over.max() <= 0), (s, over.max())
        # in place, and the same bits
        _weigh(b, cells, dQ, H, seqs, cache, lse.cuda(), dW, dW, stride, decay=decay, q_stride=H * D + gap)
        assert torch.equal(torch.where(out == 7, W.cuda(), out), dW)


@pytest.mark.parametrize("n,kv", [([1, 2], [300, 77]), ([90, 2], [120, 200])])
def test_arguments(n, kv):
    for cells in ("bf16", "e2m1"):
        b = C.batch(cells, n, kv, 2, 128, 32, seed=7, page_gap=1024)
        for scale, amplitude, max_kv, max_q in ((0.3, 1.0, 250, 100), (-0.2, 3.0, 100000, 1000), (0.0, 8.0, 201, 300)):
            Q, W, stride = _inputs(b, 4, amplitude=amplitude, stride=max(max_kv, 200) + 1000 & ~3)
            lse = _lse(b, Q, 4, scale or 128 ** -0.5)
            cache, seqs = b.on_gpu(B, max_kv=max_kv, max_q=max_q)
            out, place = torch.full_like(W, 7.0).cuda(), torch.full(W.shape, -3, dtype=torch.int32).cuda()
            pos = torch.arange(b.T, dtype=torch.int32) * 3 + 100
            _weigh(b, cells, Q.cuda(), 4, seqs, cache, lse.cuda(), W.cuda(), out, stride, scale=scale, positions=pos.cuda(), slot_positions=place)
            want, off = C.weights(b, Q, 4, lse, W, 1.0, scale or 128 ** -0.5)
            t = 0
            for s in range(2):
                if kv[s] > max_kv:                               # longer than was said: it stays as it is
                    assert (out[s] == 7).all() and (place[s] == -3).all()
                    t += n[s]
                    continue
                assert ((out[s, :, : kv[s]].cpu().double() - want[s, :, : kv[s]]).abs() <= off[s, :, : kv[s]]).all() and (out[s, :, kv[s]:] == 7).all()
                at = place[s].cpu()
                assert (at[:, : kv[s] - n[s]] == -3).all() and (at[:, kv[s] - n[s]:kv[s]] == pos[t:t + n[s]]).all() and (at[:, kv[s]:] == -3).all()
                t += n[s]


@pytest.mark.parametrize("n,kv", [([2, 1], [100, 40]), ([60, 1], [100, 40])])
def test_rows_that_saw_nothing_and_keys_that_are_not_there(n, kv):
    """A row whose lse is minus infinity adds nothing, a NaN is a NaN for what it sees; keys without a page are NaN, and no others; a sequence that is too long stays."""
    for cells in ("bf16", "e4m3", "e2m1"):
        b = C.batch(cells, n + [1], kv + [500], 2, 64, 16, seed=6)
        Q, W, stride = _inputs(b, 4, stride=512)
        lse = _lse(b, Q, 4, 0.125)
        lse[0] = -np.inf                                          # the first sequence's first token
        good = b.table.copy()
        b.table[0, 2], b.table[1, 1] = -1, b.n_pages
        cache, seqs = b.on_gpu(B, max_kv=100)
        out = torch.full_like(W, 7.0).cuda()
        _weigh(b, cells, Q.cuda(), 4, seqs, cache, lse.cuda(), W.cuda(), out, stride)
        b.table = good
        want, off = C.weights(b, Q, 4, lse, W, 1.0, 0.125)
        got = out.cpu().double()
        missing = torch.zeros(3, 512, dtype=torch.bool)
        missing[0, 32:48] = missing[1, 16:32] = True
        for s in (0, 1):
            assert torch.equal(got[s, :, : kv[s]].isnan(), missing[s, None, : kv[s]].expand(2, -1))
            fine = ~missing[s, : kv[s]]
            assert ((got[s, :, : kv[s]] - want[s, :, : kv[s]]).abs() <= off[s, :, : kv[s]])[:, fine].all()
        assert (got[2] == 7).all()
        # NaN: of the last row of the first sequence, which sees all its keys
        t = n[0] - 1
        lse[t, 1] = float("nan")
        cache, seqs = b.on_gpu(B, max_kv=100)
        _weigh(b, cells, Q.cuda(), 4, seqs, cache, lse.cuda(), W.cuda(), out, stride)
        got = out.cpu()
        assert got[0, 0, : kv[0]].isnan().all() and not got[0, 1, : kv[0]].isnan().any() and not got[1, :, : kv[1]].isnan().any()


def test_keys_that_are_not_finite_are_nobody_else_s():
    for n in (1, 50):
        b = C.batch("bf16", [n], [150], 2, 64, 16, seed=8)
        cells = 2 * 16 * 64
        for value in (float("nan"), float("inf")):
            p, old = b.table[0, 5], b.k.clone()
            b.k[p, :cells].view(2, 16, 64)[:, 3] = value             # key 83
            Q, W, stride = _inputs(b, 2)
            lse = _lse(b, Q, 2, 0.125)
            cache, seqs = b.on_gpu(B)
            out = torch.full_like(W, 7.0).cuda()
            _weigh(b, "bf16", Q.cuda(), 2, seqs, cache, lse.cuda(), W.cuda(), out, stride)
            b.k = old
            want, off = C.weights(b, Q, 2, lse, W, 1.0, 0.125)
            others = [j for j in range(150) if j != 83]
            assert ((out[0, :, :150].cpu().double() - want[0, :, :150]).abs() <= off[0, :, :150])[:, others].all()
            if value != value:
                assert out[0, :, 83].isnan().all()


def test_after_attention_and_captured():
    """Attention and the weights of its rows as a graph, replayed with the program's own work between: bit-equal to the same calls, and new weights sum to the rows."""
    for cells in ("bf16", "e2m1"):
        n, kv, H, KH, D = [1] * 5 + [40], [600, 300, 257, 1, 64, 333], 8, 2, 128
        b = C.batch(cells, n, kv, KH, D, 16, seed=11)
        cache, seqs = b.on_gpu(B)
        attend = B.patch_attention4 if cells == "e2m1" else B.patch_attention
        size = (B.patch_attention4_workspace_bytes if cells == "e2m1" else B.patch_attention_workspace_bytes)(H, seqs, cache)
        ws = torch.empty(size, device="cuda", dtype=torch.uint8)
        Q = torch.randn(b.T, H * D, device="cuda").to(torch.bfloat16)
        O, lse, W = torch.empty_like(Q), torch.empty(b.T, H, device="cuda"), torch.zeros(len(n), KH, 600, device="cuda")
        out = torch.zeros_like(W)

        def step():
            attend(Q, H, seqs, cache, O, _stream(), lse=lse, workspace=ws)
            _weigh(b, cells, Q, H, seqs, cache, lse, W, out, 600)

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for i in range(4):
            Q.copy_(torch.randn(b.T, H * D, device="cuda").to(torch.bfloat16))
            out.zero_()
            step()
            want = out.clone()
            # each row's weights sum to one: fp32 sums of some thousand terms, each some 2^-18 off at scores of up to 8 here
            total = want.double().sum(-1).cpu()
            rows = torch.tensor(n)[:, None] * (H // KH)
            assert ((total - rows).abs() <= rows * 2.0 ** -14).all()
            out.fill_(5.0)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for s in range(len(n)):
                assert torch.equal(out[s, :, : kv[s]], want[s, :, : kv[s]]) and (out[s, :, kv[s]:] == 5).all()
