"""The 4-bit cache and the weights in batches as a program with fixed sizes describes them (rows of nobody in front and behind, idle sequences, bounds that are not close), and all
four calls captured, replayed and on another stream."""
import numpy as np
import pytest
import torch

import cache4_ref as C
from paper_2509_23410_amd import binding as B
from test_gpu_cache4 import _check, _pages_after, _same_pages

pytestmark = pytest.mark.gpu


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _padded(b, lead, trail, wide=3, max_q=None, max_kv=None):
    """(cache, seqs, rows of the call): `lead` rows in front of the batch's tokens and `trail` behind, a table `wide` columns wider."""
    b.table = np.concatenate([b.table, np.full((len(b.n), wide), -7, np.int32)], 1)
    cache, _ = b.on_gpu(B)
    rows = lead + b.T + trail
    b.start = torch.as_tensor(b.q_start + lead).cuda()
    return cache, B.Seqs(len(b.n), rows, b.d[0], b.d[1], b.table.shape[1], max_q or b.max_q, max_kv or b.max_kv, q_start=b.start), rows


CASES = [([1, 1], [40, 33], 2, 3, 6, 2, 64, 16, 0), ([0, 2, 1], [50, 700, 300], 5, 0, 8, 8, 128, 32, 0), ([0, 0, 1, 2], [90, 80, 77, 500], 3, 1, 4, 1, 128, 16, 64),
         ([33, 0, 20], [33, 5, 100], 7, 40, 4, 2, 64, 16, 0), ([0, 50, 33], [100, 150, 99], 20, 9, 2, 1, 256, 64, 70), ([130], [130], 300, 1, 2, 2, 128, 64, 0),
         ([300, 0, 7], [411, 100, 70], 20, 30, 4, 2, 64, 16, 0)]


@pytest.mark.parametrize("n,kv,lead,trail,H,KH,D,page,prefix", CASES)
def test_rows_of_nobody(n, kv, lead, trail, H, KH, D, page, prefix):
    b = C.Batch4(n, kv, KH, D, page, prefix=prefix, seed=71)
    cache, seqs, rows = _padded(b, lead, trail, max_q=b.max_q + 9, max_kv=b.max_kv + page)
    mine = slice(lead, lead + b.T)
    nobody = torch.ones(rows, dtype=torch.bool)
    nobody[mine] = False
    # attention and weights
    Q = torch.randn(b.T, H * D, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    dQ = torch.full((rows, H * D), float("nan"), device="cuda", dtype=torch.bfloat16)
    dQ[mine] = Q.cuda()
    O, lse = torch.full((rows, H * D), 7.0, device="cuda", dtype=torch.bfloat16), torch.full((rows, H), 7.0, device="cuda")
    ws = torch.empty(B.patch_attention4_workspace_bytes(H, seqs, cache, prefix_len=prefix) + 16, device="cuda", dtype=torch.uint8)
    B.patch_attention4(dQ, H, seqs, cache, O, _stream(), prefix_len=prefix, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    assert (O.cpu()[nobody] == 7).all() and (lse.cpu()[nobody] == 7).all()
    _check(b, Q, H, O[mine], lse[mine])
    stride = b.max_kv + page + 3 & ~3
    W = torch.rand(len(n), KH, stride, generator=torch.Generator().manual_seed(2))
    out = torch.full_like(W, 7.0).cuda()
    B.patch_attention_weights4(dQ, H, seqs, cache, lse, W.cuda(), out, stride, _stream(), decay=0.5)
    want, off = C.weights(b, Q, H, lse[mine].cpu(), W, 0.5, D ** -0.5)
    for s in range(len(n)):
        L = kv[s] if n[s] else 0
        assert (out[s, :, L:] == 7).all() and ((out[s, :, :L].cpu().double() - want[s, :, :L]).abs() <= off[s, :, :L]).all()
    # append: rows of nobody are not in the cache, and zero where rows come back
    x = torch.randn(rows, 2 * KH * D, generator=torch.Generator().manual_seed(3))
    dx = x.cuda()
    outs = [torch.full((rows, KH * D), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    part = lambda i: B.Heads(dx.data_ptr() + 4 * i * KH * D, KH, 2 * KH * D, f32=True, out=outs[i], out_stride=KH * D)  # noqa: E731
    B.patch_kv_append4(part(0), part(1), seqs, cache, _stream())
    torch.cuda.synchronize()
    k, v = (C.encode(x[mine, i * KH * D:(i + 1) * KH * D].reshape(b.T, KH, D)) for i in (0, 1))
    _pages_after(b, n, kv, k[0], k[1], v[0], v[1])
    _same_pages(b)
    placed = torch.zeros(rows, dtype=torch.bool)
    placed[mine] = torch.cat([torch.arange(L - m, L) for m, L in zip(n, kv)]) >= 0
    for out, want in ((outs[0], k[2]), (outs[1], v[2])):
        assert (out.cpu()[~placed] == 0).all() and torch.equal(out[mine].cpu().double()[placed[mine]], want.view(b.T, -1)[placed[mine]])


def test_all_four_captured_and_on_another_stream():
    """A step of a decoder with a budget as one graph, replayed with the program's own work between, and on a stream of its own: bit for bit what the calls give."""
    n, H, KH, D, page, keep, stride = 3, 8, 2, 128, 16, 48, 64
    g = torch.Generator(device="cuda").manual_seed(5)
    rows = [torch.randn(n, (H + 2 * KH) * D, device="cuda", generator=g) for _ in range(6)]

    def state():
        b = C.Batch4([1] * n, [48, 30, 17], KH, D, page, seed=12)
        b.table = np.arange(4 * n, dtype=np.int32).reshape(n, 4)
        b.pk, b.pv, b.sk, b.sv = (torch.cat([x] * 4)[: 4 * n].contiguous() for x in (b.pk, b.pv, torch.full_like(b.sk, 126), torch.full_like(b.sv, 125)))
        b.n_pages, b.max_kv = 4 * n, stride
        cache, seqs = b.on_gpu(B)
        s = dict(b=b, cache=cache, seqs=seqs, x=torch.empty_like(rows[0]), W=torch.rand(n, KH, stride, device="cuda", generator=torch.Generator(device="cuda").manual_seed(6)),
                 pos=torch.tensor([100, 60, 40], dtype=torch.int32, device="cuda"), slots=torch.arange(stride, dtype=torch.int32, device="cuda").repeat(n, KH, 1),
                 Q=torch.zeros(n, H * D, device="cuda", dtype=torch.bfloat16), O=torch.zeros(n, H * D, device="cuda", dtype=torch.bfloat16), lse=torch.zeros(n, H, device="cuda"),
                 came=torch.zeros(n, KH, keep, dtype=torch.int32, device="cuda"), ws=torch.empty(1 << 22, device="cuda", dtype=torch.uint8))
        return s

    def step(s):
        st, part = _stream(), lambda first, heads, **kw: B.Heads(s["x"].data_ptr() + 4 * first * D, heads, s["x"].shape[1], f32=True, **kw)  # noqa: E731
        B.patch_kv_append4(part(H, KH), part(H + KH, KH), s["seqs"], s["cache"], st, q=part(0, H, out=s["Q"], out_stride=H * D))
        B.patch_attention4(s["Q"], H, s["seqs"], s["cache"], s["O"], st, lse=s["lse"], workspace=s["ws"])
        B.patch_attention_weights4(s["Q"], H, s["seqs"], s["cache"], s["lse"], s["W"], s["W"], stride, st, decay=0.9, positions=s["pos"], slot_positions=s["slots"])
        B.patch_kv_evict4(s["seqs"], s["cache"], s["W"], s["W"], stride, keep, s["came"], s["b"].d[0], st, sinks=2, recent=4, positions=s["slots"], positions_out=s["slots"])

    def seen(s):
        torch.cuda.synchronize()
        return [t.clone() for t in (s["b"].dk, s["b"].dv, s["b"].dsk, s["b"].dsv, s["b"].d[0], s["W"], s["slots"], s["O"], s["lse"], s["came"])]

    def go(s, run):
        got = []
        for x in rows:
            s["x"].copy_(x)
            s["b"].d[0].add_(1)                                    # the new token
            run()
            got.append(seen(s))
            s["pos"].add_(1)
        return got

    s = state()
    want = go(s, lambda: step(s))
    assert want[-1][4].tolist() == [48, 36, 23] and torch.isfinite(want[-1][7].float()).all()
    s = state()
    keep_state = [t.clone() for t in (s["b"].dk, s["b"].dv, s["b"].dsk, s["b"].dsv, s["b"].d[0], s["W"], s["slots"])]
    s["x"].copy_(rows[0])
    step(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s)
    for t, was in zip((s["b"].dk, s["b"].dv, s["b"].dsk, s["b"].dsv, s["b"].d[0], s["W"], s["slots"]), keep_state):
        t.copy_(was)
    for got, was in zip(go(s, graph.replay), want):
        assert all(torch.equal(x, y) for x, y in zip(got, was))
    s, other = state(), torch.cuda.Stream()

    def aside():
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            step(s)
        torch.cuda.current_stream().wait_stream(other)

    for got, was in zip(go(s, aside), want):
        assert all(torch.equal(x, y) for x, y in zip(got, was))
