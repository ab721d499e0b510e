"""patch_kv_evict and patch_kv_evict4: which tokens stay, and every byte of the cache, against plain forms (tests/cache4_ref.py)."""
import numpy as np
import pytest
import torch

import cache4_ref as C
from paper_2509_23410_amd import binding as B

pytestmark = pytest.mark.gpu
CELLS = ["bf16", "e4m3", "e2m1"]


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _raw(b, cells):
    """(device bytes, host bytes, axis of the slots, bytes of a cell) of each buffer, as n_pages x KH x ... without what is between the pages."""
    KH, D, page = b.KH, b.D, b.page
    if cells == "e2m1":
        return list(zip(b.views(b.dk, b.dv, b.dsk, b.dsv), (x.clone() for x in b.views(b.pk, b.pv, b.sk, b.sv)), (2, 3, 2, 3), ("k", "v", "k_scale", "v_scale")))
    kind = torch.uint8 if cells == "e4m3" else torch.int16
    cut = lambda x, *shape: x.view(kind)[:, : KH * D * page].view(-1, *shape)  # noqa: E731
    return [(cut(b.dk, KH, page, D), cut(b.k, KH, page, D).clone(), 2, "k"), (cut(b.dv, KH, D, page), cut(b.v, KH, D, page).clone(), 3, "v")]


def _weights(b, seed, kind):
    g = torch.Generator().manual_seed(seed)
    stride = -(-max(b.max_kv, 1) // 4) * 4 + 8
    w = torch.exp(2 * torch.randn(len(b.n), b.KH, stride, generator=g) - 3)
    if kind == "ties":
        w = torch.randint(0, 3, w.shape, generator=g).float()
    elif kind == "equal":
        w = torch.full(w.shape, 0.25)
    elif kind == "odd":                                           # zeros of both signs, infinities, NaN, negative and denormal numbers
        pick = torch.tensor([0.0, -0.0, np.inf, -np.inf, np.nan, -1.0, 1e-42, -1e-42, 1.0, 2.0])
        w = pick[torch.randint(0, 10, w.shape, generator=g)]
    elif kind == "close":                                         # next to each other in fp32
        w = (torch.full(w.shape, 1.0).view(torch.int32) + torch.randint(0, 40, w.shape, generator=g, dtype=torch.int32)).view(torch.float32)
    return w, stride


def _evict(cells, *a, **kw):
    (B.patch_kv_evict4 if cells == "e2m1" else B.patch_kv_evict)(*a, _stream(), **kw)


def _check(b, cells, kv, w, stride, keep, sinks, recent, pos=None, in_place=False, max_kv=None, follows=True):
    n = len(kv)
    cache, seqs = b.on_gpu(B, **({} if max_kv is None else dict(max_kv=max_kv)))
    dw, dpos = w.cuda(), None if pos is None else pos.cuda()
    w_out = dw if in_place else torch.full_like(dw, 7.0)
    pos_out = dpos if in_place and pos is not None else torch.full(w.shape, -3, dtype=torch.int32).cuda()
    came, kv_out = torch.full((n, b.KH, keep), -9, dtype=torch.int32).cuda(), b.d[0] if in_place else torch.full((n,), -9, dtype=torch.int32).cuda()
    raw = _raw(b, cells)
    _evict(cells, seqs, cache, dw, w_out if follows else None, stride, keep, came, kv_out, sinks=sinks, recent=recent, positions=dpos, positions_out=pos_out if follows else None)
    torch.cuda.synchronize()
    want_w, want_pos = (w if in_place else torch.full_like(w, 7.0)).clone(), (pos if in_place and pos is not None else torch.full(w.shape, -3, dtype=torch.int32)).clone()
    bound = b.max_kv if max_kv is None else max_kv
    for s in range(n):
        L = 0 if kv[s] > bound else max(kv[s], 0)
        assert kv_out[s] == (kv[s] if kv[s] > bound else min(L, keep))
        for h in range(b.KH):
            f = C.evicted(w[s, h].numpy(), None if pos is None else pos[s, h].numpy(), L, keep, sinks, recent)
            assert np.array_equal(came[s, h].cpu().numpy(), f), (s, h)
            m = min(L, keep)
            if follows:
                want_w[s, h, :m] = w[s, h, f[:m]]
                want_pos[s, h, :m] = torch.from_numpy(f[:m].astype(np.int32)) if pos is None else pos[s, h, f[:m]]
            for i in range(m):
                dst, src = int(b.table[s, i // b.page]), int(b.table[s, f[i] // b.page])
                if f[i] != i and 0 <= dst < b.n_pages and 0 <= src < b.n_pages:
                    for _, host, axis, _ in raw:
                        host[dst, h].select(axis - 2, i % b.page).copy_(host[src, h].select(axis - 2, int(f[i]) % b.page))
    assert not follows or torch.equal(w_out.cpu().view(torch.int32), want_w.view(torch.int32)) and torch.equal(pos_out.cpu(), want_pos)
    for dev, host, _, name in raw:
        assert torch.equal(dev.cpu(), host), name
    return came, kv_out


CASES = [
    # kv, KH, D, page, keep, sinks, recent
    ([1], 1, 64, 16, 1, 0, 0), ([2], 1, 64, 16, 1, 0, 1), ([100, 17, 0, 64, 65], 2, 64, 16, 64, 4, 16), ([300, 301, 299], 3, 128, 64, 300, 0, 0), ([700, 90], 2, 256, 128, 33, 1, 5),
    ([130], 4, 128, 32, 129, 129, 0), ([130, 131], 1, 64, 256, 100, 0, 100), ([1000], 2, 64, 16, 999, 10, 989), ([50, 20], 1, 128, 16, 1000, 3, 3), ([513, 4097], 1, 64, 64, 512, 7, 100)]


@pytest.mark.parametrize("cells", CELLS)
@pytest.mark.parametrize("kv,KH,D,page,keep,sinks,recent", CASES)
def test_evict(kv, KH, D, page, keep, sinks, recent, cells):
    b = C.batch(cells, [1 if L else 0 for L in kv], kv, KH, D, page, seed=sum(kv), page_gap=512)
    w, stride = _weights(b, 1, "plain")
    _check(b, cells, kv, w, stride, keep, sinks, recent)
    # tokens in no order, and everything in place
    g = torch.Generator().manual_seed(2)
    pos = torch.stack([torch.randperm(stride, generator=g).int() * 2 + 1 for _ in range(len(kv) * KH)]).view(len(kv), KH, stride)
    _check(b, cells, kv, w, stride, keep, sinks, recent, pos=pos, in_place=True)
    _check(b, cells, kv, w, stride, keep, sinks, recent, pos=pos, follows=False)


@pytest.mark.parametrize("kind", ["ties", "equal", "odd", "close"])
def test_equal_and_odd_weights(kind):
    kv = [90, 400, 5000]
    b = C.batch("e4m3", [1, 1, 1], kv, 2, 64, 16, seed=3)
    w, stride = _weights(b, 5, kind)
    for keep, sinks, recent in ((89, 0, 0), (64, 4, 10), (1, 0, 0), (3000, 0, 500)):
        _check(b, "e4m3", kv, w, stride, keep, sinks, recent)
    pos = torch.randint(-5, 100, w.shape, generator=torch.Generator().manual_seed(1), dtype=torch.int32)      # the same one many times: more than the budget stay always
    for keep, sinks, recent in ((64, 60, 4), (10, 0, 10)):
        _check(b, "e4m3", kv, w, stride, keep, sinks, recent, pos=pos)


@pytest.mark.parametrize("cells,kv,keep,recent", [("bf16", [20000], 8192, 100), ("e2m1", [9000, 30000], 9001, 3000), ("e4m3", [70000], 69999, 0), ("e2m1", [40000], 100, 10)])
def test_long_ones(cells, kv, keep, recent):
    b = C.batch(cells, [1] * len(kv), kv, 1, 64, 256, seed=3)
    w, stride = _weights(b, 5, "plain")
    _check(b, cells, kv, w, stride, keep, 4, recent)


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "odd", "close", "few equal", "runs"])
def test_long_ones_of_any_weights(kind):
    """More slots than registers hold: the border between 16384 of the ranks, and where that does not find it (too many are equal, or weights lie in no order that those show)."""
    kv = [40000, 17000, 300]
    b = C.batch("e4m3", [1] * 3, kv, 1, 64, 256, seed=3)
    w, stride = _weights(b, 5, "plain" if kind in ("few equal", "runs") else kind)
    if kind == "few equal":                                       # 700 of one weight in the middle
        for s in (0, 1):
            at = w[s, 0, : kv[s]].sort().indices[kv[s] // 2:kv[s] // 2 + 700]
            w[s, 0, at] = w[s, 0, at[0]].clone()
    if kind == "runs":                                            # heavy where the sample of fours does not look, light where it does
        for s in (0, 1):
            fours = kv[s] // 4
            seen = (torch.arange(4096) * fours // 4096 * 4)[:, None] + torch.arange(4)
            w[s, 0, :] = 1000.0 + torch.arange(stride) % 997
            w[s, 0, seen.flatten()] = 1.0
    for keep, sinks, recent in ((8192, 4, 100), (20000, 0, 0), (16999, 0, 500), (1, 0, 0), (39999, 1, 7)):
        _check(b, "e4m3", kv, w, stride, keep, sinks, recent)
    g = torch.Generator().manual_seed(2)
    pos = torch.stack([torch.randperm(stride, generator=g).int() for _ in range(3)]).view(3, 1, stride)
    _check(b, "e4m3", kv, w, stride, 20000, 4, 3000, pos=pos, in_place=True)


def test_longer_than_bits_are_kept_for():
    b = C.batch("e2m1", [1], [220000], 1, 64, 256, seed=3)
    w, stride = _weights(b, 5, "plain")
    _check(b, "e2m1", [220000], w, stride, 90000, 4, 1000)
    b = C.batch("e2m1", [1], [212992], 1, 64, 256, seed=3)
    _check(b, "e2m1", [212992], w, stride, 212990, 4, 1000)


@pytest.mark.parametrize("cells", CELLS)
def test_pages_that_are_not_there_and_lengths_that_cannot_be(cells):
    kv = [100, 90, 300, 95]
    b = C.batch(cells, [1] * 4, kv, 2, 64, 16, seed=6)
    b.table[0, 5], b.table[1, 1], b.table[3, 0] = -1, b.n_pages, 1 << 30
    w, stride = _weights(b, 5, "plain")
    _check(b, cells, kv, w, stride, 50, 2, 10, max_kv=200)
    b.kv = kv = [100, -5, 300, 0]
    _check(b, cells, kv, w, stride, 50, 2, 10, max_kv=200)


def test_evicted_again_and_again_and_captured():
    """Four evictions in place as replays of one graph, weights changed between them, against the same calls."""
    kv = [300, 150, 40]
    b = C.batch("e2m1", [1] * 3, kv, 2, 128, 16, seed=9)
    w, stride = _weights(b, 5, "plain")
    came = torch.empty(3, 2, 64, dtype=torch.int32, device="cuda")
    states = []
    for way in ("calls", "graph"):
        cache, seqs = b.on_gpu(B)
        kv_len, dw, pos = b.d[0], w.cuda(), torch.arange(stride, dtype=torch.int32).repeat(3, 2, 1).cuda()
        run = lambda: _evict("e2m1", seqs, cache, dw, dw, stride, 64, came, kv_len, sinks=2, recent=8, positions=pos, positions_out=pos)  # noqa: E731
        if way == "graph":
            keep = [x.clone() for x in (b.dk, b.dv, b.dsk, b.dsv, kv_len, dw, pos)]
            run()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                run()
            for x, y in zip((b.dk, b.dv, b.dsk, b.dsv, kv_len, dw, pos), keep):
                x.copy_(y)
        seen = []
        for i in range(4):
            torch.cuda.synchronize()
            graph.replay() if way == "graph" else run()
            seen += [x.clone() for x in (b.dk, b.dv, b.dsk, b.dsv, kv_len, dw, pos, came)]
            dw.mul_(torch.linspace(0.5 + i, 2.0, stride, device="cuda"))
            kv_len.add_(torch.tensor([3, 1, 30], dtype=torch.int32, device="cuda"))     # more tokens came
            pos[:, :, 64:100] = 1000 * (i + 1) + torch.arange(36, dtype=torch.int32, device="cuda")
        states.append(seen)
    assert all(torch.equal(x, y) for x, y in zip(*states))


def test_cells_beyond_4_gb():
    KH, D, page = 8, 128, 64
    cells = KH * page * D
    n_pages = (9 << 30) // (2 * cells)
    b = C.batch("bf16", [1, 1], [200, 70], KH, D, page, seed=13)
    cache, seqs = b.on_gpu(B)
    k, v = (torch.empty(n_pages, cells, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    where = [n_pages - 1 - 7 * i for i in range(b.n_pages)]
    for i, p in enumerate(where):
        k[p], v[p] = b.dk[i], b.dv[i]
    moved = torch.tensor([[where[p] if p >= 0 else -1 for p in r] for r in b.table.tolist()], dtype=torch.int32, device="cuda")
    far = B.KVCache(k, v, n_pages, page, KH, D)
    w, stride = _weights(b, 5, "plain")
    outs = [(torch.empty(2, KH, 50, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")) for _ in range(2)]
    _evict("bf16", seqs, cache, w.cuda(), None, stride, 50, *outs[0])
    _evict("bf16", B.Seqs(2, b.T, b.d[0], moved, b.table.shape[1], 1, b.max_kv, q_start=b.d[2]), far, w.cuda(), None, stride, 50, *outs[1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    for i, p in enumerate(where):
        assert torch.equal(k[p].view(torch.int16), b.dk[i].view(torch.int16)) and torch.equal(v[p].view(torch.int16), b.dv[i].view(torch.int16))
