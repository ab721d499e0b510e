"""patch_qk_rope, patch_kv_append and patch_attention against plain 64-bit forms (tests/attention_ref.py)."""
import numpy as np
import pytest
import torch

import attention_ref as R
from paper_2509_23410_amd import binding as B

pytestmark = pytest.mark.gpu


def _stream():
    return torch.cuda.current_stream().cuda_stream


# ---- norm and rotation ------------------------------------------------------------------------------------------------

# One rounding to bf16 of the result, and before it some 20 operations in fp32 (the mean of up to 256 squares in pairs, the root, the factors, the angle,
# a difference): each off by 2^-24 of what went into it.
def _rope_bound(y, mag):
    return R.BF16_HALF * y.abs() + 40 * 2.0 ** -24 * mag * (1 + R.BF16_HALF)


@pytest.mark.parametrize("T,H,KH,D,rot,interleaved,f32,norm,gap", [
    (1, 14, 2, 64, 64, False, True, True, 0), (1, 1, 0, 64, 8, False, False, False, 0), (3, 32, 8, 128, 128, False, True, True, 8), (257, 5, 3, 128, 64, True, False, True, 0),
    (33, 4, 1, 256, 256, True, True, True, 24), (65, 8, 4, 256, 72, False, False, False, 16), (130, 40, 40, 128, 128, False, False, True, 0), (1000, 3, 7, 64, 24, True, True, False, 8),
    (77, 9, 1, 128, 0, False, True, True, 0)])
def test_qk_rope(T, H, KH, D, rot, interleaved, f32, norm, gap):
    g = torch.Generator().manual_seed(T + H)
    kind = torch.float32 if f32 else torch.bfloat16
    row = (H + KH) * D + gap
    x = torch.randn(T, row, generator=g).mul_(torch.exp(torch.randn(T, row, generator=g))).to(kind)
    gam = [1 + 0.5 * torch.randn(D, generator=g) if norm else None for _ in range(2)]
    n_pos = 70000
    table = R.table_of(n_pos, rot) if rot else None
    pos = torch.randint(0, n_pos, (T,), generator=g, dtype=torch.int32)
    pos[-1] = n_pos - 1
    dx, dpos, dgam, dtable = x.cuda(), pos.cuda(), [None if v is None else v.cuda() for v in gam], None if table is None else table.cuda()
    q_out, k_out = torch.full((T, H * D + 8), 7.0, device="cuda", dtype=torch.bfloat16), torch.full((T, max(KH, 1) * D + 16), 7.0, device="cuda", dtype=torch.bfloat16)
    q = B.Heads(dx, H, row, f32=f32, gamma=dgam[0], out=q_out, out_stride=H * D + 8)
    k = B.Heads(dx.data_ptr() + H * D * dx.element_size(), KH, row, f32=f32, gamma=dgam[1], out=k_out, out_stride=KH * D + 16) if KH else None
    rope = B.Rope(dtable, n_pos, rot, interleaved=interleaved, eps=1e-5) if rot else None
    B.patch_qk_rope(q, k, dpos, T, D, rope, _stream())
    torch.cuda.synchronize()
    for out, first, heads, gamma in ((q_out, 0, H, gam[0]), (k_out, H, KH, gam[1])):
        if heads:
            y, mag = R.rotated(x[:, first * D:(first + heads) * D].reshape(T, heads, D), gamma, 1e-5 if rot else 1e-6, table, pos, rot, interleaved)
            got = out[:, : heads * D].cpu().double().view(T, heads, D)
            over = (got - y).abs() - _rope_bound(y, mag)
            assert over.max() <= 0, over.max()
        assert (out[:, heads * D:] == 7).all()


def test_qk_rope_in_place_and_without_a_place():
    T, H, D = 50, 6, 128
    g = torch.Generator().manual_seed(3)
    x = torch.randn(T, H * D, generator=g).to(torch.bfloat16)
    table = R.table_of(64, D)
    pos = torch.arange(T, dtype=torch.int32)
    pos[5], pos[6], pos[7], pos[8], pos[9] = -1, 64, -(1 << 31), (1 << 31) - 1, 63
    dx, dt = x.cuda(), table.cuda()
    B.patch_qk_rope(B.Heads(dx, H, H * D, out=dx, out_stride=H * D), None, pos.cuda(), T, D, B.Rope(dt, 64, 128), _stream())
    y, mag = R.rotated(x.view(T, H, D), None, 0, table, pos, D, False)
    got = dx.cpu().double().view(T, H, D)
    assert (got[[5, 7]] == 0).all() and got[[6, 8]].isnan().all()
    fine = [i for i in range(T) if i not in (5, 6, 7, 8)]
    assert ((got - y).abs() - _rope_bound(y, mag))[fine].max() <= 0


def test_qk_rope_of_extreme_heads():
    """Zeros, a single huge value, infinities and NaN: a head's own affair."""
    x = torch.zeros(6, 128)
    x[1, 3], x[2, 5], x[3, 7] = 1e15, float("inf"), float("nan")
    x[4] = 1e-20
    x[5] = torch.arange(128)
    dx, out = x.cuda(), torch.empty(6, 128, device="cuda", dtype=torch.bfloat16)
    B.patch_qk_rope(B.Heads(dx, 1, 128, f32=True, gamma=torch.ones(128, device="cuda"), out=out, out_stride=128), None, torch.zeros(6, device="cuda", dtype=torch.int32), 6, 128, None, _stream())
    got = out.cpu().double()
    assert (got[0] == 0).all() and abs(got[1, 3] - 128 ** 0.5) < 128 ** 0.5 * (R.BF16_HALF + 2e-6) and got[1].abs().sum() == got[1, 3].abs()
    assert got[2].isnan().any() and got[3].isnan().all()
    want = x[5].double() / torch.sqrt((x[5].double() ** 2).mean() + 1e-6)
    assert ((got[5] - want).abs() <= want.abs() * (R.BF16_HALF + 2e-6)).all() and (got[4].abs() <= 1.01e-17).all()


# ---- append -----------------------------------------------------------------------------------------------------------

APPENDS = [
    # n, kv, KH, D, page, prefix, e4m3, H, f32, norm, rot, interleaved, gap
    ([1], [1], 2, 64, 16, 0, False, 14, True, True, 64, False, 0), ([1, 1, 1], [17, 16, 5], 8, 128, 64, 0, False, 0, False, False, 0, False, 64),
    ([1] * 5, [100, 33, 1, 64, 65], 3, 128, 32, 33, True, 6, True, True, 128, False, 0), ([5, 0, 3, 70], [5, 40, 130, 70], 2, 128, 16, 0, False, 4, False, True, 64, True, 16),
    ([40, 129, 1], [300, 129, 1], 2, 256, 128, 0, True, 2, True, False, 256, True, 32), ([3, 2, 4], [2, 0, 9], 2, 64, 256, 0, False, 2, True, True, 16, False, 0),
    ([200], [1000], 5, 64, 64, 512, True, 0, False, False, 64, False, 0), ([17, 64, 63], [80, 64, 127], 1, 128, 16, 0, True, 1, False, True, 8, False, 0),
    # enough tokens for tiles of V, and (the last two) for several heads a thread
    ([300, 7, 64], [411, 7, 64], 2, 64, 16, 0, False, 3, True, True, 64, False, 0), ([130, 200], [100, 333], 3, 128, 32, 0, True, 0, False, False, 0, False, 32),
    ([256], [256], 1, 256, 256, 0, False, 4, False, True, 256, True, 0), ([65, 300, 1], [200, 300, 40], 2, 256, 64, 0, True, 0, True, False, 64, False, 0),
    ([9] * 40, [100 + 3 * i for i in range(40)], 2, 64, 128, 64, False, 0, False, False, 64, False, 16), ([1100], [1203], 7, 256, 128, 0, False, 12, True, True, 128, False, 0),
    ([600, 450], [600, 777], 9, 128, 64, 0, True, 24, False, True, 128, True, 0)]


@pytest.mark.parametrize("n,kv,KH,D,page,prefix,e4m3,H,f32,norm,rot,interleaved,gap", APPENDS)
def test_kv_append(n, kv, KH, D, page, prefix, e4m3, H, f32, norm, rot, interleaved, gap):
    b = R.Batch(n, kv, KH, D, page, prefix=prefix, e4m3=e4m3, seed=len(n) + D, page_gap=gap)
    g = torch.Generator().manual_seed(9)
    T, kind = b.T, torch.float32 if f32 else torch.bfloat16
    row = (H + 2 * KH) * D + 16
    x = (3 * torch.randn(T, row, generator=g)).to(kind)
    x[0, H * D + KH * D] = 1e4     # beyond the range of e4m3 cells
    gam = [1 + 0.5 * torch.randn(D, generator=g) if norm else None for _ in range(2)]
    table = R.table_of(b.max_kv, rot) if rot else None
    cache, seqs = b.on_gpu(B)
    dx, dgam, dtable = x.cuda(), [None if v is None else v.cuda() for v in gam], None if table is None else table.cuda()
    part = lambda first, heads, **kw: B.Heads(dx.data_ptr() + first * D * dx.element_size(), heads, row, f32=f32, **kw)  # noqa: E731
    q_out = torch.full((T, H * D), 7.0, device="cuda", dtype=torch.bfloat16)
    q = part(0, H, gamma=dgam[0], out=q_out, out_stride=H * D) if H else None
    B.patch_kv_append(part(H, KH, gamma=dgam[1]), part(H + KH, KH), seqs, cache, _stream(), rope=B.Rope(dtable, b.max_kv, rot, interleaved=interleaved) if rot else None, q=q)
    torch.cuda.synchronize()
    pos = torch.cat([torch.arange(L - m, L) for m, L in zip(n, kv)])
    want_k, mag_k = R.rotated(x[:, H * D:(H + KH) * D].reshape(T, KH, D), gam[1], 1e-6, table, pos, rot, interleaved)
    ksc = torch.ones(KH) if b.k_scale is None else b.k_scale
    vsc = torch.ones(KH) if b.v_scale is None else b.v_scale
    got_k, got_v = b.dk.cpu(), b.dv.cpu()
    cells = KH * page * D
    same_k, same_v = torch.ones(b.n_pages, cells, dtype=torch.bool).view(b.n_pages, KH, page, D), torch.ones(b.n_pages, cells, dtype=torch.bool).view(b.n_pages, KH, D, page)
    seq = np.repeat(np.arange(len(n)), n)
    for t in range(T):
        p = int(pos[t])
        if p < 0:
            if H:
                assert (q_out[t] == 0).all()
            continue
        pg, slot = b.table[seq[t], p // page], p % page
        k = got_k[pg, :cells].view(KH, page, D)[:, slot].double()
        v = got_v[pg, :cells].view(KH, D, page)[:, :, slot].float()
        same_k[pg, :, slot], same_v[pg, :, :, slot] = False, False
        fv = x[t, (H + KH) * D:(H + 2 * KH) * D].view(KH, D).float()
        if e4m3:
            w, m = want_k[t] / ksc.double()[:, None], mag_k[t] / ksc.double()[:, None]
            w = w.clamp(-448, 448)
            # a rounding to e4m3 (half a step: 2^-4 of the value, 2^-10 below its normal range) after fp32 work
            assert ((k - w).abs() <= (R.E4M3_HALF * w.abs()).clamp(min=2.0 ** -10) + 60 * 2.0 ** -24 * m).all()
            assert torch.equal(v, (fv / vsc[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).float())
        else:
            assert ((k - want_k[t]).abs() <= _rope_bound(want_k[t], mag_k[t])).all()
            assert torch.equal(v, fv.to(torch.bfloat16).float())
    bits = lambda a: a.view(torch.uint8 if e4m3 else torch.int16)  # noqa: E731
    for got, was, same in ((got_k, b.k, same_k), (got_v, b.v, same_v)):
        flat = torch.ones(b.n_pages, b.stride, dtype=torch.bool)
        flat[:, :cells] = same.reshape(b.n_pages, cells)
        assert torch.equal(bits(got)[flat], bits(was)[flat])        # nothing else is touched
    if H:
        y, mag = R.rotated(x[:, : H * D].reshape(T, H, D), gam[0], 1e-6, table, pos, rot, interleaved)
        there = pos >= 0
        assert ((q_out.cpu().double().view(T, H, D) - y).abs() - _rope_bound(y, mag))[there].max() <= 0


def test_kv_append_writes_nothing_where_there_is_no_page():
    b = R.Batch([2, 2, 2, 2], [33, 34, 35, 500], 2, 64, 16, seed=4)       # positions 31 and 32, 32 and 33, 33 and 34, 498 and 499
    written = sorted([[int(b.table[0, 1]), 15], [int(b.table[2, 2]), 1], [int(b.table[2, 2]), 2]])
    b.table[0, 2], b.table[1, 2] = -1, b.n_pages
    cache, seqs = b.on_gpu(B, max_kv=40)              # the last sequence is longer than the caller said
    x = torch.ones(8, 2 * 64, device="cuda")
    B.patch_kv_append(B.Heads(x, 2, 128, f32=True), B.Heads(x, 2, 128, f32=True), seqs, cache, _stream())
    torch.cuda.synchronize()
    was, got = b.k.view(torch.int16), b.dk.cpu().view(torch.int16)
    changed = (was != got).view(b.n_pages, 2, 16, 64).any(-1).any(1).nonzero().tolist()
    assert sorted(changed) == written
    changed = (b.v.view(torch.int16) != b.dv.cpu().view(torch.int16)).view(b.n_pages, 2, 64, 16).any(2).any(1).nonzero().tolist()
    assert sorted(changed) == written


# ---- attention --------------------------------------------------------------------------------------------------------


def _check(b, Q, H, got, lse, scale=None, skip=()):
    """Of a result sum p v / sum p: each p is off by one rounding to bf16 and by what its score is off (the products of bf16 are exact, D of them are added in
    fp32; e4m3 values too, times a scale); the result is rounded to bf16 once.  The sums are fp32: 2^-24 of what is in them for each of some hundred additions."""
    D, G = b.D, H // b.KH
    scale = D ** -0.5 if scale is None else scale
    o, want_lse, av, qk = R.attention(Q.view(b.T, H, D).float(), b.ks, b.vs, G, scale, b.n, b.kv)
    score = (2 * D + 16) * 2.0 ** -24 * qk + 2.0 ** -20
    bound = R.BF16_HALF * o.abs() + (av * (R.BF16_HALF + 2 * score[..., None] + 256 * 2.0 ** -24)) * (1 + R.BF16_HALF)
    rows = [t for t in range(b.T) if t not in skip]
    got = got.cpu().double().view(b.T, H, D)
    over = ((got - o).abs() - bound)[rows]
    assert not got[rows].isnan().any() and over.max() <= 0, (over.max(), over.argmax())
    if lse is not None:
        lse, empty = lse.cpu().double(), want_lse == -np.inf
        assert (lse[rows][empty[rows]] == -np.inf).all()
        d = ((lse - want_lse).abs() - (2 * score + 2.0 ** -21 * (1 + want_lse.abs())))[rows][~empty[rows]]
        assert d.numel() == 0 or d.max() <= 0, d.max()


def _run(b, H, prefix=None, workspace="all", seed=1, q_gap=0, o_gap=0, amplitude=1.0, scale=0.0, q_start=True, with_lse=True, **kw):
    g = torch.Generator().manual_seed(seed)
    Q = (amplitude * torch.randn(b.T, H * b.D, generator=g)).to(torch.bfloat16)
    cache, seqs = b.on_gpu(B, q_start=q_start, **kw)
    dQ, O = torch.full((b.T, H * b.D + q_gap), 9.0, device="cuda", dtype=torch.bfloat16), torch.full((b.T, H * b.D + o_gap), 7.0, device="cuda", dtype=torch.bfloat16)
    dQ[:, : H * b.D] = Q.cuda()
    lse = torch.full((b.T, H), 7.0, device="cuda") if with_lse else None
    prefix = b.prefix if prefix is None else prefix
    need = B.patch_attention_workspace_bytes(H, seqs, cache, prefix_len=prefix)
    size = dict(all=need, none=0, half=need // 2).get(workspace, workspace)
    guard = 4096
    ws = torch.full(((size if isinstance(size, int) else 0) // 4 + guard,), float("nan"), device="cuda")
    B.patch_attention(dQ, H, seqs, cache, O, _stream(), scale=scale, prefix_len=prefix, lse=lse, workspace=ws if size else None, workspace_bytes=size or 0,
                      q_stride=H * b.D + q_gap, o_stride=H * b.D + o_gap)
    torch.cuda.synchronize()
    assert ws[size // 4:].isnan().all() and (O[:, H * b.D:] == 7).all()
    return Q, O[:, : H * b.D], lse


ATTENDS = [
    # n, kv, H, KH, D, page, prefix, e4m3
    ([1], [1], 1, 1, 64, 16, 0, False), ([1], [500], 14, 2, 64, 16, 0, False), ([1, 1, 1, 1], [31, 32, 33, 0], 32, 8, 128, 64, 0, False),
    ([1, 1, 1], [1000, 3, 257], 8, 8, 128, 32, 0, False), ([1, 1], [700, 2100], 4, 2, 256, 128, 0, False), ([1, 1, 1], [513, 127, 2049], 32, 8, 128, 16, 0, True),
    ([1] * 9, [600, 601, 640, 700, 513, 514, 900, 1, 0], 8, 2, 128, 64, 512, False), ([1] * 5, [400, 401, 402, 403, 404], 12, 4, 64, 16, 391, False),
    ([5] * 3, [300, 310, 205], 10, 10, 128, 16, 153, False), ([4, 0, 7, 1], [40, 17, 300, 60], 16, 1, 128, 32, 0, True), ([3, 2], [300, 299], 14, 2, 64, 256, 290, True),
    ([8, 3], [3, 3], 4, 2, 128, 16, 0, False), ([33, 1, 20], [33, 90, 100], 8, 2, 64, 16, 0, False), ([130], [130], 2, 1, 128, 64, 0, False),
    ([90, 150, 7], [200, 150, 500], 4, 1, 256, 64, 0, False), ([64, 100], [164, 200], 7, 1, 128, 16, 100, True), ([300], [300], 2, 2, 64, 128, 0, True),
    ([270, 40], [600, 333], 3, 3, 128, 32, 290, False), ([1] * 40, list(range(130, 170)), 4, 1, 256, 16, 128, True), ([150, 1], [222, 222], 16, 2, 128, 64, 64, False),
    ([1] * 150, [64 + i % 70 for i in range(150)], 2, 2, 64, 16, 64, False), ([257], [1300], 2, 2, 256, 256, 0, True)]


@pytest.mark.parametrize("n,kv,H,KH,D,page,prefix,e4m3", ATTENDS)
def test_attention(n, kv, H, KH, D, page, prefix, e4m3):
    b = R.Batch(n, kv, KH, D, page, prefix=prefix, e4m3=e4m3, seed=sum(kv))
    for workspace in ("all", "none", "half"):
        print(f"attention n={n[:4]} kv={kv[:4]} H={H} KH={KH} D={D} page={page} prefix={prefix} e4m3={e4m3} workspace={workspace}", flush=True)
        Q, O, lse = _run(b, H, workspace=workspace)
        _check(b, Q, H, O, lse)


@pytest.mark.parametrize("kw", [dict(q_gap=8, o_gap=24), dict(scale=0.3), dict(scale=-0.2), dict(amplitude=12.0), dict(with_lse=False), dict(max_q=1000, max_kv=100000), dict(amplitude=0.0)])
def test_attention_arguments(kw):
    b = R.Batch([3, 1, 100], [303, 700, 150], 2, 128, 32, prefix=40, seed=7, page_gap=48)
    Q, O, lse = _run(b, 4, **kw)
    _check(b, Q, 4, O, lse, scale=kw.get("scale"))


def test_attention_without_q_start_and_without_a_shared_front_taken():
    b = R.Batch([1] * 6, [100, 0, 300, 64, 65, 1], 2, 64, 16, seed=2)
    for q_start in (True, False):
        Q, O, lse = _run(b, 6, q_start=q_start)
        _check(b, Q, 6, O, lse)
    b = R.Batch([2] * 4, [100, 90, 300, 64], 2, 64, 16, prefix=50, seed=2)
    for prefix in (0, 16, 49, 50):
        Q, O, lse = _run(b, 6, prefix=prefix)
        _check(b, Q, 6, O, lse)


def test_results_do_not_change_from_call_to_call():
    b = R.Batch([1] * 7 + [60], [900, 800, 700, 1200, 300, 2000, 1, 500], 2, 128, 16, prefix=0, seed=5)
    first = _run(b, 8)[1].clone()
    for _ in range(3):
        assert torch.equal(_run(b, 8)[1], first)


@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_that_are_not_there_make_their_readers_nan(e4m3):
    b = R.Batch([1, 1, 2, 1, 1], [100, 100, 100, 100, 900], 2, 64, 16, e4m3=e4m3, seed=6)
    good = b.table.copy()
    b.table[0, 3], b.table[1, 3], b.table[2, 6] = -1, b.n_pages, 1 << 30       # the last: only keys 96 .. 99
    b.table[3, 7] = -5                                                          # beyond its keys: nobody's
    Q, O, lse = _run(b, 4, max_kv=200)                                          # the last sequence is longer than that
    b.table = good
    _check(b, Q, 4, O, None, skip=(0, 1, 2, 3, 5))
    assert O[[0, 1, 2, 3, 5]].isnan().all()


def test_infinities_and_nan_where_a_row_does_not_look():
    """Keys and values after a row's position, of any kind, are not in its result; those at or before are."""
    n, kv = [40, 1], [90, 30]
    for H, KH, D, page in ((4, 2, 64, 16), (2, 2, 128, 64)):
        b = R.Batch(n, kv, KH, D, page, seed=8)
        for value in (float("nan"), float("inf"), -float("inf")):
            j = 70                                                             # key 70 of sequence 0: rows 0 .. 19 are before it
            p = b.table[0, j // page]
            cells = KH * page * D
            old_k, old_v = b.k.clone(), b.v.clone()
            b.k[p, :cells].view(KH, page, D)[:, j % page] = value
            b.v[p, :cells].view(KH, D, page)[:, :, j % page] = value
            Q, O, lse = _run(b, H)
            b.k, b.v = old_k, old_v
            _check(b, Q, H, O, lse, skip=range(20, 40))
            assert not torch.isfinite(O[20:40].float()).all()


def test_scores_of_any_size():
    """All scores at the lowest and the highest that are finite in fp32, and equal ones."""
    b = R.Batch([1, 20], [300, 64], 1, 64, 16, seed=9)
    Q, O, lse = _run(b, 1, amplitude=0.0)
    _check(b, Q, 1, O, lse)
    for sign in (1.0, -1.0):
        b = R.Batch([1], [200], 1, 64, 16, seed=9)
        b.ks[0][:] = 0
        b.ks[0][:, :, 0] = 2.0 ** 60
        b.k[:, : 16 * 64] = torch.where(b.k[:, : 16 * 64].isnan(), b.k[:, : 16 * 64], torch.zeros(1, dtype=torch.bfloat16))
        kview = b.k[:, : 16 * 64].view(-1, 1, 16, 64)
        kview[..., 0] = torch.where(kview[..., 0].isnan(), kview[..., 0], torch.tensor(2.0 ** 60, dtype=torch.bfloat16))
        cache, seqs = b.on_gpu(B)
        q = torch.zeros(1, 64, dtype=torch.bfloat16, device="cuda")
        q[0, 0] = sign * 2.0 ** 66
        O = torch.empty_like(q)
        B.patch_attention(q, 1, seqs, cache, O, _stream(), scale=1.0)
        mean = b.vs[0][:, 0].mean(0)
        av = b.vs[0][:, 0].abs().mean(0)
        assert ((O[0].cpu().double() - mean).abs() <= R.BF16_HALF * mean.abs() + av * (R.BF16_HALF + 2.0 ** -16)).all()


def test_captured_with_append_and_on_another_stream():
    """A decoding step (append, then attention) as a graph, replayed with the program's own work between; the same on a stream of its own."""
    n, kv, H, KH, D, page = [1] * 6, [600, 300, 257, 900, 1, 64], 8, 2, 128, 16
    b = R.Batch(n, kv, KH, D, page, prefix=0, seed=11)
    g = torch.Generator().manual_seed(12)
    row = (H + 2 * KH) * D
    x = torch.randn(b.T, row, generator=g).cuda()
    table = R.table_of(b.max_kv, D).cuda()
    cache, seqs = b.on_gpu(B)
    rope = B.Rope(table, b.max_kv, D)
    part = lambda first, heads, **kw: B.Heads(x.data_ptr() + first * D * 4, heads, row, f32=True, **kw)  # noqa: E731
    Q, O = torch.empty(b.T, H * D, device="cuda", dtype=torch.bfloat16), torch.empty(b.T, H * D, device="cuda", dtype=torch.bfloat16)
    ws = torch.empty(B.patch_attention_workspace_bytes(H, seqs, cache), device="cuda", dtype=torch.uint8)
    k, v, q = part(H, KH), part(H + KH, KH), part(0, H, out=Q, out_stride=H * D)

    def step():
        s = _stream()
        B.patch_kv_append(k, v, seqs, cache, s, rope=rope, q=q)
        B.patch_attention(Q, H, seqs, cache, O, s, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.normal_(generator=None)
        step()
        want = O.clone()
        O.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want) and not O.isnan().any()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    O.fill_(5.0)
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        step()
    torch.cuda.current_stream().wait_stream(other)
    assert torch.equal(O, want)


def test_pages_beyond_4_gb():
    """A cache of 5 GB: pages at its end, cells beyond 2^32 bytes and 2^31 elements."""
    KH, D, page = 8, 128, 64
    cells = KH * page * D
    n_pages = (5 << 30) // (2 * cells)
    k, v = (torch.empty(n_pages, cells, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    b = R.Batch([3, 1], [200, 70], KH, D, page, seed=13)
    cache, seqs = b.on_gpu(B)
    where = [n_pages - 1 - 7 * i for i in range(b.n_pages)]
    for i, w in enumerate(where):
        k[w], v[w] = b.dk[i], b.dv[i]
    moved = torch.tensor([[where[p] if p >= 0 else -1 for p in r] for r in b.table.tolist()], dtype=torch.int32, device="cuda")
    seqs = B.Seqs(2, b.T, b.d[0], moved, b.table.shape[1], b.max_q, b.max_kv, q_start=b.d[2])
    cache = B.KVCache(k, v, n_pages, page, KH, D)
    g = torch.Generator().manual_seed(1)
    Q = torch.randn(b.T, 8 * D, generator=g).to(torch.bfloat16)
    O, x = torch.empty(b.T, 8 * D, device="cuda", dtype=torch.bfloat16), torch.randn(b.T, KH * D, device="cuda").to(torch.bfloat16)
    B.patch_attention(Q.cuda(), 8, seqs, cache, O, _stream())
    _check(b, Q, 8, O, None)
    B.patch_kv_append(B.Heads(x, KH, KH * D), B.Heads(x, KH, KH * D), seqs, cache, _stream())
    torch.cuda.synchronize()
    last = k[where[b.table[0, 3]]].view(KH, page, D)
    assert torch.equal(last[:, 199 % page], x[2].view(KH, D)) and torch.equal(v[where[b.table[1, 1]]].view(KH, D, page)[:, :, 69 % page], x[3].view(KH, D))


def test_scales_of_any_kind():
    """Heads whose keys' scale is zero or negative, and one whose values' is."""
    for n, kv in (([1, 1], [300, 77]), ([90], [120])):
        b = R.Batch(n, kv, 4, 128, 16, e4m3=True, seed=21)
        raw_k, raw_v = [x / b.k_scale.double()[:, None] for x in b.ks], [x / b.v_scale.double()[:, None] for x in b.vs]
        b.k_scale[1], b.k_scale[2], b.v_scale[3] = 0.0, -b.k_scale[2], -b.v_scale[3]
        b.ks, b.vs = [x * b.k_scale.double()[:, None] for x in raw_k], [x * b.v_scale.double()[:, None] for x in raw_v]
        Q, O, lse = _run(b, 8)
        _check(b, Q, 8, O, lse)


def test_more_sequences_than_a_wavefront_has_lanes():
    """Empty ones, ones without new tokens, short and long, in the order of nothing; with a shared front and without."""
    kv = [(37 * i) % 400 if i % 5 else 0 for i in range(200)]
    n = [0 if i % 7 == 3 else 1 + (i % 3 == 1) for i in range(200)]
    for prefix in (0, 70):
        lens = [L if L == 0 else L + prefix for L in kv]
        b = R.Batch(n, lens, 2, 64, 32, prefix=prefix, seed=22)
        for workspace in ("all", "half", "none"):
            # rows of sequences of nothing see nothing of the shared front, either
            Q, O, lse = _run(b, 6, workspace=workspace)
            _check(b, Q, 6, O, lse)
