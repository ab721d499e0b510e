"""Refusals of the attention side of a layer, what its kernels make of numbers that only the device knows, and how a call splits its keys (no GPU)."""
import ctypes
import random

import pytest

from paper_2509_23410_amd import binding as B

P = 1 << 20     # an address that is aligned and never followed


def heads(**kw):
    a = dict(x=P, heads=8, stride=8 * 128, f32=False, gamma=None, out=P, out_stride=8 * 128)
    a.update(kw)
    return B.Heads(**a)


def rope(**kw):
    a = dict(table=P, n_pos=100, rot_dim=128)
    a.update(kw)
    return B.Rope(**a)


def cache(**kw):
    a = dict(k=P, v=P, n_pages=10, page_size=16, kv_heads=8, head_dim=128)
    a.update(kw)
    return B.KVCache(**a)


def seqs(**kw):
    a = dict(n_seqs=4, n_tokens=0, kv_len=P, page_table=P, table_stride=8, max_q=1, max_kv=128, q_start=P)
    a.update(kw)
    return B.Seqs(**a)


def status(call, *a, **kw):
    try:
        call(*a, **kw)
        return B.OK
    except B.PatchError as e:
        return e.status


BAD_HEADS = [(dict(x=None), B.ERR_ARG), (dict(x=P + 8), B.ERR_ARG), (dict(heads=0), B.ERR_ARG), (dict(gamma=P + 4), B.ERR_ARG), (dict(stride=8 * 128 - 8), B.ERR_SHAPE),
             (dict(stride=8 * 128 + 4), B.ERR_SHAPE), (dict(stride=-8 * 128), B.ERR_SHAPE)]
BAD_OUT = [(dict(out=None), B.ERR_ARG), (dict(out=P + 2), B.ERR_ARG), (dict(out_stride=8 * 128 - 8), B.ERR_SHAPE), (dict(out_stride=8 * 128 + 4), B.ERR_SHAPE)]
BAD_ROPE = [(dict(table=None), B.ERR_ARG), (dict(table=P + 4), B.ERR_ARG), (dict(n_pos=0), B.ERR_ARG), (dict(eps=-1.0), B.ERR_ARG), (dict(eps=float("nan")), B.ERR_ARG),
            (dict(rot_dim=0), B.ERR_SHAPE), (dict(rot_dim=12), B.ERR_SHAPE), (dict(rot_dim=136), B.ERR_SHAPE)]
BAD_CACHE = [(dict(k=None), B.ERR_ARG), (dict(v=None), B.ERR_ARG), (dict(k=P + 8), B.ERR_ARG), (dict(n_pages=0), B.ERR_ARG), (dict(n_pages=1 << 31), B.ERR_ARG),
             (dict(kv_heads=0), B.ERR_ARG), (dict(k_scale=P), B.ERR_ARG), (dict(e4m3=True, v_scale=P + 2), B.ERR_ARG), (dict(head_dim=96), B.ERR_SHAPE),
             (dict(page_size=8), B.ERR_SHAPE), (dict(page_size=48), B.ERR_SHAPE), (dict(page_size=512), B.ERR_SHAPE), (dict(page_size=0), B.ERR_SHAPE),
             (dict(page_stride=8 * 16 * 128 - 16), B.ERR_SHAPE), (dict(page_stride=8 * 16 * 128 + 8), B.ERR_SHAPE)]
BAD_SEQS = [(dict(kv_len=None), B.ERR_ARG), (dict(page_table=None), B.ERR_ARG), (dict(kv_len=P + 2), B.ERR_ARG), (dict(n_seqs=0), B.ERR_ARG), (dict(n_seqs=65536), B.ERR_ARG),
            (dict(n_tokens=-1), B.ERR_ARG), (dict(n_tokens=(1 << 23) + 1), B.ERR_ARG), (dict(max_q=-1), B.ERR_ARG), (dict(max_kv=-1), B.ERR_ARG),
            (dict(table_stride=0), B.ERR_ARG), (dict(q_start=None), B.ERR_SHAPE)]


@pytest.mark.parametrize("which,kw,want", [("q", *x) for x in BAD_HEADS + BAD_OUT] + [("k", *x) for x in BAD_HEADS + BAD_OUT] + [("rope", *x) for x in BAD_ROPE])
def test_qk_rope_refuses(which, kw, want):
    q, k, r = heads(**(kw if which == "q" else {})), heads(**(kw if which == "k" else {})), rope(**(kw if which == "rope" else {}))
    assert status(B.patch_qk_rope, q, k, P, 0, 128, r) == want


def test_qk_rope_refuses_more():
    assert status(B.patch_qk_rope, heads(), None, P, 0, 128, None) == B.OK
    assert status(B.patch_qk_rope, heads(), heads(), None, 0, 128, rope()) == B.ERR_ARG
    assert status(B.patch_qk_rope, heads(), heads(), P + 2, 0, 128, rope()) == B.ERR_ARG
    assert status(B.patch_qk_rope, heads(), heads(), P, -1, 128, rope()) == B.ERR_ARG
    assert status(B.patch_qk_rope, heads(), heads(), P, (1 << 23) + 1, 128, rope()) == B.ERR_ARG
    assert status(B.patch_qk_rope, heads(), heads(), P, 0, 96, rope()) == B.ERR_SHAPE
    assert status(B.patch_qk_rope, heads(), heads(f32=True), P, 0, 128, rope()) == B.ERR_ARG      # one type for both
    assert B.lib().patch_qk_rope(None, None, P, 0, 128, None, None) == B.ERR_ARG


@pytest.mark.parametrize("which,kw,want", [(w, *x) for w in ("q", "k", "v") for x in BAD_HEADS] + [("q", *x) for x in BAD_OUT] + [("rope", *x) for x in BAD_ROPE] +
                         [("cache", *x) for x in BAD_CACHE] + [("seqs", *x) for x in BAD_SEQS] + [("v", dict(gamma=P), B.ERR_ARG), ("v", dict(f32=True), B.ERR_ARG),
                          ("k", dict(heads=4), B.ERR_SHAPE), ("v", dict(heads=16, stride=16 * 128), B.ERR_SHAPE)])
def test_kv_append_refuses(which, kw, want):
    pick = lambda name: kw if which == name else {}  # noqa: E731
    k, v, q = heads(**pick("k")), heads(**pick("v")), heads(**pick("q"))
    got = status(B.patch_kv_append, k, v, seqs(**pick("seqs")), cache(**pick("cache")), rope=rope(**pick("rope")), q=q)
    assert got == (B.ERR_SHAPE if (which, kw) in (("k", dict(heads=0)), ("v", dict(heads=0))) else want)      # not the cache's heads, either


def test_kv_append_takes_no_tokens():
    assert status(B.patch_kv_append, heads(out=None), heads(out=None), seqs(), cache()) == B.OK


@pytest.mark.parametrize("which,kw,want", [("cache", *x) for x in BAD_CACHE] + [("seqs", *x) for x in BAD_SEQS] + [
    ("call", dict(Q=None), B.ERR_ARG), ("call", dict(O=None), B.ERR_ARG), ("call", dict(Q=P + 8), B.ERR_ARG), ("call", dict(heads=0), B.ERR_ARG),
    ("call", dict(heads=12), B.ERR_SHAPE), ("call", dict(q_stride=31 * 128), B.ERR_SHAPE), ("call", dict(o_stride=32 * 128 + 4), B.ERR_SHAPE),
    ("call", dict(prefix_len=-1), B.ERR_ARG), ("call", dict(scale=float("nan")), B.ERR_ARG), ("call", dict(scale=float("inf")), B.ERR_ARG),
    ("call", dict(lse=P + 2), B.ERR_ARG), ("call", dict(workspace=P + 4, workspace_bytes=100), B.ERR_ARG), ("seqs", dict(n_tokens=1 << 21), B.ERR_SHAPE)])
def test_attention_refuses(which, kw, want):
    pick = lambda name: kw if which == name else {}  # noqa: E731
    a = dict(Q=P, heads=32, O=P)
    a.update(pick("call"))
    c, s = cache(**pick("cache")), seqs(**pick("seqs"))
    Q, H, O = a.pop("Q"), a.pop("heads"), a.pop("O")
    assert status(B.patch_attention, Q, H, s, c, O, **a) == want
    if which in ("cache", "seqs"):
        assert B.patch_attention_workspace_bytes(H, s, c) == 0


def test_attention_takes_no_tokens():
    assert status(B.patch_attention, P, 32, seqs(), cache(), P) == B.OK
    assert B.patch_attention_workspace_bytes(32, seqs(), cache()) == 0


def test_what_a_sequence_is_whatever_the_device_says():
    """The tokens of a sequence lie inside the batch and its keys inside the table, for any integers."""
    far = [-(1 << 31), -5, -1, 0, 1, 3, 10, 11, 4096, (1 << 31) - 1]
    out = (ctypes.c_int * 5)()
    for n_tokens in (0, 1, 10, 1 << 23):
        for max_kv in (0, 1, 128, 1 << 30):
            for t0 in far:
                for t1 in far:
                    for L in far:
                        B.lib().patch_test_seq(t0, t1, L, n_tokens, max_kv, out)
                        first, n, length, pos0, bad = out
                        assert 0 <= first <= n_tokens and 0 <= n <= n_tokens - first and 0 <= length <= max_kv and pos0 == length - n and bad == (L > max_kv)
                        if 0 <= t0 <= t1 <= n_tokens and 0 <= L <= max_kv:
                            assert (first, n, length) == (t0, t1 - t0, L)


def test_page_numbers_out_of_range_are_none():
    for n_pages in (1, 7, (1 << 31) - 1):
        for i in [-(1 << 31), -1, 0, 1, 6, 7, 8, (1 << 31) - 1]:
            assert B.lib().patch_test_page(i, n_pages) == (i if 0 <= i < n_pages else -1)


def plan(H, KH, D, n_seqs, n_tokens, max_q, max_kv, prefix, ws, page=64):
    s = B.Seqs(n_seqs, n_tokens, P, P, -(-max(max_kv, 1) // page), max_q, max_kv, q_start=P)
    c = B.KVCache(P, P, 1 << 20, page, KH, D)
    o, out = B.AttentionOpts(0.0, prefix, None, None, 0), (ctypes.c_int64 * 10)()
    assert B.lib().patch_test_attention_plan(H, s.ref, c.ref, ctypes.byref(o), ctypes.c_size_t(ws), out) == 0
    return tuple(out)


def stretches(lens, KH, prefix, waves, least_steps, step):
    """What the wavefronts of a launch for few rows take, as the kernel finds it: {(sequence, head): [(wavefront, part, first step, last step, steps)]}."""
    base = prefix & ~63
    n = [-(-(L - base) // step) if L > prefix else 0 for L in lens]
    line = [(s, h, i) for s in range(len(lens)) for h in range(KH) for i in range(n[s])]
    stretch = max(-(-len(line) // waves), least_steps)
    start, at = {}, 0
    for s in range(len(lens)):
        for h in range(KH):
            start[s, h], at = at, at + n[s]
    took = {}
    for i, (s, h, b) in enumerate(line):
        me = i // stretch
        part = me - start[s, h] // stretch
        took.setdefault((s, h), {}).setdefault((me, part), []).append(b)
    assert not line or (len(line) - 1) // stretch < waves
    return {u: sorted((me, part, min(b), max(b), len(b)) for (me, part), b in t.items()) for u, t in took.items()}, n


@pytest.mark.parametrize("H,KH,D", [(14, 2, 64), (32, 32, 128), (32, 8, 128), (8, 4, 256), (1, 1, 64), (128, 1, 128)])
def test_every_key_is_in_one_part_that_the_workspace_holds(H, KH, D):
    for n_seqs, max_q, max_kv, prefix in [(1, 1, 1, 0), (1, 1, 65000, 0), (64, 1, 9000, 8192), (64, 1, 8192, 8192), (7, 5, 2600, 1531), (3, 700, 2500, 33), (2, 1, 1 << 30, 0),
                                          (2, 1, 1 << 30, 1 << 29), (1, 4096, 4096, 17), (5, 3, 0, 0), (5, 3, 40, 90), (300, 1, 300, 0), (3, 1 << 18 if H < 32 else 1 << 16, 1 << 24, 1 << 20)]:
        T = n_seqs * max_q
        for ws in (0, 15, T * H * (D + 2) * 4, 2 * T * H * (D + 2) * 4 + 16, 9 * T * H * (D + 2) * 4, 1 << 28, 1 << 62):
            P_, own, front, front_parts, parts, used, few, front_blocks, waves, least_steps = plan(H, KH, D, n_seqs, T, max_q, max_kv, prefix, ws)
            assert used <= ws and P_ in (0, min(prefix, max_kv)) and own > 0 and own % 128 == 0
            rest, step = max_kv - (P_ & ~63), 32 if D == 256 else 64
            if parts == 1:
                assert P_ == 0 and own >= rest and waves == 0
            if P_:
                assert front % 128 == 0 and front_parts == -(-P_ // front) >= 1
            else:
                assert front_parts == front_blocks == 0
            if not few:
                assert waves == 0 and parts - front_parts == max(1, -(-rest // own))
                assert (parts - front_parts) * -(-max_q * H // KH // 16) <= 1 << 23
            elif waves:
                # a head of the longest sequence is in no more stretches than it has parts, wherever it begins, and the line's steps are counted in 32 bits
                assert waves % 4 == 0 and least_steps * (parts - front_parts - 1) >= -(-rest // step) and n_seqs * KH * (-(-rest // step) + 1) < 1 << 30


@pytest.mark.parametrize("H,KH,D,max_q,prefix", [(14, 2, 64, 1, 0), (32, 32, 128, 1, 0), (32, 8, 128, 2, 1000), (8, 4, 256, 3, 500), (1, 1, 64, 1, 77)])
@pytest.mark.parametrize("ws", [1 << 18, 1 << 21, 1 << 28])
def test_stretches_of_ragged_batches(H, KH, D, max_q, prefix, ws):
    rng = random.Random(H + prefix)
    for n_seqs in (1, 2, 13, 70):
        lens = [rng.choice([0, prefix, prefix + 1, prefix + 128, prefix + 129, rng.randrange(4000), rng.randrange(prefix, prefix + 9000)]) for _ in range(n_seqs)]
        for scale in (1.0, 1.7):                         # the caller's bound may be loose
            max_kv = int(max(max(lens), 1) * scale)
            P_, own, front, front_parts, parts, used, few, front_blocks, waves, least_steps = plan(H, KH, D, n_seqs, n_seqs * max_q, max_q, max_kv, prefix, ws)
            if not waves:
                continue
            took, n = stretches(lens, KH, P_, waves, least_steps, 32 if D == 256 else 64)
            for u, t in took.items():
                assert [part for _, part, *_ in t] == list(range(len(t))) and len(t) <= parts - front_parts
                assert t[0][2] == 0 and t[-1][3] == n[u[0]] - 1 and all(x[3] + 1 == y[2] for x, y in zip(t, t[1:])) and all(x[3] - x[2] + 1 == x[4] for x in t)
