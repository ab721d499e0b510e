"""Refusals of the 4-bit cache, the weights of its tokens and the eviction, and how an attention call over 4-bit cells splits its keys (no GPU)."""
import ctypes

import pytest

from paper_2509_23410_amd import binding as B

P = 1 << 20     # an address that is aligned and never followed


def heads(**kw):
    return B.Heads(**dict(dict(x=P, heads=8, stride=8 * 128, f32=False, gamma=None, out=P + 4096, out_stride=8 * 128), **kw))


def cache4(**kw):
    return B.KVCache4(**dict(dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=10, page_size=16, kv_heads=8, head_dim=128), **kw))


def cache(**kw):
    return B.KVCache(**dict(dict(k=P, v=P, n_pages=10, page_size=16, kv_heads=8, head_dim=128), **kw))


def seqs(**kw):
    return B.Seqs(**dict(dict(n_seqs=4, n_tokens=0, kv_len=P, page_table=P, table_stride=8, max_q=1, max_kv=128, q_start=P), **kw))


def status(call, *a, **kw):
    try:
        call(*a, **kw)
        return B.OK
    except B.PatchError as e:
        return e.status


BAD_CACHE4 = [(dict(k=None), B.ERR_ARG), (dict(v=None), B.ERR_ARG), (dict(k_scale=None), B.ERR_ARG), (dict(v_scale=None), B.ERR_ARG), (dict(k=P + 8), B.ERR_ARG),
              (dict(v=P + 4), B.ERR_ARG), (dict(k_scale=P + 8), B.ERR_ARG), (dict(v_scale=P + 1), B.ERR_ARG), (dict(n_pages=0), B.ERR_ARG), (dict(n_pages=1 << 31), B.ERR_ARG),
              (dict(kv_heads=0), B.ERR_ARG), (dict(kv_heads=65536), B.ERR_ARG), (dict(head_dim=96), B.ERR_SHAPE), (dict(head_dim=32), B.ERR_SHAPE), (dict(page_size=8), B.ERR_SHAPE),
              (dict(page_size=48), B.ERR_SHAPE), (dict(page_size=512), B.ERR_SHAPE), (dict(page_stride=8 * 16 * 128 - 512), B.ERR_SHAPE), (dict(page_stride=8 * 16 * 128 + 256), B.ERR_SHAPE),
              (dict(page_stride=1 << 33), B.ERR_SHAPE), (dict(page_stride=-512), B.ERR_SHAPE)]
BAD_SEQS = [(dict(kv_len=None), B.ERR_ARG), (dict(page_table=None), B.ERR_ARG), (dict(kv_len=P + 2), B.ERR_ARG), (dict(n_seqs=0), B.ERR_ARG), (dict(n_seqs=65536), B.ERR_ARG),
            (dict(max_kv=-1), B.ERR_ARG), (dict(table_stride=0), B.ERR_ARG)]
BAD_ROWS = [(dict(n_tokens=-1), B.ERR_ARG), (dict(n_tokens=(1 << 23) + 1), B.ERR_ARG), (dict(max_q=-1), B.ERR_ARG), (dict(q_start=None), B.ERR_SHAPE), (dict(q_start=P + 2), B.ERR_ARG)]


@pytest.mark.parametrize("which,kw,want", [("cache", *x) for x in BAD_CACHE4] + [("seqs", *x) for x in BAD_SEQS + BAD_ROWS] + [
    ("k", dict(x=None), B.ERR_ARG), ("k", dict(heads=4), B.ERR_SHAPE), ("v", dict(gamma=P), B.ERR_ARG), ("v", dict(f32=True, stride=2048), B.ERR_ARG), ("k", dict(out=P + 2), B.ERR_ARG),
    ("v", dict(out_stride=8 * 128 + 4), B.ERR_SHAPE), ("k", dict(out_stride=8 * 128 - 8), B.ERR_SHAPE), ("q", dict(out=None), B.ERR_ARG), ("q", dict(x=P + 4), B.ERR_ARG),
    ("rope", dict(rot_dim=12), B.ERR_SHAPE), ("rope", dict(n_pos=0), B.ERR_ARG), ("positions", P + 2, B.ERR_ARG)])
def test_append_refuses(which, kw, want):
    pick = lambda name: kw if which == name else {}  # noqa: E731
    rope = B.Rope(**dict(dict(table=P, n_pos=100, rot_dim=128), **pick("rope")))
    got = status(B.patch_kv_append4, heads(**pick("k")), heads(**pick("v")), seqs(**pick("seqs")), cache4(**pick("cache")), rope=rope, q=heads(**pick("q")),
                 positions=kw if which == "positions" else None)
    assert got == want


def test_append_refuses_rows_that_would_move_in_place():
    f = dict(n_tokens=4, n_seqs=4)
    assert status(B.patch_kv_append4, heads(x=P, out=P, f32=True), heads(f32=True), seqs(**f), cache4()) == B.ERR_ARG
    assert status(B.patch_kv_append4, heads(), heads(x=P, out=P, out_stride=8 * 128 + 8), seqs(**f), cache4()) == B.ERR_ARG
    assert B.lib().patch_kv_append4(None, None, None, None, None, None, None, None) == B.ERR_ARG
    assert status(B.patch_kv_append4, heads(out=None), heads(out=None), seqs(), cache4()) == B.OK


@pytest.mark.parametrize("which,kw,want", [("cache", *x) for x in BAD_CACHE4] + [("seqs", *x) for x in BAD_SEQS + BAD_ROWS] + [
    ("call", dict(Q=None), B.ERR_ARG), ("call", dict(O=None), B.ERR_ARG), ("call", dict(heads=12), B.ERR_SHAPE), ("call", dict(q_stride=31 * 128), B.ERR_SHAPE),
    ("call", dict(prefix_len=-1), B.ERR_ARG), ("call", dict(scale=float("nan")), B.ERR_ARG), ("call", dict(lse=P + 2), B.ERR_ARG), ("seqs", dict(n_tokens=1 << 21), B.ERR_SHAPE)])
def test_attention_refuses(which, kw, want):
    pick = lambda name: kw if which == name else {}  # noqa: E731
    a = dict(dict(Q=P, heads=32, O=P + 4096), **pick("call"))
    c, s = cache4(**pick("cache")), seqs(**pick("seqs"))
    Q, H, O = a.pop("Q"), a.pop("heads"), a.pop("O")
    assert status(B.patch_attention4, Q, H, s, c, O, **a) == want
    if which in ("cache", "seqs"):
        assert B.patch_attention4_workspace_bytes(H, s, c) == 0
    assert status(B.patch_attention4, P, 32, seqs(), cache4(), P + 4096) == B.OK


CALLS = [("call", dict(Q=None), B.ERR_ARG), ("call", dict(Q=P + 8), B.ERR_ARG), ("call", dict(heads=0), B.ERR_ARG), ("call", dict(heads=12), B.ERR_SHAPE), ("call", dict(lse=None), B.ERR_ARG),
         ("call", dict(lse=P + 2), B.ERR_ARG), ("call", dict(W=None), B.ERR_ARG), ("call", dict(W_out=None), B.ERR_ARG), ("call", dict(W=P + 4), B.ERR_ARG),
         ("call", dict(stride=124), B.ERR_SHAPE), ("call", dict(stride=130), B.ERR_SHAPE), ("call", dict(decay=float("nan")), B.ERR_ARG), ("call", dict(scale=float("inf")), B.ERR_ARG),
         ("call", dict(slot_positions=P), B.ERR_ARG), ("call", dict(positions=P, slot_positions=P + 1), B.ERR_ARG), ("call", dict(q_stride=31 * 128), B.ERR_SHAPE),
         ("call", dict(q_stride=32 * 128 + 4), B.ERR_SHAPE), ("seqs", dict(n_tokens=1 << 21), B.ERR_SHAPE)]


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("which,kw,want", [("seqs", *x) for x in BAD_SEQS + BAD_ROWS] + CALLS)
def test_weights_refuse(which, kw, want, four):
    a = dict(dict(Q=P, heads=32, lse=P, W=P, W_out=P, stride=128), **(kw if which == "call" else {}))
    args = [a.pop(x) for x in ("Q", "heads")], [a.pop(x) for x in ("lse", "W", "W_out", "stride")]
    call, c = (B.patch_attention_weights4, cache4()) if four else (B.patch_attention_weights, cache())
    assert status(call, *args[0], seqs(**(kw if which == "seqs" else {})), c, *args[1], **a) == want
    assert status(call, P, 32, seqs(), c, P, P, P, 128) == B.OK


EVICTS = [("call", dict(W=None), B.ERR_ARG), ("call", dict(W=P + 4), B.ERR_ARG), ("call", dict(W_out=P + 4), B.ERR_ARG), ("call", dict(stride=124), B.ERR_SHAPE), ("call", dict(stride=129), B.ERR_SHAPE),
          ("call", dict(keep=0), B.ERR_ARG), ("call", dict(keep=-1), B.ERR_ARG), ("call", dict(keep=(1 << 29) + 1), B.ERR_ARG), ("call", dict(sinks=-1), B.ERR_ARG),
          ("call", dict(recent=-1), B.ERR_ARG), ("call", dict(sinks=33, recent=32), B.ERR_ARG), ("call", dict(sinks=65), B.ERR_ARG), ("call", dict(recent=1 << 62, sinks=1), B.ERR_ARG),
          ("call", dict(moved_from=None), B.ERR_ARG), ("call", dict(moved_from=P + 2), B.ERR_ARG), ("call", dict(kv_len_out=None), B.ERR_ARG), ("call", dict(kv_len_out=P + 1), B.ERR_ARG),
          ("call", dict(positions=P + 4), B.ERR_ARG), ("call", dict(positions_out=P + 4), B.ERR_ARG), ("seqs", dict(n_seqs=65535), B.ERR_SHAPE), ("seqs", dict(n_seqs=16385), B.ERR_SHAPE)]


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("which,kw,want", [("seqs", *x) for x in BAD_SEQS] + EVICTS)
def test_evict_refuses(which, kw, want, four):
    a = dict(dict(W=P, W_out=P, stride=128, keep=64, moved_from=P, kv_len_out=P), **(kw if which == "call" else {}))
    args = [a.pop(x) for x in ("W", "W_out", "stride", "keep", "moved_from", "kv_len_out")]
    wide = dict(kv_heads=128) if "n_seqs" in kw and kw["n_seqs"] in (65535, 16385) else {}
    call, c = (B.patch_kv_evict4, cache4(**wide)) if four else (B.patch_kv_evict, cache(**wide))
    assert status(call, seqs(**(kw if which == "seqs" else {})), c, *args, **a) == want


def test_no_descriptors():
    L = B.lib()
    o = B.EvictOpts(1, 0, 0, None, None, None, P, P)
    for f, c in ((L.patch_kv_evict, cache()), (L.patch_kv_evict4, cache4())):
        assert f(None, c.ref, P, 128, ctypes.byref(o), None) == f(seqs().ref, None, P, 128, ctypes.byref(o), None) == f(seqs().ref, c.ref, P, 128, None, None) == B.ERR_ARG
    w = B.WeightsOpts(0.0, 1.0, None, None)
    for f, c in ((L.patch_attention_weights, cache()), (L.patch_attention_weights4, cache4())):
        assert f(P, 4096, 32, None, c.ref, P, P, P, 128, None, ctypes.byref(w)) == f(P, 4096, 32, seqs().ref, None, P, P, P, 128, None, ctypes.byref(w)) == B.ERR_ARG
        assert f(P, 4096, 32, seqs().ref, c.ref, P, P, P, 128, None, None) == B.ERR_ARG
