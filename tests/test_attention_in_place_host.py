"""Heads normed and rotated in place: only where each goes where it came from (no GPU: what is refused is not launched)."""
from paper_2509_23410_amd import binding as B
from test_attention_host import P, cache, heads, rope, seqs, status


def test_in_place_is_refused_where_heads_would_move():
    apart = heads(x=P, out=2 * P)
    for moving in (heads(x=P, out=P, stride=9 * 128), heads(x=P, out=P, out_stride=10 * 128), heads(x=P, out=P, f32=True)):
        other = heads(x=P, out=2 * P, f32=bool(moving.c.f32))
        assert status(B.patch_qk_rope, moving, None, P, 2, 128, rope()) == B.ERR_ARG
        assert status(B.patch_qk_rope, other, moving, P, 2, 128, rope()) == B.ERR_ARG
        assert status(B.patch_kv_append, other, other, seqs(n_tokens=2), cache(), rope=rope(), q=moving) == B.ERR_ARG
    # the same place, or nothing to move
    for still, n in ((heads(x=P, out=P), 0), (heads(x=P, out=P, stride=9 * 128, out_stride=9 * 128), 0), (heads(x=P, out=P, stride=9 * 128), 0), (apart, 0)):
        assert status(B.patch_qk_rope, still, None, P, n, 128, rope()) == B.OK
