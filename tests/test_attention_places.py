"""Where the tokens of a batch are, as the kernels work it out from what only the device knows (no GPU)."""
import ctypes

import pytest

from paper_2509_23410_amd import binding as B

TURN = 64


@pytest.mark.parametrize("n_tokens,max_kv", [(300, 1 << 20), (1 << 23, 1 << 30), (256, 100)])
def test_tiles_of_v_read_rows_of_their_sequence_alone(n_tokens, max_kv):
    out = (ctypes.c_int * (3 + TURN))()
    ends = [0, 1, 7, 100, 256, n_tokens - 1, n_tokens, n_tokens + 5, -3]
    for t0 in ends:
        for t1 in ends:
            for length in (-5, 0, 1, 63, 64, 65, 99, 100, 128, 1000, max_kv, max_kv + 1):
                first, last = min(max(t0, 0), n_tokens), min(max(t1, 0), n_tokens)
                n = max(last - first, 0)
                begin = max(length - n, 0)
                seen = set()
                for tile in sorted({0, 1, 2, 3, max(-(-(length - (begin & ~63)) // TURN) - 1, 0)}):
                    B.lib().patch_test_new_tile(t0, t1, length, n_tokens, max_kv, tile, out)
                    base, there = (begin & ~63) + tile * TURN, 0 <= length <= max_kv and n > 0 and length > (begin & ~63) + tile * TURN
                    assert out[0] == there, (t0, t1, length, tile)
                    if there:
                        assert (out[1], out[2]) == (begin, base)
                        for i in range(TURN):
                            assert first <= out[3 + i] < first + n, (t0, t1, length, tile, i)
                            if begin <= base + i < length:
                                assert out[3 + i] == first + base + i - (length - n)
                                seen.add(base + i)
                if length <= 3 * TURN:
                    assert seen == (set(range(begin, length)) if n and 0 < length <= max_kv else set())


def test_rows_that_no_sequence_has():
    place = B.lib().patch_test_place
    for n_tokens in (10, 1 << 23):
        for t0, t1 in [(0, 3), (3, 5), (3, 3), (10, 10), (4, 10), (0, 10)]:
            for t in range(10):
                assert place(t0, t1, n_tokens, t) == (t - t0 if t0 <= t < t1 else -1), (t0, t1, t)
