"""A shared front that is longer than any sequence, which patch_attention takes: all their tokens are then the same ones."""
import pytest

from padded_batch import Padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kv,H,KH,D,page", [
    ([1, 1], [10, 90], 6, 2, 64, 16), ([1, 1, 1], [0, 80, 50], 8, 8, 128, 32), ([3, 2, 5], [5, 33, 70], 4, 1, 128, 16), ([1] * 70, [1 + i % 64 for i in range(70)], 2, 2, 64, 16),
    ([40, 60], [40, 95], 4, 2, 64, 16), ([20, 50, 33], [0, 50, 99], 2, 1, 256, 64)])
def test_front_longer_than_every_sequence(n, kv, H, KH, D, page):
    # bounds that are not close: the host cannot tell that nobody has 100 tokens
    p = Padded(n, kv, KH, D, page, wide=20, max_kv=200, prefix=100, seed=41)
    for workspace in ("all", "half", "none"):
        p.check_attention(H, prefix=100, workspace=workspace)


@pytest.mark.parametrize("n,kv,H,KH,D,page", [([0, 1, 1], [150, 120, 130], 6, 2, 64, 16), ([0, 40, 50], [150, 150, 160], 4, 2, 128, 32)])
def test_front_not_from_a_sequence_without_tokens(n, kv, H, KH, D, page):
    """An idle slot keeps its length, and its pages are others' by now: nobody of the call has tokens there."""
    p = Padded(n, kv, KH, D, page, prefix=100, seed=42, spare=3)
    spare = [i for i in range(p.b.n_pages) if i not in p.b.table]
    p.b.table[0] = spare[0]                                          # (NaN cells)
    for workspace in ("all", "none"):
        p.check_attention(H, workspace=workspace)
