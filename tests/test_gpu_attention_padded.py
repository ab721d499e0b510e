"""Rows in front of the first sequence's tokens and behind the last one's: nobody's, not appended and left as they are by the attention."""
import pytest

from padded_batch import Padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kv,lead,trail,H,KH,D,page,prefix", [
    ([1, 1], [40, 33], 2, 3, 6, 2, 64, 16, 0), ([0, 2, 1], [50, 700, 300], 5, 0, 8, 8, 128, 32, 0), ([0, 0, 1, 2], [90, 80, 77, 500], 3, 1, 4, 1, 128, 16, 64),
    ([2, 1, 5], [60, 99, 45], 70, 60, 10, 10, 64, 64, 40), ([33, 0, 20], [33, 5, 100], 7, 40, 4, 2, 64, 16, 0), ([0, 50, 33], [100, 150, 99], 20, 9, 2, 1, 256, 64, 70),
    ([130], [130], 300, 1, 2, 2, 128, 64, 0), ([4, 1], [300, 299], 1, 200, 14, 2, 64, 256, 290)])
def test_attention_leaves_rows_of_nobody(n, kv, lead, trail, H, KH, D, page, prefix):
    p = Padded(n, kv, KH, D, page, lead=lead, trail=trail, prefix=prefix, seed=71)
    for workspace in ("all", "half", "none"):
        p.check_attention(H, workspace=workspace)


@pytest.mark.parametrize("n,kv,lead,trail,KH,D,page", [
    ([1, 1], [40, 33], 2, 3, 2, 64, 16), ([0, 2, 1], [50, 70, 30], 5, 0, 8, 128, 32), ([3], [3], 9, 1, 1, 256, 16),
    # enough tokens for tiles of V
    ([300, 0, 7], [411, 100, 70], 20, 30, 2, 64, 16), ([0, 40, 50], [64, 200, 300], 200, 100, 3, 128, 64)])
def test_append_leaves_rows_of_nobody(n, kv, lead, trail, KH, D, page):
    Padded(n, kv, KH, D, page, lead=lead, trail=trail, seed=72).check_append(H=2, rot=16)


def test_the_prompts_of_a_mixed_batch():
    """Decoding tokens in front, prompts behind them, each half with a call of its own on the same rows."""
    p = Padded([60, 35], [200, 35], 2, 64, 32, lead=11, seed=73)
    p.check_append(H=3, rot=64)
    p.check_attention(6)
