"""Prompts of some sequences and nothing of others, enough tokens for tiles of V."""
import pytest

from padded_batch import Padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kv,KH,D,page", [([0, 300, 0, 5, 0], [100, 411, 77, 70, 33], 2, 64, 16), ([260, 0], [260, 1], 3, 128, 64), ([0, 0, 290], [63, 65, 333], 1, 256, 32),
                                            ([30, 0] * 12, [100 + 7 * i for i in range(24)], 2, 64, 128), ([400, 3, 8], [300, 0, 5], 2, 64, 16)])
def test_append_beside_sequences_without_new_tokens(n, kv, KH, D, page):
    Padded(n, kv, KH, D, page, seed=61).check_append(H=2, rot=32)
