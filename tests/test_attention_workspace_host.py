"""A workspace of the size that patch_attention_workspace_bytes names gives the split that any larger one gives (no GPU)."""
import random

import pytest

from test_attention_host import plan

SHAPES = [(14, 2, 64), (32, 32, 128), (32, 8, 128), (40, 40, 128), (8, 4, 256), (1, 1, 64), (3, 1, 256), (128, 1, 128)]


def _cases():
    yield from [(32, 8, 128, 64, 64, 1, 9000, 8192), (8, 4, 256, 2, 90, 60, 3000, 1000), (1, 1, 64, 2, 67, 40, 700, 300), (1, 1, 64, 1, 1, 1, 500, 0), (2, 2, 128, 1, 300, 300, 300, 0)]
    rng = random.Random(5)
    for _ in range(400):
        H, KH, D = rng.choice(SHAPES)
        n_seqs, max_q = int(2 ** rng.uniform(0, 8)), int(2 ** rng.uniform(0, 10))
        n_tokens = max(1, rng.randrange(n_seqs * max_q + 1))
        max_kv = int(2 ** rng.uniform(0, 17))
        yield H, KH, D, n_seqs, n_tokens, max_q, max_kv, rng.choice([0, rng.randrange(max_kv + 1), max_kv])


@pytest.mark.parametrize("case", list(_cases()), ids=str)
def test_the_size_asked_for_is_enough(case):
    split = lambda p: p if p[4] > 1 else p[:1] + p[2:]  # noqa: E731  (in one part, how long it could be tells nothing)
    most = plan(*case, 1 << 62)
    used = most[5]
    for ws in (used, used + 1, used + 4096):
        assert split(plan(*case, ws)) == split(most)
    if used:
        assert plan(*case, used - 1)[5] < used      # and no more than enough
