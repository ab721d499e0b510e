"""Lengths beyond what the caller said: every row of such a sequence is NaN, whichever kernel has it, and nobody else's."""
import numpy as np
import pytest
import torch

from padded_batch import Padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kv,H,KH,D,max_kv,prefix", [
    ([1, 5, 3], [30, 60, 40], 4, 2, 64, 40, 0), ([50, 3, 45], [60, 20, 44], 4, 2, 64, 44, 0), ([50, 3, 45], [60, 20, 44], 2, 2, 256, 44, 0), ([4, 12, 2], [40, 90, 9], 2, 2, 128, 41, 16),
    ([50, 60], [50, 900], 4, 4, 128, 55, 32), ([5, 2], [7, 0], 4, 2, 64, 0, 0), ([50, 2], [50, 0], 4, 2, 128, 0, 0)])
def test_rows_of_a_length_that_cannot_be(n, kv, H, KH, D, max_kv, prefix):
    p = Padded(n, kv, KH, D, 16, max_kv=max_kv, prefix=prefix, seed=51)
    seq = np.repeat(np.arange(len(n)), n)
    bad = [t for t in range(p.b.T) if kv[seq[t]] > max_kv]
    for workspace in ("all", "none"):
        O, lse = p.check_attention(H, workspace=workspace, skip=bad)
        assert O[bad].isnan().all() and lse[bad].isnan().all()
