"""Drafted tokens and pieces of prompts whose last key is not finite, behind a shared front and in parts: only the last row sees that."""
import numpy as np
import pytest
import torch

from padded_batch import Padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kv,H,KH,D,page,prefix", [
    ([5, 3, 4], [300, 310, 205], 4, 2, 128, 16, 150), ([4, 2, 0, 3], [900, 70, 40, 64], 16, 1, 64, 32, 0), ([3, 2], [400, 500], 4, 1, 256, 64, 390),
    ([33, 40], [420, 130], 4, 2, 64, 16, 64), ([50, 7, 20], [700, 130, 20], 2, 1, 256, 128, 0), ([3, 5], [60, 61], 4, 2, 128, 16, 100)])
def test_the_last_key_is_the_last_rows_alone(n, kv, H, KH, D, page, prefix):
    for value in (float("nan"), float("inf"), -float("inf")):
        p = Padded(n, kv, KH, D, page, lead=2, trail=1, prefix=min(prefix, min(kv)), wide=10, max_kv=max(kv) + 30, seed=81)
        b, cells = p.b, KH * page * D
        if prefix >= max(kv):                    # all of it shared: the longest sequence's last key is nobody else's
            last = [int(np.argmax(kv))]
        else:
            last = [s for s in range(len(n)) if n[s]]
        for s in last:
            at, slot = b.table[s, (kv[s] - 1) // page], (kv[s] - 1) % page
            b.k[at, :cells].view(KH, page, D)[:, slot] = value
            b.v[at, :cells].view(KH, D, page)[:, :, slot] = value
        ends = np.cumsum(n) - 1
        skip = [int(ends[s]) for s in last]
        for workspace in ("all", "none"):
            O, lse = p.check_attention(H, prefix=prefix, workspace=workspace, skip=skip)
            assert not torch.isfinite(O[skip].float()).all(1).any()
