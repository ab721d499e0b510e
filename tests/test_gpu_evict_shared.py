"""Eviction from sequences that share the pages of a front all of whose tokens are sinks: those pages stay as they are, bit for bit, and what is behind them is evicted."""
import pytest
import torch

import cache4_ref as C
from test_gpu_evict import _check, _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cells", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("prefix,sinks,keep,recent", [(64, 64, 90, 8), (70, 70, 71, 1), (48, 64, 64, 0)])
def test_a_shared_front_of_sinks(prefix, sinks, keep, recent, cells):
    kv = [300, 91, 250, 130]
    b = C.batch(cells, [1] * 4, kv, 2, 64, 16, prefix=prefix, seed=prefix)
    assert all((b.table[s, : prefix // 16] == b.table[0, : prefix // 16]).all() for s in range(4))
    w, stride = _weights(b, 3, "plain")
    w[:, :, :sinks] = 0                                           # nothing but their positions keeps them
    came, _ = _check(b, cells, kv, w, stride, keep, sinks, recent)
    assert torch.equal(came[:, :, :sinks].cpu(), torch.arange(sinks, dtype=torch.int32).expand(4, 2, -1))
