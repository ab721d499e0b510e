"""Few rows a sequence, and bounds far beyond the lengths: the split is made for what the host was told, the result is not."""
import pytest

from padded_batch import Padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kv,H,KH,D,prefix,e4m3", [([1] * 6, [600, 300, 257, 900, 0, 64], 8, 2, 128, 0, False), ([1] * 9, [600, 601, 640, 700, 513, 514, 900, 20, 0], 8, 2, 128, 512, False),
                                                     ([5, 3], [2000, 1000], 4, 4, 64, 391, True), ([2, 1], [300, 299], 4, 1, 256, 290, False)])
@pytest.mark.parametrize("max_q,max_kv", [(None, 100000), (16, 65536), (200, 100000)])
def test_bounds_that_are_not_close(n, kv, H, KH, D, prefix, e4m3, max_q, max_kv):
    p = Padded(n, kv, KH, D, 16, wide=8000, max_q=max_q, max_kv=max_kv, prefix=prefix, e4m3=e4m3, seed=91)
    for workspace in ("all", "half", "none"):
        p.check_attention(H, workspace=workspace)
