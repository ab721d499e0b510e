"""A single token in place, whose strides tell nothing, and rows of q, k and v side by side in place."""
import pytest
import torch

import attention_ref as R
from paper_2509_23410_amd import binding as B
from test_gpu_attention import _rope_bound

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,stride,out_stride", [(1, 9 * 128, 8 * 128), (1, 8 * 128, 16 * 128), (40, 9 * 128, 9 * 128), (1300, 24 * 128, 24 * 128)])
def test_in_place(T, stride, out_stride):
    H, D = 8, 128
    x = torch.randn(T, max(stride, out_stride), generator=torch.Generator().manual_seed(T)).to(torch.bfloat16)
    table, pos = R.table_of(T + 5, D), torch.arange(T, dtype=torch.int32) + 3
    dx, dt = x.cuda(), table.cuda()
    B.patch_qk_rope(B.Heads(dx, H, stride, out=dx, out_stride=out_stride), None, pos.cuda(), T, D, B.Rope(dt, T + 5, D), torch.cuda.current_stream().cuda_stream)
    y, mag = R.rotated(x[:, : H * D].reshape(T, H, D), None, 0, table, pos, D, False)
    got = dx.cpu()
    assert ((got[:, : H * D].double().view(T, H, D) - y).abs() - _rope_bound(y, mag)).max() <= 0
    assert torch.equal(got[:, H * D:], x[:, H * D:])
