"""Decoding batches with idle slots: as many rows as sequences and at most one token each, but not a token for every one of them."""
from types import SimpleNamespace

import pytest
import torch

from padded_batch import Padded
from paper_2509_23410_amd import binding as B
from test_gpu_attention import _check

pytestmark = pytest.mark.gpu

# new tokens and lengths of the sequences; the rows that are left over belong to nobody
IDLE = [([0, 1, 1], [40, 33, 70]), ([1, 1, 0], [40, 33, 70]), ([1, 0, 1, 1], [17, 300, 64, 129]), ([0, 0, 0], [5, 6, 7]),
        ([0 if i % 7 == 3 else 1 for i in range(130)], [1 + (37 * i) % 200 for i in range(130)])]


@pytest.mark.parametrize("n,kv", IDLE)
@pytest.mark.parametrize("prefix", [0, 30])
def test_attention_of_idle_slots(n, kv, prefix):
    p = Padded(n, [L + prefix for L in kv], 2, 64, 16, trail=len(n) - sum(n), max_q=1, prefix=prefix, seed=31)
    for workspace in ("all", "half", "none"):
        p.check_attention(6, workspace=workspace)


@pytest.mark.parametrize("n,kv", IDLE)
def test_append_with_idle_slots(n, kv):
    Padded(n, kv, 2, 64, 16, trail=len(n) - sum(n), max_q=1, seed=32).check_append(H=3, rot=64)


def test_a_step_that_is_captured_once_and_replayed_as_slots_come_and_go():
    """The graph knows the sizes only; which slots have a token is on the device."""
    n, kv, H, KH, D = [1, 1, 1, 1, 1], [90, 33, 64, 200, 17], 4, 2, 64
    p = Padded(n, kv, KH, D, 16, max_q=1, seed=33)
    cache, seqs = p.on_gpu()
    Q = torch.randn(5, H * D, device="cuda").to(torch.bfloat16)
    O = torch.empty_like(Q)
    ws = torch.empty(B.patch_attention_workspace_bytes(H, seqs, cache), device="cuda", dtype=torch.uint8)
    call = lambda: B.patch_attention(Q, H, seqs, cache, O, torch.cuda.current_stream().cuda_stream, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for idle in ((), (1,), (0, 4), (), (2, 3)):
        live = [s for s in range(5) if s not in idle]
        p.start.copy_(torch.tensor([sum(s < i for s in live) for i in range(6)], dtype=torch.int32))
        Q.normal_()
        O.fill_(5.0)
        call()
        eager = O.clone()
        O.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, eager) and (O[len(live):] == 5).all()
        b = p.b
        _check(SimpleNamespace(T=len(live), D=D, KH=KH, n=[1] * len(live), kv=[kv[s] for s in live], ks=[b.ks[s] for s in live], vs=[b.vs[s] for s in live]),
               Q[: len(live)].cpu(), H, O[: len(live)], None)
