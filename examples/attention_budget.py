"""Decoding within a budget of memory: a paged cache of 4-bit cells in which no sequence has more than `keep` tokens of any key head.

A prompt goes in whole and is cut down to the budget; then every step appends one token to each sequence, attends, adds up the attention weights that the
cached tokens got, and evicts the token of each key head that has the least.  Tokens keep the positions that they had in the text; what stays of the cache lies in its first slots,
in no order.

    python examples/attention_budget.py            # on an MI355X; prints the time of a decoding step
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.attention_layer import rope_table  # noqa: E402
from paper_2509_23410_amd import binding as B  # noqa: E402


class BudgetCache:
    """The cache of one layer for n_seqs sequences: `keep` tokens of each key head, the first `sinks` and the last `recent` always, and room for `most` before a cut."""

    def __init__(self, n_seqs, heads, kv_heads, head_dim, keep, sinks, recent, most, n_pos, page_size=64, decay=1.0, workspace_bytes=64 << 20):
        self.n, self.heads, self.kv_heads, self.head_dim = n_seqs, heads, kv_heads, head_dim
        self.keep, self.sinks, self.recent, self.decay = keep, sinks, recent, decay
        per = -(-most // page_size)
        self.most, pages = per * page_size, per * n_seqs
        byte = lambda *shape: torch.zeros(*shape, device="cuda", dtype=torch.uint8)  # noqa: E731
        self.k, self.v = byte(pages, kv_heads, page_size, head_dim // 2), byte(pages, kv_heads, head_dim // 2, page_size)
        self.k_scale, self.v_scale = byte(pages, kv_heads, page_size, head_dim // 32), byte(pages, kv_heads, head_dim // 32, page_size)
        self.cache = B.KVCache4(self.k, self.v, self.k_scale, self.v_scale, pages, page_size, kv_heads, head_dim)
        self.table = torch.arange(pages, device="cuda", dtype=torch.int32).view(n_seqs, per)
        self.rope = B.Rope(rope_table(n_pos, head_dim), n_pos, head_dim)
        self.kv_len = torch.zeros(n_seqs, device="cuda", dtype=torch.int32)
        self.weights = torch.zeros(n_seqs, kv_heads, self.most, device="cuda")
        self.slot_positions = torch.zeros(n_seqs, kv_heads, self.most, device="cuda", dtype=torch.int32)
        self.moved_from = torch.empty(n_seqs, kv_heads, keep, device="cuda", dtype=torch.int32)
        self.workspace = torch.empty(workspace_bytes, device="cuda", dtype=torch.uint8)

    def step(self, qkv, O, positions, q_start, n_tokens, max_q):
        """O (n_tokens x heads * head_dim bf16) = attention of the new tokens, whose q, k and v lie side by side in qkv's fp32 rows, appended to what there is.
        positions: of the tokens in their texts; kv_len has them counted already.  -> lse"""
        st, H, KH, D, row = torch.cuda.current_stream().cuda_stream, self.heads, self.kv_heads, self.head_dim, qkv.shape[1]
        part = lambda first, heads, **kw: B.Heads(qkv.data_ptr() + 4 * first * D, heads, row, f32=True, **kw)  # noqa: E731
        Q, lse = torch.empty_like(O), torch.empty(n_tokens, H, device="cuda")
        seqs = B.Seqs(self.n, n_tokens, self.kv_len, self.table, self.table.shape[1], max_q, self.most, q_start=q_start)
        B.patch_kv_append4(part(H, KH), part(H + KH, KH), seqs, self.cache, st, rope=self.rope, q=part(0, H, out=Q, out_stride=H * D), positions=positions)
        B.patch_attention4(Q, H, seqs, self.cache, O, st, lse=lse, workspace=self.workspace)
        B.patch_attention_weights4(Q, H, seqs, self.cache, lse, self.weights, self.weights, self.most, st, decay=self.decay, positions=positions,
                                   slot_positions=self.slot_positions)
        B.patch_kv_evict4(seqs, self.cache, self.weights, self.weights, self.most, self.keep, self.moved_from, self.kv_len, st, sinks=self.sinks, recent=self.recent,
                          positions=self.slot_positions, positions_out=self.slot_positions)
        return lse


def run(prompt=(3000, 1700, 2500, 4000), heads=32, kv_heads=8, head_dim=128, keep=1024, sinks=4, recent=128, steps=32, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, most = len(prompt), max(max(prompt), keep + 1)
    c = BudgetCache(n, heads, kv_heads, head_dim, keep, sinks, recent, most, max(prompt) + steps)
    width = (heads + 2 * kv_heads) * head_dim
    start = torch.tensor([0, *torch.tensor(prompt).cumsum(0).tolist()], device="cuda", dtype=torch.int32)
    positions = torch.cat([torch.arange(p, device="cuda", dtype=torch.int32) for p in prompt])
    c.kv_len.add_(start[1:] - start[:-1])
    O = torch.empty(sum(prompt), heads * head_dim, device="cuda", dtype=torch.bfloat16)
    c.step(torch.randn(sum(prompt), width, device="cuda", generator=g), O, positions, start, sum(prompt), max(prompt))
    one, positions = torch.arange(n + 1, device="cuda", dtype=torch.int32), torch.tensor(prompt, device="cuda", dtype=torch.int32)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for t in range(steps):
        if t == steps // 2:
            begin.record()
        c.kv_len.add_(1)
        c.step(torch.randn(n, width, device="cuda", generator=g), O[:n], positions, one, n, 1)
        positions.add_(1)
    end.record()
    torch.cuda.synchronize()
    print(f"decoding step of {n} sequences within {keep} tokens: {1e3 * begin.elapsed_time(end) / (steps - steps // 2):.1f} us")
    return c, O[:n]


if __name__ == "__main__":
    run()
