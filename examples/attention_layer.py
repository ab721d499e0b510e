"""The attention half of a decoder layer on pruned weights: q / k / v product, append to a paged cache, attention, output product.

A prompt that all sequences share goes through the layer once and fills its pages; then every sequence brings a prompt of its own
(ragged lengths), and after that the batch decodes token by token.  The shared pages are in every sequence's row of the page table, and
every call after the first reads their keys once for the whole batch.

    python examples/attention_layer.py            # on an MI355X; prints the time of a decoding step
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_23410_amd import binding as B, synth  # noqa: E402

WORKSPACE_BYTES = 64 << 20


def rope_table(n_pos: int, rot_dim: int, base: float = 10000.0) -> torch.Tensor:
    """n_pos x 2 x rot_dim / 2 cosines and sines, angles in 64 bits."""
    angle = np.arange(n_pos)[:, None] * base ** (-2.0 * np.arange(rot_dim // 2) / rot_dim)
    return torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], 1).astype(np.float32)).cuda()


class AttentionLayer:
    """Weights w["q"], w["k"], w["v"] (out x hidden) and w["o"] (hidden x heads * head_dim), bf16, pruned to their tile maps."""

    def __init__(self, w, tile_maps, heads, kv_heads, head_dim, tile, n_pages, page_size, max_tokens, n_pos, e4m3=False, scales=(1.0, 1.0)):
        st = torch.cuda.current_stream().cuda_stream
        self.heads, self.kv_heads, self.head_dim, self.page_size = heads, kv_heads, head_dim, page_size
        self.packed = {n: B.patch_pack(w[n], w[n].shape[0], w[n].shape[1], tile_maps[n], tile, st) for n in "qkvo"}
        kind = torch.float8_e4m3fn if e4m3 else torch.bfloat16
        self.k = torch.zeros(n_pages, kv_heads, page_size, head_dim, device="cuda").to(kind)
        self.v = torch.zeros(n_pages, kv_heads, head_dim, page_size, device="cuda").to(kind)
        self.scales = [torch.full((kv_heads,), x, device="cuda") for x in scales] if e4m3 else [None, None]
        self.cache = B.KVCache(self.k, self.v, n_pages, page_size, kv_heads, head_dim, e4m3=e4m3, k_scale=self.scales[0], v_scale=self.scales[1])
        self.table = rope_table(n_pos, head_dim)
        self.rope = B.Rope(self.table, n_pos, head_dim)
        self.gamma = {n: torch.ones(head_dim, device="cuda") for n in "qk"}
        width = heads * head_dim
        self.rows = {n: torch.empty(max_tokens, (heads if n == "q" else kv_heads) * head_dim, device="cuda") for n in "qkv"}
        self.Q = torch.empty(max_tokens, width, device="cuda", dtype=torch.bfloat16)
        self.O = torch.empty_like(self.Q)
        self.workspace = torch.empty(WORKSPACE_BYTES, device="cuda", dtype=torch.uint8)

        def part(n, **kw):
            return B.Heads(self.rows[n], heads if n == "q" else kv_heads, self.rows[n].shape[1], f32=True, **kw)

        self.parts = {"q": part("q", gamma=self.gamma["q"], out=self.Q, out_stride=width), "k": part("k", gamma=self.gamma["k"]), "v": part("v")}

    def forward(self, X, Y, seqs: B.Seqs, n_tokens: int, prefix_len: int = 0) -> None:
        """Y (n_tokens x hidden fp32) = the layer of X (n_tokens x hidden bf16), the batch's new tokens appended."""
        st, ws = torch.cuda.current_stream().cuda_stream, self.workspace
        if n_tokens == 0:
            return
        B.patch_gemm_many(X, n_tokens, [self.packed[n] for n in "qkv"], [self.rows[n] for n in "qkv"], st, workspace=ws)
        B.patch_kv_append(self.parts["k"], self.parts["v"], seqs, self.cache, st, rope=self.rope, q=self.parts["q"])
        B.patch_attention(self.Q, self.heads, seqs, self.cache, self.O, st, prefix_len=prefix_len, workspace=ws)
        B.patch_gemm(self.O, n_tokens, self.packed["o"], Y, st, workspace=ws)


def batch(n_new, kv_len, table, max_kv=None):
    """Seqs of a batch (host lists and a page table on the device)."""
    start = torch.tensor(np.concatenate([[0], np.cumsum(n_new)]), dtype=torch.int32, device="cuda")
    lens = torch.tensor(kv_len, dtype=torch.int32, device="cuda")
    return B.Seqs(len(n_new), int(sum(n_new)), lens, table, table.shape[1], max(n_new), max_kv or max(kv_len), q_start=start)


def make_weights(hidden, heads, kv_heads, head_dim, tile, sparse, seed=0):
    """Seeded weights pruned by a tile map and a 2:4 mask each (bf16, on the device), and the tile maps."""
    st = torch.cuda.current_stream().cuda_stream
    w, maps = {}, {}
    for i, n in enumerate("qkvo"):
        out, k = (hidden, heads * head_dim) if n == "o" else ((heads if n == "q" else kv_heads) * head_dim, hidden)
        c = synth.make_case(f"attention_{n}", out, k, 1, tile, sparse, seed=seed + i)
        W = torch.from_numpy(c.W.view(np.int16)).cuda().view(torch.bfloat16).view(out, k)
        w[n] = torch.empty_like(W)
        B.patch_apply_mask(W, torch.from_numpy(c.mask24).cuda(), c.tile_map, out, k, tile, w[n], st)
        maps[n] = c.tile_map
    return w, maps


def run(hidden=4096, heads=32, kv_heads=8, head_dim=128, tile=128, sparse=0.5, page_size=64, shared=1000, own=(70, 33, 1, 257, 64, 128, 5, 90), steps=16, e4m3=False,
        seed=0):
    """-> (inputs of the shared prompt, of every sequence's tokens, outputs of the last step, the layer's weights)."""
    w, maps = make_weights(hidden, heads, kv_heads, head_dim, tile, sparse, seed)
    last = shared + max(own) + steps
    per = -(-last // page_size)
    whole = shared // page_size
    n_seqs = len(own)
    layer = AttentionLayer(w, maps, heads, kv_heads, head_dim, tile, whole + n_seqs * (per - whole), page_size, max(shared, sum(own)), last, e4m3=e4m3, scales=(0.02, 0.02))
    g = torch.Generator(device="cuda").manual_seed(seed)
    X_shared = torch.randn(shared, hidden, device="cuda", generator=g).to(torch.bfloat16)
    X_own = [torch.randn(n + steps, hidden, device="cuda", generator=g).to(torch.bfloat16) for n in own]
    # page tables: the shared pages, then each sequence's own; the page that the shared prompt ends in is copied for each of them
    table = torch.tensor([list(range(whole)) + [whole + b * (per - whole) + i for i in range(per - whole)] for b in range(n_seqs)], dtype=torch.int32, device="cuda")
    Y = torch.empty(max(shared, sum(own)), hidden, device="cuda")
    layer.forward(X_shared, Y, batch([shared], [shared], table[:1]), shared)
    if shared % page_size:
        for cells in (layer.k.view(torch.uint8), layer.v.view(torch.uint8)):
            cells[table[1:, whole].long()] = cells[table[:1, whole].long()].clone()
    seqs = batch(list(own), [shared + n for n in own], table)
    layer.forward(torch.cat([x[:n] for x, n in zip(X_own, own)]), Y, seqs, sum(own), prefix_len=shared)
    # decoding: one token each; lengths grow on the device, launches are sized for the last step
    kv_len = torch.tensor([shared + n for n in own], dtype=torch.int32, device="cuda")
    seqs = B.Seqs(n_seqs, n_seqs, kv_len, table, table.shape[1], 1, last)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    tokens = [torch.stack([x[n + t] for x, n in zip(X_own, own)]) for t in range(steps)]
    for t in range(steps):
        if t == steps // 2:                                   # (the first ones load what they use)
            begin.record()
        kv_len.add_(1)
        layer.forward(tokens[t], Y, seqs, n_seqs, prefix_len=shared)
    end.record()
    torch.cuda.synchronize()
    print(f"decoding step of {n_seqs} sequences behind {shared} shared tokens: {1e3 * begin.elapsed_time(end) / (steps - steps // 2):.1f} us")
    return X_shared, X_own, Y[:n_seqs], w


if __name__ == "__main__":
    run()
