"""A cache that has to hold more: cells of 4 bits, and fewer tokens, as a serving program calls them.

Four operators of ``paper_2509_23410_amd.binding`` beside the append and the attention over a paged cache of bf16 or e4m3 cells:

  op "append"   patch_kv_append4: the new tokens' K and V into a cache of 4-bit cells, and what those cells stand for
     "attend"   patch_attention4: causal attention of the new tokens over the pages of such a cache
     "weigh"    patch_attention_weights (4): every cached token's sum of attention weights, faded and with the new rows' added
     "evict"    patch_kv_evict (4): of each key head's tokens those of the largest weight stay, in pages that are dense again

Cells of 4 bits ("e2m1": 0 .5 1 1.5 2 3 4 6 and a sign) stand two to a byte, beside one power of two for 32 features of a token: a byte, 2^(byte - 127), 255
for a NaN.  It is the smallest power of two of which the largest of the 32 values is at most seven, from 2^-100 to 2^125.  All of that is exact
arithmetic, so bytes of such pages are compared as they are; the append also gives the values that they stand for.

Sizes are those of the decoders this repository measures its linear layers on (14 query heads over 2 of 64, 32 over 32 and 32
over 8 of 128, 40 over 40 of 128) and a few generic ones.  A case is a dict:
  q_heads, kv_heads, head_dim
  cells      "bf16", "e4m3" (8-bit floats with a factor per head) or "e2m1"
  f32        rows to append are fp32 (else bf16)
  page       tokens in a page
  seqs, q    sequences, and the most new tokens of any
  context    tokens of the longest sequence, the shared ones and the new ones among them; the others have less
  spread     how much less: the shortest has (1 - spread) of what the longest has of its own
  prefix     tokens at the front that all sequences share
  lse        the logarithm of every softmax' sum is asked for, too
  decay      what a weight keeps of itself
  moved      tokens of the cache are in no order any more (it was evicted from before): their positions go with them
  keep, sinks, recent   tokens that stay, the first ones and the last ones that always do
"""
import math

import numpy as np
import torch

own = False
WORKSPACE_BYTES = 256 << 20   # one scratch buffer per program


def _case(name, op, heads, **kw):
    q_heads, kv_heads, head_dim = heads
    c = dict(name=name, op=op, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, cells="e2m1", f32=False, page=64, seqs=1, q=1, context=1, spread=0.0, prefix=0,
             lse=False, decay=1.0, moved=False, keep=0, sinks=0, recent=0)
    c.update(kw)
    return c


def listed():
    return [
        # a serving batch's new tokens into their pages: latency, and writes of single bytes
        _case("append4_decode_64", "append", (32, 8, 128), seqs=64, context=8192, spread=0.9),
        # two prompts of ragged lengths, straight from an fp32 product
        _case("append4_prompt", "append", (32, 32, 128), f32=True, page=32, seqs=2, q=1100, context=1100, spread=0.3),
        # one sequence of a small model, a few hundred tokens in: the smallest attention
        _case("attend4_1_small", "attend", (14, 2, 64), page=16, seqs=1, context=500),
        # one very long sequence: the only rows are its heads, the work is its keys
        _case("attend4_1_long", "attend", (32, 8, 128), seqs=1, context=131000),
        # a batch of ragged contexts, no shared front, one key head per query head
        _case("attend4_decode_29", "attend", (40, 40, 128), page=32, seqs=29, context=8000, spread=0.95, lse=True),
        # a batch behind one long system prompt, drafted tokens
        _case("attend4_shared_64", "attend", (32, 8, 128), seqs=64, q=3, context=9000, spread=0.9, prefix=8192),
        # pieces of ragged prompts behind what they have in the cache
        _case("attend4_pieces_700", "attend", (32, 8, 128), page=128, seqs=6, q=700, context=2500, spread=0.6),
        # weights after a step of a batch, over 4-bit cells that were evicted from before
        _case("weigh_decode_32", "weigh", (32, 8, 128), seqs=32, context=8000, spread=0.7, decay=0.99, moved=True),
        # weights of a whole prompt
        _case("weigh_prompt_4096", "weigh", (32, 32, 128), cells="bf16", seqs=1, q=4096, context=4096),
        # one token too many in each sequence: the step of a batch that lives within a budget
        _case("evict_step_64", "evict", (32, 8, 128), cells="bf16", seqs=64, context=4097, keep=4096, sinks=4, recent=512, moved=True),
        # prompts cut down to their budget, 8-bit cells
        _case("evict_prompt_4", "evict", (32, 32, 128), cells="e4m3", page=32, seqs=4, context=16000, spread=0.5, keep=2048, sinks=4, recent=256),
        # a quarter of one very long sequence stays, 4-bit cells
        _case("evict_1_long", "evict", (32, 8, 128), seqs=1, context=131000, keep=32768, sinks=4, recent=1024),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    heads = rng.choice([(14, 2, 64), (32, 32, 128), (32, 8, 128), (40, 40, 128), (32, 8, 64), (8, 4, 256), (16, 1, 128), (12, 4, 64), (4, 1, 256)])
    op = rng.choice(["append", "attend", "attend", "weigh", "evict"])
    c = _case("", op, heads, page=rng.choice([16, 32, 64, 128]), spread=round(rng.random(), 3))
    del c["name"]
    per_token = heads[1] * heads[2]
    if op in ("weigh", "evict"):
        c["cells"] = rng.choice(["bf16", "e4m3", "e2m1"])
        c["moved"] = rng.random() < 0.5
    if op == "append":
        c["f32"] = rng.random() < 0.5
        c["seqs"] = _log(rng, 1, 128)
        c["q"] = _log(rng, 1, max(1, 2200 * 32 * 128 // (per_token * c["seqs"])))
        c["context"] = c["q"] + _log(rng, 1, 65536 // c["seqs"])
    elif op == "evict":
        c["seqs"] = _log(rng, 1, 128)
        most = min(131000, 131_000_000 // (c["seqs"] * per_token))      # cells of K: those of the long listed case
        c["context"] = _log(rng, min(64, most), most)
        c["keep"] = c["context"] - 1 if rng.random() < 0.3 else _log(rng, 1, c["context"])
        c["keep"] = max(1, c["keep"])
        c["sinks"] = min(c["keep"], rng.choice([0, 1, 4, 64]))
        c["recent"] = rng.randrange(c["keep"] - c["sinks"] + 1)
    elif rng.random() < 0.6:     # decoding: few new tokens each
        c["seqs"] = _log(rng, 1, 128)
        c["q"] = rng.choice([1, 1, 1, _log(rng, 1, 8)])
        most = max(16, 131_000_000 // (c["seqs"] * per_token))
        c["context"] = c["q"] + _log(rng, min(64, most), min(131000, most))
    else:                        # prompts and pieces of them
        c["seqs"] = _log(rng, 1, 8)
        c["q"] = _log(rng, 9, 2048 // c["seqs"])
        c["context"] = c["q"] + _log(rng, 1, 2048)
    if op == "attend":
        c["lse"] = rng.random() < 0.3
        c["prefix"] = rng.choice([0, rng.randrange(c["context"] - c["q"] + 1)])
    if op == "weigh":
        c["decay"] = rng.choice([1.0, 0.99, 0.5])
    return c


def lengths(case):
    """(new tokens, tokens in the cache) of every sequence: whole numbers that the case alone fixes."""
    n, front = [], []
    for s in range(case["seqs"]):
        part = 1.0 - case["spread"] * ((0.61803398875 * s) % 1.0)
        n.append(max(1, int(case["q"] * part)))
        front.append(int((case["context"] - case["prefix"] - case["q"]) * part))
    return n, [case["prefix"] + f + k for f, k in zip(front, n)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n_q, kv = lengths(case)
    T, B, H, KH, D, page, prefix = sum(n_q), case["seqs"], case["q_heads"], case["kv_heads"], case["head_dim"], case["page"], case["prefix"]
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    i32 = lambda a: torch.tensor(a, device="cuda", dtype=torch.int32)  # noqa: E731
    s = dict(case=case, T=T, q_start=i32(np.concatenate([[0], np.cumsum(n_q)]).tolist()), kv_len=i32(kv), max_q=max(n_q), max_kv=max(kv),
             stream=torch.cuda.current_stream().cuda_stream)
    s["positions"] = i32(np.concatenate([np.arange(L - n, L) for n, L in zip(n_q, kv)]).tolist())
    # the cache: pages in no order, those of the shared front in every row of the table
    per = [-(-L // page) for L in kv]
    shared = prefix // page
    n_pages = shared + sum(p - shared for p in per) + 3
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table, at = np.full((B, max(per)), -1, np.int32), shared
    for b in range(B):
        table[b, :shared] = order[:shared]
        table[b, shared:per[b]] = order[at:at + per[b] - shared]
        at += per[b] - shared
    s["page_table"] = i32(table.tolist())
    s["k_scale"] = s["v_scale"] = None
    if case["cells"] == "e2m1":
        byte = lambda lo, hi, *shape: torch.randint(lo, hi, shape, device="cuda", generator=gen, dtype=torch.uint8)  # noqa: E731
        s["k"], s["v"] = byte(0, 256, n_pages, KH, page, D // 2), byte(0, 256, n_pages, KH, D // 2, page)
        # 2^-2 for most, as values of around 1 have, and larger and smaller ones
        s["k_scale"], s["v_scale"] = byte(124, 127, n_pages, KH, page, D // 32), byte(124, 127, n_pages, KH, D // 32, page)
    else:
        s["k"], s["v"] = normal(n_pages, KH, page, D).to(torch.bfloat16), normal(n_pages, KH, D, page).to(torch.bfloat16)
        if case["cells"] == "e4m3":
            s["k_scale"], s["v_scale"] = 0.01 + 0.02 * torch.rand(KH, device="cuda", generator=gen), 0.01 + 0.02 * torch.rand(KH, device="cuda", generator=gen)
            s["k"] = (s["k"].float() / s["k_scale"][:, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
            s["v"] = (s["v"].float() / s["v_scale"][:, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    rest = prefix - shared * page
    if rest:                                                            # a page that the front ends in: each sequence has a copy
        copies = s["page_table"][:, shared].long()
        for name, axis in (("k", 2), ("v", 3), ("k_scale", 2), ("v_scale", 3)):
            if s[name] is not None:
                part = s[name].narrow(axis, 0, rest)
                part[copies] = part[copies[0]].clone()
    if case["op"] == "append":
        # rows of a product whose features are k and v side by side; some features are larger than others
        s["kv"] = (normal(T, 2 * KH * D) * torch.exp(0.3 * normal(2 * KH * D))).to(torch.float32 if case["f32"] else torch.bfloat16)
        s["K_out"], s["V_out"] = (torch.empty(T, KH * D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    if case["op"] in ("attend", "weigh"):
        s["Q"] = normal(T, H * D).to(torch.bfloat16)
        s["lse"] = torch.empty(T, H, device="cuda")
    if case["op"] == "attend":
        s["O"] = torch.empty_like(s["Q"])
        s["workspace"] = torch.empty(WORKSPACE_BYTES, device="cuda", dtype=torch.uint8)
    if case["op"] in ("weigh", "evict"):
        s["stride"] = max(per) * page
        # sums of weights so far: a few tokens have most, and many that nobody looked at have nothing
        w = torch.exp(2 * normal(B, KH, s["stride"]) - 6)
        s["w"] = torch.where(w > 2e-4, w, 0.0)
        s["w_out"] = torch.zeros_like(s["w"])
        s["slot_pos"] = s["pos_out"] = None
        if case["moved"]:
            # where each slot's token was in the text; the last tokens of the call are in the last slots
            s["slot_pos"] = torch.zeros(B, KH, s["stride"], device="cuda", dtype=torch.int32)
            for b in range(B):
                L = kv[b] - n_q[b]
                s["slot_pos"][b, :, :L] = torch.rand(KH, L, device="cuda", generator=gen).argsort(1).int()
                s["slot_pos"][b, :, L:kv[b]] = torch.arange(L, kv[b], device="cuda", dtype=torch.int32)
            s["pos_out"] = s["slot_pos"].clone()
    if case["op"] == "weigh":
        _plain_lse(s)                                                   # what the step's attention said
    if case["op"] == "evict":
        s["from"] = torch.empty(B, KH, case["keep"], device="cuda", dtype=torch.int32)
        s["kv_len_out"] = torch.empty_like(s["kv_len"])
    return s


# ---- the plain form -------------------------------------------------------------------------------------------------


def _e2m1_values(device="cuda"):
    half = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=device)
    return torch.cat([half, -half])


def _power(byte):
    """2^(byte - 127), NaN for 255."""
    return torch.where(byte == 255, math.nan, torch.exp2(byte.float() - 127))


def _encode(x):
    """... x D values in 32 bits -> (codes 0 .. 15, bytes of the powers of two, the values that they stand for)."""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    mantissa, exponent = torch.frexp(top)                               # top = mantissa * 2^exponent, mantissa in [1/2, 1)
    power = (exponent - 3 + (mantissa > 0.875)).clamp(-100, 125)
    power = torch.where(top == 0, -100, power)
    y = (x.abs() * torch.exp2(-power.float())[..., None]).clamp(max=6)
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))        # round() gives ties to the even multiple of the step, which is the even code
    y = torch.round(y / step) * step
    code = torch.bucketize(y, _e2m1_values()[:8].contiguous()) + 8 * torch.signbit(x)
    value = torch.where(x < 0, -y, y) * torch.exp2(power.float())[..., None]
    return code.flatten(-2).to(torch.uint8), (power + 127).to(torch.uint8), value.flatten(-2)


def _plain_append(s):
    case, page, KH, D = s["case"], s["case"]["page"], s["case"]["kv_heads"], s["case"]["head_dim"]
    seq = torch.bucketize(torch.arange(s["T"], device="cuda", dtype=torch.int32), s["q_start"][1:], right=True)
    at = s["positions"].long()
    where, slot = s["page_table"][seq, at // page].long(), at % page
    k, v = s["kv"].view(s["T"], 2, KH, D).float().unbind(1)
    code, power, value = _encode(k)
    s["k"][where, :, slot] = code[..., 0::2] | code[..., 1::2] << 4
    s["k_scale"][where, :, slot] = power
    s["K_out"].copy_(value.flatten(1))
    code, power, value = _encode(v)
    s["v"][where, :, :, slot] = code[..., 0::2] | code[..., 1::2] << 4
    s["v_scale"][where, :, :, slot] = power
    s["V_out"].copy_(value.flatten(1))


def _keys(s):
    """K in 32 bits of all sequences' pages, B x KH x tokens x D."""
    table = s["page_table"].clamp(min=0).long()
    if s["case"]["cells"] == "e2m1":
        values, k = _e2m1_values(), s["k"][table].int()
        k = torch.stack([values[k & 15], values[k >> 4]], -1).flatten(-2)
        k = (k.unflatten(-1, (-1, 32)) * _power(s["k_scale"][table])[..., None]).flatten(-2)
    elif s["case"]["cells"] == "e4m3":
        k = s["k"].view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * s["k_scale"][:, None, None]
    else:
        k = s["k"][table].float()
    return k.transpose(1, 2).flatten(2, 3)


def _values(s):
    """V of 4-bit cells in 32 bits, B x KH x tokens x D."""
    table = s["page_table"].clamp(min=0).long()
    values, v = _e2m1_values(), s["v"][table].int()
    v = torch.stack([values[v & 15], values[v >> 4]], -2).flatten(-3, -2) # pages x KH x D x tokens
    v = v * _power(s["v_scale"][table]).repeat_interleave(32, -2)
    return v.permute(0, 2, 1, 4, 3).flatten(2, 3)


def _scores(s):
    """(scores in 32 bits, minus infinity where a row does not see a key: B x KH x G x n x tokens; which of the n are tokens, and of which rows)."""
    case, n = s["case"], s["max_q"]
    KH, G, D = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["head_dim"]
    new = s["q_start"][1:] - s["q_start"][:-1]
    i = torch.arange(n, device="cuda", dtype=torch.int32)
    real = i < new[:, None]
    token = (s["q_start"][:-1, None] + i).clamp(max=s["T"] - 1).long()
    last = torch.where(real, (s["kv_len"] - new)[:, None] + i, -1)      # the last key that a row sees
    q = s["Q"].view(s["T"], KH, G, D)[token].float().permute(0, 2, 3, 1, 4)
    k = _keys(s)
    score = (q.flatten(2, 3) @ k.transpose(2, 3)).view(case["seqs"], KH, G, n, -1) * D ** -0.5
    sees = torch.arange(k.shape[2], device="cuda", dtype=torch.int32) <= last[..., None]
    return torch.where(sees[:, None, None], score, -math.inf), real, token


def _plain_lse(s):
    score, real, _ = _scores(s)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    lse = (top + torch.log(torch.exp(score - top).sum(-1, keepdim=True)))[..., 0]
    s["lse"].copy_(lse.permute(0, 3, 1, 2)[real].view(s["T"], -1))


def _plain_attend(s):
    score, real, _ = _scores(s)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1)
    used = torch.arange(p.shape[-1], device="cuda", dtype=torch.int32) < s["kv_len"][:, None]
    v = torch.where(used[:, None, :, None], _values(s), 0.0)
    out = (p.flatten(2, 3) @ v).view(*p.shape[:4], -1)
    s["O"].copy_(out.permute(0, 3, 1, 2, 4)[real].view(s["T"], -1))
    if s["case"]["lse"]:
        s["lse"].copy_((top + torch.log(total))[..., 0].permute(0, 3, 1, 2)[real].view(s["T"], -1))


def _plain_weigh(s):
    case = s["case"]
    score, real, token = _scores(s)
    lse = s["lse"].view(s["T"], case["kv_heads"], -1)[token].permute(0, 2, 3, 1)
    p = torch.exp(score - lse[..., None])
    p = torch.where(real[:, None, None, :, None], p, 0.0).sum((2, 3))   # B x KH x tokens
    new = s["q_start"][1:] - s["q_start"][:-1]
    slot = torch.arange(s["stride"], device="cuda", dtype=torch.int32)
    old, there = slot < (s["kv_len"] - new)[:, None], slot < s["kv_len"][:, None]
    s["w_out"].copy_(torch.where(there[:, None], p + torch.where(old[:, None], case["decay"] * s["w"], 0.0), s["w_out"]))
    if case["moved"]:
        at = (s["q_start"][:-1, None] + slot - (s["kv_len"] - new)[:, None]).clamp(0, s["T"] - 1).long()
        s["pos_out"].copy_(torch.where((there & ~old)[:, None], s["positions"][at][:, None], s["slot_pos"]))


def _plain_evict(s):
    case, keep = s["case"], s["case"]["keep"]
    B, KH, page, L = case["seqs"], case["kv_heads"], case["page"], s["stride"]
    slot = torch.arange(L, device="cuda", dtype=torch.int32)
    there = (slot < s["kv_len"][:, None])[:, None].expand(B, KH, L)
    pos = s["slot_pos"] if case["moved"] else slot.expand(B, KH, L)
    newest = torch.where(there, pos, -1).amax(-1, keepdim=True)
    always = (pos < case["sinks"]) | (pos > newest - case["recent"])
    rank = torch.where(there, torch.where(always, math.inf, s["w"]), -math.inf)
    best = rank.sort(stable=True, dim=-1, descending=True).indices
    stays = torch.zeros(B, KH, L, device="cuda", dtype=torch.bool).scatter_(-1, best[..., :keep], True) & there
    # slots behind the budget whose tokens stay, and slots within it whose tokens do not, both from the first on
    within = slot < keep
    mover, hole = stays & ~within, there & within & ~stays
    source = torch.where(mover, slot, L).sort(dim=-1).values
    rank_of_hole = (hole.cumsum(-1) - 1).clamp(min=0)
    came = torch.where(stays & within, slot, torch.where(hole, source.gather(-1, rank_of_hole), -1))[..., :keep].int()
    s["from"].copy_(came)
    s["kv_len_out"].copy_(s["kv_len"].clamp(max=keep))
    real, at = came >= 0, came.clamp(min=0).long()
    s["w_out"][..., :keep] = torch.where(real, s["w"].gather(-1, at), s["w_out"][..., :keep])
    if case["moved"]:
        s["pos_out"][..., :keep] = torch.where(real, s["slot_pos"].gather(-1, at), s["pos_out"][..., :keep])
    b, h, to = torch.nonzero(came != torch.where(real, slot[:keep], -1), as_tuple=True)
    source = at[b, h, to]
    src, dst = s["page_table"][b, source // page].long(), s["page_table"][b, to // page].long()
    for name in ("k", "k_scale"):
        if case["cells"] == "e2m1" or name == "k":
            cells = s[name].view(torch.uint8)
            cells[dst, h, to % page] = cells[src, h, source % page]
    for name in ("v", "v_scale"):
        if case["cells"] == "e2m1" or name == "v":
            cells = s[name].view(torch.int16 if case["cells"] == "bf16" else torch.uint8)
            cells[dst, h, :, to % page] = cells[src, h, :, source % page]


# ---- the framework's calls ------------------------------------------------------------------------------------------


def _handles(s):
    """What a program makes once for its model and its batch: descriptors of the buffers above."""
    from paper_2509_23410_amd import binding as B
    case = s["case"]
    KH, D, pages = case["kv_heads"], case["head_dim"], s["k"].shape[0]
    h = dict(B=B)
    if case["cells"] == "e2m1":
        h["cache"] = B.KVCache4(s["k"], s["v"], s["k_scale"], s["v_scale"], pages, case["page"], KH, D)
    else:
        h["cache"] = B.KVCache(s["k"], s["v"], pages, case["page"], KH, D, e4m3=case["cells"] == "e4m3", k_scale=s["k_scale"], v_scale=s["v_scale"])
    h["seqs"] = B.Seqs(case["seqs"], s["T"], s["kv_len"], s["page_table"], s["page_table"].shape[1], s["max_q"], s["max_kv"], q_start=s["q_start"])
    if case["op"] == "append":
        part = lambda i, out: B.Heads(s["kv"].data_ptr() + i * KH * D * s["kv"].element_size(), KH, 2 * KH * D, f32=case["f32"], out=out, out_stride=KH * D)  # noqa: E731
        h["k"], h["v"] = part(0, s["K_out"]), part(1, s["V_out"])
    return h


def _own(s):
    case = s["case"]
    h = s.get("handles") or s.setdefault("handles", _handles(s))
    B, four = h["B"], case["cells"] == "e2m1"
    if case["op"] == "append":
        B.patch_kv_append4(h["k"], h["v"], h["seqs"], h["cache"], s["stream"])
    elif case["op"] == "attend":
        B.patch_attention4(s["Q"], case["q_heads"], h["seqs"], h["cache"], s["O"], s["stream"], prefix_len=case["prefix"], lse=s["lse"] if case["lse"] else None,
                           workspace=s["workspace"])
    elif case["op"] == "weigh":
        weigh = B.patch_attention_weights4 if four else B.patch_attention_weights
        weigh(s["Q"], case["q_heads"], h["seqs"], h["cache"], s["lse"], s["w"], s["w_out"], s["stride"], s["stream"], decay=case["decay"],
              positions=s["positions"] if case["moved"] else None, slot_positions=s["pos_out"])
    else:
        evict = B.patch_kv_evict4 if four else B.patch_kv_evict
        evict(h["seqs"], h["cache"], s["w"], s["w_out"], s["stride"], case["keep"], s["from"], s["kv_len_out"], s["stream"], sinks=case["sinks"], recent=case["recent"],
              positions=s["slot_pos"], positions_out=s["pos_out"])


def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if own:
        _own(s)
    else:
        dict(append=_plain_append, attend=_plain_attend, weigh=_plain_weigh, evict=_plain_evict)[op](s)
    out = dict(append=("k", "v", "k_scale", "v_scale", "K_out", "V_out"), attend=("O",) + (("lse",) if case["lse"] else ()), weigh=("w_out",),
               evict=("from", "kv_len_out", "w_out", "k", "v") + (("k_scale", "v_scale") if case["cells"] == "e2m1" else ()))[op]
    return {name: s[name] for name in out + (("pos_out",) if case["moved"] else ())}


def work(case):
    n_q, kv = lengths(case)
    T, H, KH, D = sum(n_q), case["q_heads"], case["kv_heads"], case["head_dim"]
    cell = {"bf16": 2, "e4m3": 1, "e2m1": 17 / 32}[case["cells"]]       # bytes, the powers of two among them
    seen = sum(n * (L - n) + n * (n + 1) // 2 for n, L in zip(n_q, kv))  # pairs of a token and a key
    if case["op"] == "append":
        return {"bytes": T * KH * D * 2 * ((4 if case["f32"] else 2) + cell + 2), "flops": T * KH * D * 2 * 3}
    if case["op"] == "attend":
        P = case["prefix"]
        return {"bytes": (P + sum(L - P for L in kv)) * KH * D * 2 * cell + 2 * T * H * D * 2 + (4 * T * H if case["lse"] else 0), "flops": 4 * H * D * seen}
    if case["op"] == "weigh":
        return {"bytes": sum(kv) * KH * (D * cell + 8) + T * H * (2 * D + 4), "flops": 2 * H * D * seen}
    b = f = 0
    for L in kv:
        n = min(L, case["keep"])
        b += KH * (L * (8 if case["moved"] else 4) + n * (12 if case["moved"] else 8))
        f += KH * L
        # about as many tokens move as stay from behind the budget: all the last ones there, and of the others the share that stays
        behind = L - n
        last = min(behind, case["recent"])
        b += KH * D * 2 * cell * 2 * (last + (behind - last) * (n - last) // max(1, L - last))
    return {"bytes": b, "flops": f}


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------------


def _exact_cells(s, name, pages):
    """K or V of these pages in 64 bits, KH x tokens x D."""
    case = s["case"]
    raw = s[name].view(torch.int16 if case["cells"] == "bf16" else torch.uint8)[pages].view(s[name].dtype)
    if name == "v":
        raw = raw.transpose(-1, -2)                                     # a token's cells side by side
    if case["cells"] == "e2m1":
        low, high = (raw % 16).long(), (raw // 16).long()
        code = torch.empty(*raw.shape[:-1], 2 * raw.shape[-1], device=raw.device, dtype=torch.long)
        code[..., 0::2], code[..., 1::2] = low, high
        e, m = code // 2 % 4, code % 2
        x = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * 2.0 ** (e - 1).double()) * (1 - 2 * (code // 8))
        scale = s[name + "_scale"][pages]
        scale = scale.transpose(-1, -2) if name == "v" else scale
        x = x.double() * (2.0 ** (scale.double() - 127)).repeat_interleave(32, -1)
    else:
        x = raw.double()
        if s[name + "_scale"] is not None:
            x = x * s[name + "_scale"].double()[:, None, None]
    return x.permute(1, 0, 2, 3).flatten(1, 2)


def _exact_stored(x):
    """What 4-bit cells stand for, from the definition: every candidate's distance, ties to the even one."""
    values = torch.tensor([0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0], device=x.device, dtype=torch.float64)   # even codes first: argmin takes the first of a tie
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    power = torch.full_like(top, -100)
    for p in range(-100, 126):
        power = torch.where(top > 7 * 2.0 ** p, min(p + 1, 125), power)
    y = x.abs() / (2.0 ** power)[..., None]
    return (values[(y[..., None] - values).abs().argmin(-1)] * x.sign() * (2.0 ** power)[..., None]).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    n_q, kv = lengths(case)
    H, KH, D, page, T = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"], s["T"]
    if case["op"] == "append":
        k, v = s["kv"].view(T, 2, KH, D).unbind(1)
        return dict(k=None, v=None, k_scale=None, v_scale=None, K_out=_exact_stored(k).flatten(1), V_out=_exact_stored(v).flatten(1))
    if case["op"] == "evict":
        w, w_out = s["w"].cpu().numpy(), s["w_out"].double().cpu().numpy()
        for b in range(case["seqs"]):
            for h in range(KH):
                pos = s["slot_pos"][b, h, : kv[b]].cpu().numpy() if case["moved"] else np.arange(kv[b])
                stays = set(np.lexsort((np.arange(kv[b]), -w[b, h, : kv[b]].astype(np.float64), ~((pos < case["sinks"]) | (pos > pos.max() - case["recent"]))))[: case["keep"]].tolist())
                late = iter(sorted(i for i in stays if i >= case["keep"]))
                for i in range(min(kv[b], case["keep"])):
                    w_out[b, h, i] = w[b, h, i if i in stays else next(late)]
        none = {name: None for name in ("from", "kv_len_out", "k", "v", "k_scale", "v_scale", "pos_out")}
        return dict(none, w_out=torch.from_numpy(w_out))
    Q, t = s["Q"].double(), 0
    O, lse = torch.empty(T, H, D, device="cuda", dtype=torch.float64), torch.empty(T, H, device="cuda", dtype=torch.float64)
    w_out = s["w_out"].double() if case["op"] == "weigh" else None
    for b in range(case["seqs"]):
        pages = s["page_table"][b, : -(-kv[b] // page)].long()
        k = _exact_cells(s, "k", pages)[:, : kv[b]]
        v = _exact_cells(s, "v", pages)[:, : kv[b]] if case["op"] == "attend" else None
        hidden = torch.arange(kv[b], device="cuda")[None, :] > torch.arange(kv[b] - n_q[b], kv[b], device="cuda")[:, None]
        if w_out is not None:
            old = kv[b] - n_q[b]
            w_out[b, :, :old] = s["w"][b, :, :old].double() * case["decay"]
        for h in range(H):
            z = (Q[t:t + n_q[b], h * D:(h + 1) * D] @ k[h * KH // H].T / math.sqrt(D)).masked_fill(hidden, -math.inf)
            if w_out is not None:
                w_out[b, h * KH // H, : kv[b]] += torch.exp(z - s["lse"][t:t + n_q[b], h, None].double()).sum(0)
            else:
                lse[t:t + n_q[b], h] = z.logsumexp(1)
                O[t:t + n_q[b], h] = z.softmax(1) @ v[h * KH // H]
        t += n_q[b]
    if w_out is not None:
        return dict(w_out=w_out, pos_out=None)
    out = dict(O=O.reshape(T, H * D))
    return dict(out, lse=lse) if case["lse"] else out
