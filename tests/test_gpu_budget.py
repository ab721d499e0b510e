"""Append, attention, weights and eviction together, as a decoder with a budget runs them (examples/attention_budget.py): against the same steps in 64 bits on the CPU, which
take only the choice of who stays from the weights that the card has."""
import numpy as np
import pytest
import torch

import attention_ref as R
import cache4_ref as C
from examples.attention_budget import BudgetCache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prompt,H,KH,D,keep,sinks,recent,decay", [((70, 9, 40), 4, 2, 64, 32, 2, 8, 1.0), ((50, 33), 8, 1, 128, 33, 0, 1, 0.9), ((20, 90), 4, 2, 256, 16, 4, 4, 0.5)])
def test_decoding_within_a_budget(prompt, H, KH, D, keep, sinks, recent, decay):
    n, G, n_pos, scale = len(prompt), H // KH, 200, D ** -0.5
    c = BudgetCache(n, H, KH, D, keep, sinks, recent, max(max(prompt), keep + 3), n_pos, page_size=16, decay=decay)
    table = R.table_of(n_pos, D)
    g = torch.Generator().manual_seed(1)
    # of each sequence and key head: what its slots stand for, their weights and positions
    state = [[dict(k=torch.zeros(0, D).double(), v=torch.zeros(0, D).double(), w=torch.zeros(0).double(), off=torch.zeros(0).double(), pos=np.zeros(0, np.int64)) for _ in range(KH)]
             for _ in range(n)]
    seen = [0] * n
    for new in [list(prompt)] + [[1] * n] * 5 + [[3, *[0] * (n - 1)], [2] * n]:
        T = sum(new)
        qkv = torch.randn(T, (H + 2 * KH) * D, generator=g)
        positions = torch.cat([torch.arange(seen[s], seen[s] + new[s]) for s in range(n)])
        start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
        O = torch.full((T, H * D), 7.0, device="cuda", dtype=torch.bfloat16)
        c.kv_len.add_(torch.tensor(new, dtype=torch.int32, device="cuda"))
        lse = c.step(qkv.cuda(), O, positions.int().cuda(), start, T, max(new)).cpu().double()
        torch.cuda.synchronize()
        O, came, w_after, pos_after, lens = O.cpu().double().view(T, H, D), c.moved_from.cpu().numpy(), c.weights.cpu(), c.slot_positions.cpu(), c.kv_len.tolist()
        q, _ = R.rotated(qkv[:, : H * D].reshape(T, H, D), None, 0, table, positions, D, False)
        k, _ = R.rotated(qkv[:, H * D:(H + KH) * D].reshape(T, KH, D), None, 0, table, positions, D, False)
        q = q.to(torch.bfloat16).double()                          # (off by a rounding of its neighbours at most: a step of bf16)
        v = C.encode(qkv[:, (H + KH) * D:].reshape(T, KH, D))[2]
        cells = [x.cpu() for x in (c.k, c.k_scale)]
        for s in range(n):
            rows = slice(int(start[s]), int(start[s + 1]))
            for h in range(KH):
                x = state[s][h]
                old = len(x["w"])
                # K after its rotation in fp32 may be a cell off where that falls on the other side of a border: what the card has is taken, and held against k.  Those
                # that moved since are where came says.
                where = {int(f): i for i, f in enumerate(came[s, h]) if f >= 0}
                for i in range(new[s]):
                    slot, t = old + i, rows.start + i
                    kk = C.encode(k[t, h][None])[2][0]
                    if slot in where:
                        at = where[slot]
                        page, p = int(c.table[s, at // 16]), at % 16
                        code = torch.stack([cells[0][page, h, p] & 15, cells[0][page, h, p] >> 4], -1).flatten()
                        got = C.decode(code, cells[1][page, h, p])
                        power = k[t, h].abs().unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32)
                        assert ((got - k[t, h]).abs() <= power * (1.0 / 3.5 + 2.0 ** -16)).all()     # a power is less than the largest over 3.5, half the widest step one of it
                        kk = got
                    x["k"], x["v"] = torch.cat([x["k"], kk[None]]), torch.cat([x["v"], v[t, h][None]])
                x["pos"] = np.concatenate([x["pos"], positions[rows].numpy()])
                if new[s]:
                    gone = [j for j in range(old, old + new[s]) if j not in where]
                    x["w"], x["off"] = torch.cat([x["w"] * decay, torch.zeros(new[s])]), torch.cat([x["off"] * decay + (x["w"] * decay).abs() * 2.0 ** -22, torch.zeros(new[s])])
                    for i in range(new[s]):
                        t, upto = rows.start + i, old + i + 1
                        for e in range(G):
                            head = h * G + e
                            z = x["k"][:upto] @ q[t, head] * scale
                            # a query is off by a step of bf16 (2^-7 of it), a key that has gone already by a cell's step
                            dz = (x["k"][:upto].abs() @ q[t, head].abs()) * scale * 2.0 ** -7 + 1e-4
                            loose = bool(gone)
                            p = torch.exp(z - torch.logsumexp(z, 0))
                            if not loose:
                                assert abs(float(lse[t, head] - torch.logsumexp(z, 0))) <= float(dz.max())
                                o = p @ x["v"][:upto]
                                av = p @ x["v"][:upto].abs()
                                assert ((O[t, head] - o).abs() <= R.BF16_HALF * o.abs() + av * (2 * float(dz.max()) + 2.0 ** -7)).all()
                            x["w"][:upto] += p
                            x["off"][:upto] += p * 2 * float(dz.max()) + 1e-6 + (p + 0.5 if loose else 0)
                # who stays, by the card's own weights: those in slots below `keep` now hold what was weighed; all are known only before the moves
                L = old + new[s]
                f = came[s, h]
                m = min(L, keep)
                assert lens[s] == m and (f[m:] == -1).all() and len(set(f[:m].tolist())) == m
                got_w = w_after[s, h, :m].double()
                assert ((got_w - x["w"][f[:m]]).abs() <= x["off"][f[:m]]).all()
                pos = x["pos"]
                must = {j for j in range(L) if pos[j] < sinks or pos[j] > pos.max() - recent}
                stays = set(f[:m].tolist())
                assert must <= stays
                if L > keep:                                       # nobody who went weighs more than who stayed, as far as 64 bits can tell
                    free = [j for j in stays if j not in must]
                    went = [j for j in range(L) if j not in stays]
                    if free:
                        assert max(float(x["w"][j] - x["off"][j]) for j in went) <= min(float(x["w"][j] + x["off"][j]) for j in free)
                    late = iter(sorted(j for j in stays if j >= keep))
                    assert [j if j in stays else next(late) for j in range(keep)] == f[:keep].tolist()
                for name in ("k", "v", "w", "off"):
                    x[name] = x[name][torch.from_numpy(f[:m].astype(np.int64))]
                x["pos"] = pos[f[:m]]
                x["w"] = got_w                                     # (from here on the card's)
                x["off"] = torch.zeros(m).double()
                assert np.array_equal(pos_after[s, h, :m].numpy(), x["pos"])
            seen[s] += new[s]


def test_the_example_runs():
    from examples.attention_budget import run
    c, O = run(prompt=(300, 90), heads=8, kv_heads=2, head_dim=64, keep=64, recent=16, steps=6)
    assert torch.isfinite(O.float()).all() and c.kv_len.tolist() == [64, 64]
