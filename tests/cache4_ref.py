"""Plain 64-bit forms of cells of 4 bits, of the weights of cached tokens and of an eviction, on the CPU; shared by the tests of the kernels."""
import numpy as np
import torch

import attention_ref as R

VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def encode(x):
    """... x D (any float) -> (codes 0 .. 15, bytes of the powers ... x D / 32, what they stand for in float64): by the definition, value by value."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    odd = ~torch.isfinite(x).all(-1)
    power = torch.full(top.shape, -100, dtype=torch.int64)
    for p in range(-100, 125):
        power = torch.where(top > 7 * 2.0 ** p, p + 1, power)
    y = x.abs() * 2.0 ** -power.double()[..., None]
    code = torch.zeros(y.shape, dtype=torch.int64)
    for c, (lo, hi) in enumerate(zip(VALUES, VALUES[1:])):        # beyond the middle, or in it where the higher code is the even one
        mid = (lo + hi) / 2
        code = torch.where((y >= mid) if c % 2 else (y > mid), c + 1, code)
    code += 8 * torch.signbit(x)
    code, byte = torch.where(odd[..., None], 0, code), torch.where(odd, 255, power + 127)
    return code.flatten(-2).to(torch.uint8), byte.to(torch.uint8), decode(code.flatten(-2), byte)


def decode(code, byte):
    v = torch.tensor(VALUES + [-x for x in VALUES], dtype=torch.float64)[code.long()]
    scale = torch.where(byte == 255, float("nan"), 2.0 ** (byte.double() - 127))
    return v * scale.repeat_interleave(32, -1)


class Batch4(R.Batch):
    """attention_ref's batch with its keys and values in cells of 4 bits.  Cells that no token is in are NaN by their power."""

    def __init__(self, n, kv, KH, D, page, prefix=0, seed=0, page_gap=0, spare=3, amplitude=1.0, wide=False):
        super().__init__(n, kv, KH, D, page, prefix=prefix, seed=seed, spare=spare, amplitude=amplitude)
        g = torch.Generator().manual_seed(seed + 1)
        self.stride = KH * page * D + page_gap
        self.pk, self.pv = (torch.randint(0, 256, (self.n_pages, self.stride // 2), generator=g, dtype=torch.uint8) for _ in range(2))
        self.sk, self.sv = (torch.full((self.n_pages, self.stride // 32), 255, dtype=torch.uint8) for _ in range(2))
        done = {}
        for b in range(len(n)):
            k, v = self.ks[b], self.vs[b]
            if wide:                                             # tokens of very different size
                size = 2.0 ** torch.randint(-20, 20, (k.shape[0], 1, 1), generator=torch.Generator().manual_seed(7)).double()
                k, v = k, v * size
            (ck, bk, self.ks[b]), (cv, bv, self.vs[b]) = encode(k), encode(v)
            for j in range(k.shape[0]):
                p = int(self.table[b, j // page])
                if j < prefix and (p, j % page) in done:
                    continue
                done[p, j % page] = True
                self.put(p, j % page, ck[j], bk[j], cv[j], bv[j])

    def views(self, pk, pv, sk, sv):
        """Of raw pages: K n x KH x page x D / 2, V n x KH x D / 2 x page, and their powers."""
        KH, D, page = self.KH, self.D, self.page
        cut = lambda x, *shape: x[:, : shape[0] * shape[1] * shape[2]].view(-1, *shape)  # noqa: E731
        return cut(pk, KH, page, D // 2), cut(pv, KH, D // 2, page), cut(sk, KH, page, D // 32), cut(sv, KH, D // 32, page)

    def put(self, p, slot, ck, bk, cv, bv):
        k, v, sk, sv = self.views(self.pk, self.pv, self.sk, self.sv)
        k[p, :, slot], sk[p, :, slot] = ck[:, 0::2] | ck[:, 1::2] << 4, bk
        v[p, :, :, slot], sv[p, :, :, slot] = cv[:, 0::2] | cv[:, 1::2] << 4, bv

    def on_gpu(self, B, q_start=True, **kw):
        dev = lambda a: torch.as_tensor(a).cuda()  # noqa: E731
        self.dk, self.dv, self.dsk, self.dsv = (x.cuda() for x in (self.pk, self.pv, self.sk, self.sv))
        self.d = [dev(self.kv32()), dev(self.table), dev(self.q_start)]
        cache = B.KVCache4(self.dk, self.dv, self.dsk, self.dsv, self.n_pages, self.page, self.KH, self.D,
                           page_stride=0 if self.stride == self.KH * self.page * self.D else self.stride)
        return cache, B.Seqs(len(self.n), self.T, self.d[0], self.d[1], self.table.shape[1], kw.get("max_q", self.max_q), kw.get("max_kv", self.max_kv),
                             q_start=self.d[2] if q_start else None)


def batch(cells, *a, **kw):
    return Batch4(*a, **kw) if cells == "e2m1" else R.Batch(*a, e4m3=cells == "e4m3", **kw)


def weights(b, Q, H, lse, W, decay, scale):
    """patch_attention_weights of the batch b: (n_seqs x KH x stride float64, how far fp32 may be off).  lse: T x H as given, W: float32."""
    D, G = b.D, H // b.KH
    out, off, t = W.double().clone(), torch.zeros(W.shape).double(), 0
    for s in range(len(b.n)):
        L, n = max(b.kv[s], 0), b.n[s]
        old = max(L - n, 0)
        if n:
            out[s, :, :old] *= decay
            off[s, :, :old] = out[s, :, :old].abs() * 2.0 ** -23
            out[s, :, old:L] = 0
        for i in range(n):
            seen = L - n + i + 1
            if seen > 0:
                k = b.ks[s][:seen].double().transpose(0, 1)                    # KH x seen x D
                q = Q[t].double().view(b.KH, G, D)
                z, mag = q @ k.transpose(1, 2) * scale, (q.abs() @ k.abs().transpose(1, 2) * abs(scale)).amax(-1, keepdim=True)
                l = lse[t].double().view(b.KH, G, 1)
                p = torch.where(l == -np.inf, 0.0, torch.exp(z - l))
                # the products are exact, D of them are added in fp32; the argument of exp2 is two roundings and a product off, exp2 itself by 2^-23
                d = (2 * D + 16) * 2.0 ** -24 * mag + 2.0 ** -22 * (1 + z.abs() + torch.where(l == -np.inf, 0.0, l.abs()))
                out[s, :, :seen] += p.sum(1)
                off[s, :, :seen] += (p * 2 * d).sum(1)
            t += 1
        off[s, :, :L] += out[s, :, :L].abs() * (n * G + 16) * 2.0 ** -24       # the sums
    return out, off


def evicted(w, pos, length, keep, sinks, recent):
    """One key head: the slot that each of the first `keep` slots' tokens come from, -1 where there is none (w, pos: numpy)."""
    if length <= keep:
        return np.array([i if i < length else -1 for i in range(keep)])
    pos = np.arange(length) if pos is None else pos[:length].astype(np.int64)
    always = (pos < sinks) | (pos > pos.max() - recent)
    heavy = np.where(np.isnan(w[:length]), -np.inf, w[:length].astype(np.float64))
    order = sorted(range(length), key=lambda i: (0, 0.0, False, i) if always[i] else (1, -heavy[i], bool(np.isnan(w[i])), i))
    stays = set(order[:keep])
    late = iter(sorted(i for i in stays if i >= keep))
    return np.array([i if i in stays else next(late) for i in range(keep)])
