"""Plain 64-bit forms of the attention side of a layer, on the CPU, and caches laid out as the library's; shared by the tests of the kernels."""
import numpy as np
import torch

BF16_HALF, E4M3_HALF = 2.0 ** -8, 2.0 ** -4     # half a step, relative


def table_of(n_pos, rot):
    """n_pos x 2 x rot / 2, angles in 64 bits."""
    angle = np.arange(n_pos)[:, None] * 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    return torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], 1).astype(np.float32))


def rotated(x, gamma, eps, table, positions, rot, interleaved):
    """x: T x heads x D (float64) -> (normed and rotated, the sum of the magnitudes that went into each value)."""
    x = x.double().clone()
    if gamma is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gamma.double()
    if not rot:
        return x, x.abs()
    half = rot // 2
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
    c, s = (table[positions.long().clamp(0, table.shape[0] - 1), i].double()[:, None] for i in (0, 1))
    y, mag = x.clone(), x.abs()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    mag[..., a] = mag[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, mag


def attention(Q, ks, vs, G, scale, n, kv):
    """Q: T x H x D, ks / vs: per sequence kv x KH x D (what its cells stand for) -> (o, lse, sum of p |v|, largest sum |q k| scale), float64."""
    T, H, D = Q.shape
    o, lse, av, qk = torch.zeros(T, H, D).double(), torch.full((T, H), -np.inf).double(), torch.zeros(T, H, D).double(), torch.zeros(T, H).double()
    t = 0
    for s in range(len(n)):
        for i in range(n[s]):
            pos = kv[s] - n[s] + i
            if pos >= 0:
                k, v = (x[s][: pos + 1].double().repeat_interleave(G, 1) for x in (ks, vs))
                q = Q[t].double()
                z = torch.einsum("hd,jhd->hj", q, k) * scale
                lse[t] = torch.logsumexp(z, 1)
                p = torch.exp(z - lse[t][:, None])
                o[t], av[t] = torch.einsum("hj,jhd->hd", p, v), torch.einsum("hj,jhd->hd", p, v.abs())
                qk[t] = (torch.einsum("hd,jhd->hj", q.abs(), k.abs()) * abs(scale)).amax(1)
            t += 1
    return o, lse, av, qk


class Batch:
    """Sequences with random keys in a cache whose pages lie in no order.  Cells that no token is in hold NaN."""

    def __init__(self, n, kv, KH, D, page, prefix=0, e4m3=False, seed=0, scales=True, page_gap=0, spare=3, amplitude=1.0):
        g = torch.Generator().manual_seed(seed)
        self.n, self.kv, self.KH, self.D, self.page, self.prefix, self.e4m3 = n, kv, KH, D, page, prefix, e4m3
        B, kind = len(n), torch.float8_e4m3fn if e4m3 else torch.bfloat16
        self.k_scale = self.v_scale = None
        if e4m3 and scales:
            self.k_scale, self.v_scale = 0.01 + 0.02 * torch.rand(KH, generator=g), 0.01 + 0.02 * torch.rand(KH, generator=g)
        per = [-(-max(L, 0) // page) for L in kv]
        whole = prefix // page
        n_pages = whole + sum(max(p - whole, 0) for p in per) + spare
        order = torch.randperm(n_pages, generator=g).tolist()
        self.table = np.full((B, max(max(per), 1) + 1), -7, np.int32)
        at = whole
        for b in range(B):
            shared = min(whole, per[b])
            self.table[b, :shared] = order[:shared]
            self.table[b, shared:per[b]] = order[at:at + per[b] - shared]
            at += per[b] - shared
        front = [torch.randn(prefix, KH, D, generator=g) * amplitude for _ in range(2)]
        self.ks, self.vs = [], []
        cells = KH * page * D
        self.stride = cells + page_gap
        raw_k, raw_v = (torch.full((n_pages, self.stride), float("nan")) for _ in range(2))
        stored = lambda x, scale: (x / (scale[:, None] if scale is not None else 1.0)).clamp(-448, 448).to(kind) if e4m3 else x.to(kind)  # noqa: E731
        for b in range(B):
            L = max(kv[b], 0)
            k, v = (torch.cat([f[: min(prefix, L)], amplitude * torch.randn(max(L - prefix, 0), KH, D, generator=g)]) for f in front)
            k, v = stored(k, self.k_scale), stored(v, self.v_scale)
            for j in range(per[b]):
                m = min(page, L - j * page)
                p = self.table[b, j]
                raw_k[p, :cells].view(KH, page, D)[:, :m] = k[j * page:j * page + m].float().transpose(0, 1)
                raw_v[p, :cells].view(KH, D, page)[:, :, :m] = v[j * page:j * page + m].float().permute(1, 2, 0)
            self.ks.append(k.double() * (self.k_scale.double()[:, None] if self.k_scale is not None else 1.0))
            self.vs.append(v.double() * (self.v_scale.double()[:, None] if self.v_scale is not None else 1.0))
        self.k, self.v, self.n_pages = raw_k.to(kind), raw_v.to(kind), n_pages
        self.q_start = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.T, self.max_q, self.max_kv = int(sum(n)), max(n), max(max(kv), 0)

    def on_gpu(self, B, q_start=True, **kw):
        """(cache, seqs) of the binding; the device tensors are kept here."""
        dev = lambda a: None if a is None else torch.as_tensor(a).cuda()  # noqa: E731
        self.dk, self.dv = self.k.cuda(), self.v.cuda()
        self.d = [dev(x) for x in (self.kv32(), self.table, self.q_start, self.k_scale, self.v_scale)]
        kv_len, table, start, ksc, vsc = self.d
        cache = B.KVCache(self.dk, self.dv, self.n_pages, self.page, self.KH, self.D, e4m3=self.e4m3, k_scale=ksc, v_scale=vsc,
                          page_stride=0 if self.stride == self.KH * self.page * self.D else self.stride)
        seqs = B.Seqs(len(self.n), self.T, kv_len, table, self.table.shape[1], kw.get("max_q", self.max_q), kw.get("max_kv", self.max_kv),
                      q_start=start if q_start else None)
        return cache, seqs

    def kv32(self):
        return np.asarray(self.kv, np.int32)
