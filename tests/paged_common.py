"""Ragged batches over paged keys and values for the tests of the operators of include/ppd_layers.h, and the operators in 64 bits on
the host, sequence by sequence and row by row."""
import math

import numpy as np
import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}      # half a step of the smallest numbers, or more


class Batch:
    """new[s] rows of sequence s, which has kv[s] positions with them; `spare` pages that belong to no one, `pad` rows behind the last
    sequence.  Page numbers are shuffled; layout: order of the cache's dimensions in memory."""

    def __init__(self, new, kv, heads, kv_heads, hd, dtype, page=16, seed=0, spare=3, pad=0, layout="phkd", extra_pages=0):
        g = torch.Generator().manual_seed(seed)
        self.new, self.kv, self.heads, self.kv_heads, self.hd, self.dtype, self.page = list(new), list(kv), heads, kv_heads, hd, dtype, page
        self.rows, self.n = sum(new), sum(new) + pad
        need = [-(-x // page) for x in kv]
        self.n_pages = sum(need) + spare
        perm = torch.randperm(self.n_pages, generator=g)
        self.pages = torch.full((len(kv), max(1, max(need)) + extra_pages), -1, dtype=torch.int32)
        at = 0
        for s, m in enumerate(need):
            self.pages[s, :m] = perm[at:at + m]
            at += m
        self.q_start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
        self.kv_len = torch.tensor(kv, dtype=torch.int32)
        dims = {"p": self.n_pages, "k": page, "h": kv_heads, "d": hd}
        self.layout = layout

        def cache():
            t = torch.randn([dims[c] for c in layout], generator=g).to(dtype)
            return t.permute([layout.index(c) for c in "pkhd"])

        self.k_cache, self.v_cache = cache(), cache()
        self.q, self.k, self.v = (torch.randn(self.n, h, hd, generator=g).to(dtype) for h in (heads, kv_heads, kv_heads))

    def cuda(self):
        """The same on the GPU (strides kept)."""
        def up(t):
            order = sorted(range(t.dim()), key=lambda i: -t.stride(i))
            back = [order.index(i) for i in range(t.dim())]
            return t.permute(order).contiguous().cuda().permute(back)
        b = object.__new__(Batch)
        b.__dict__ = {k: up(v) if isinstance(v, torch.Tensor) else v for k, v in self.__dict__.items()}
        return b

    def slot(self, s, p):
        """(page, slot) of a position, or None."""
        i = p // self.page
        if p < 0 or i >= self.pages.shape[1]:
            return None
        page = int(self.pages[s, i])
        return (page, p % self.page) if 0 <= page < self.n_pages else None


def attention64(b, scale=None, window=0):
    """(out, lse, sum of p |v|, the largest scale * sum |q| |k| that a row sees) in 64 bits; rows of no sequence: NaN."""
    scale = b.hd ** -0.5 if scale is None else scale
    out, size = (torch.full((b.n, b.heads, b.hd), math.nan, dtype=torch.float64) for _ in range(2))
    lse, reach = (torch.full((b.n, b.heads), math.nan, dtype=torch.float64) for _ in range(2))
    group = b.heads // b.kv_heads
    for s, m in enumerate(b.new):
        row0 = sum(b.new[:s])
        where = [(p, b.slot(s, p)) for p in range(b.kv[s])]
        where = [(p, w) for p, w in where if w is not None]
        pos = torch.tensor([p for p, _ in where], dtype=torch.int64)
        if where:
            pg, sl = torch.tensor([w[0] for _, w in where]), torch.tensor([w[1] for _, w in where])
            k, v = b.k_cache[pg, sl].double(), b.v_cache[pg, sl].double()
        for i in range(m):
            r, at = row0 + i, b.kv[s] - m + i
            see = (pos <= at) & (pos > at - window if window else pos >= 0)
            out[r], size[r], lse[r], reach[r] = 0.0, 0.0, -math.inf, 0.0
            if not bool(see.any()):
                continue
            kk, vv = k[see], v[see]
            q = b.q[r].double().view(b.kv_heads, group, b.hd)
            z = torch.einsum("hgd,jhd->hgj", q, kk) * scale
            reach[r] = (torch.einsum("hgd,jhd->hgj", q.abs(), kk.abs()) * scale).amax(-1).view(-1)
            l = torch.logsumexp(z, -1)
            p = torch.exp(z - l[..., None])
            out[r] = torch.einsum("hgj,jhd->hgd", p, vv).reshape(b.heads, b.hd)
            size[r] = torch.einsum("hgj,jhd->hgd", p, vv.abs()).reshape(b.heads, b.hd)
            lse[r] = l.view(-1)
    return out, lse, size, reach


def append64(b, q_gain=None, k_gain=None, eps=1e-5, rotary=0, theta=10000.0):
    """(q, k rows, per-element sizes of both) in 64 bits; the rows' positions and slots."""
    half = rotary // 2
    place = []
    for s, m in enumerate(b.new):
        place += [(b.kv[s] - m + i, b.slot(s, b.kv[s] - m + i)) for i in range(m)]

    def one(x, gain):
        x = x[:b.rows].double()
        if gain is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
        size = x.abs()
        if rotary:
            pos = torch.tensor([float(p) for p, _ in place], dtype=torch.float64)[:, None, None]
            a = pos * theta ** (-2.0 * torch.arange(half, dtype=torch.float64) / rotary)
            lo, hi, rest = x[..., :half], x[..., half:rotary], x[..., rotary:]
            x = torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin(), rest], -1)
            both = size[..., :half] + size[..., half:rotary]
            size = torch.cat([both, both, size[..., rotary:]], -1)
        return x, size
    return one(b.q, q_gain), one(b.k, k_gain), place
