"""The paged cache, the append and the attention over it, written out in 64 bits from
their definitions, on the CPU, one sequence after the other; and the batches that the
tests make of them."""
from __future__ import annotations

import math

import torch

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
# unit roundoff, half an ulp at the low end of a binade: 8 and 11 significant bits
HALF_ULP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


class Batch:
    """Sequences of lengths `lens` with `new` new tokens each, their pages in random order
    in a pool whose unwritten rows are NaN; all on the CPU."""

    def __init__(self, lens, new, kv_heads, page, dim, dtype, seed, spare=3, pad_tokens=0, interleave=False, vscale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.g, self.lens, self.new, self.kv, self.page, self.dim, self.dtype = g, lens, new, kv_heads, page, dim, dtype
        need = [-(-max(0, n) // page) for n in lens]
        pages = sum(need) + spare
        order = torch.randperm(pages, generator=g).to(torch.int32)
        width = max(1, max(need, default=1))
        self.table = torch.full((len(lens), width), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        pool = torch.full((pages, 2, kv_heads, page, dim), float("nan"), dtype=DT[dtype])
        self.pool = pool
        if interleave:  # keys and values of a page side by side
            self.k, self.v = pool[:, 0], pool[:, 1]
        else:
            self.k, self.v = pool[:, 0].contiguous(), pool[:, 1].contiguous()
        for b, n in enumerate(lens):
            j = torch.arange(max(0, n))
            rows = self.table[b, j // page].long(), j % page
            for c, sc in ((self.k, 1.0), (self.v, vscale)):
                c[rows[0], :, rows[1]] = (sc * torch.randn(len(j), kv_heads, dim, generator=g)).to(DT[dtype])
        self.cu = [0]
        for n in new:
            self.cu.append(self.cu[-1] + n)
        self.tokens = self.cu[-1] + pad_tokens

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.g).to(DT[self.dtype])

    def rows(self, c, b, h, first, end):
        j = torch.arange(first, end)
        return c[self.table[b, j // self.page].long(), h, j % self.page].double()

    def device(self, mc, cu=True, interleave=False):
        """(KVCache, KVBatch) on the GPU."""
        if interleave:
            pool = self.pool.cuda()
            cache = mc.KVCache(pool[:, 0], pool[:, 1])
        else:
            cache = mc.KVCache(self.k.cuda(), self.v.cuda())
        i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
        batch = mc.KVBatch(i32(self.lens), self.table.cuda(), i32(self.cu) if cu else None, self.tokens if cu else None)
        return cache, batch


def attention(B, q, scale, softcap=0.0, window=0, slopes=None, prefix=None):
    """(out, lse, mean |v| under the probabilities) in 64 bits; rows without keys: 0, -inf, 0."""
    Hq, G = q.shape[1], q.shape[1] // B.kv
    out = torch.zeros(q.shape, dtype=torch.float64)
    mass = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    for b, (n, length) in enumerate(zip(B.new, B.lens)):
        for i in range(n):
            p = length - n + i
            if p < 0:
                continue
            end = min(length, max(p + 1, prefix[b] if prefix else 0))
            first = max(0, p - window + 1) if window else 0
            if first >= end:
                continue
            t = B.cu[b] + i
            for h in range(B.kv):
                k, v = B.rows(B.k, b, h, first, end), B.rows(B.v, b, h, first, end)
                x = q[t, h * G:(h + 1) * G].double() @ k.T * scale
                if softcap:
                    x = softcap * torch.tanh(x / softcap)
                if slopes is not None:
                    x = x + slopes[h * G:(h + 1) * G, None].double() * (torch.arange(first, end) - p)
                w = torch.softmax(x, -1)
                lse[t, h * G:(h + 1) * G] = torch.logsumexp(x, -1)
                out[t, h * G:(h + 1) * G] = w @ v
                mass[t, h * G:(h + 1) * G] = w @ v.abs()
    return out, lse, mass


def assert_attention(got, got_lse, want, dtype, max_len, vmax, rows=None):
    """Bounds, from the roundings that the call documents: each probability is rounded
    once (half an ulp of it, so half an ulp of the mean |v|; in fp16 also at most 2^-25 for
    each key below the type's normal range), the output once (half an ulp of itself, which
    is at most the mean |v|).  fp32 scores, sums and exponentials: 1e-4 of the mean |v|
    covers 128-term dot products of a few units (128 * 2^-24 * 64 < 5e-4 of a score in
    the worst case, a fortieth of it in the mean) and lse to 1e-4."""
    out, lse, mass = want
    rows = slice(None) if rows is None else rows
    h = HALF_ULP[dtype]
    tol = (2 * h + 1e-4) * mass + 1e-30
    if dtype == "fp16":
        tol = tol + 2.0 ** -24 + max_len * 2.0 ** -25 * vmax
    err = (got.double().cpu() - out).abs()
    assert torch.isfinite(got[rows]).all()
    assert (err[rows] <= tol[rows]).all(), float((err / tol)[rows].max())
    if got_lse is not None:
        g = got_lse.double().cpu()[rows]
        empty = torch.isinf(lse[rows])
        assert torch.equal(torch.isinf(g), empty) and (g[empty] < 0).all()
        assert ((g - lse[rows])[~empty].abs() <= 1e-4 * (1 + lse[rows][~empty].abs())).all()


def append(B, q, k, v, rope=None, interleaved=False, q_norm=None, k_norm=None, eps=1e-6):
    """(queries, key cache, value cache) after the append, in 64 bits."""
    kc, vc = B.k.double().clone(), B.v.double().clone()
    q_out = torch.zeros(q.shape, dtype=torch.float64)

    def side(x, gain, pos):
        x = x.double()
        if gain is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
        if rope is not None:
            half = rope.shape[1] // 2
            y = x.clone()
            for i in range(half):
                c, s = rope[pos, i].double(), rope[pos, half + i].double()
                a, b = (2 * i, 2 * i + 1) if interleaved else (i, half + i)
                y[:, a], y[:, b] = x[:, a] * c - x[:, b] * s, x[:, b] * c + x[:, a] * s
            x = y
        return x

    for b, (n, length) in enumerate(zip(B.new, B.lens)):
        for i in range(n):
            pos, t = length - n + i, B.cu[b] + i
            if pos < 0:
                continue
            q_out[t] = side(q[t], q_norm, pos)
            page, row = int(B.table[b, pos // B.page]), pos % B.page
            kc[page, :, row] = side(k[t], k_norm, pos)
            vc[page, :, row] = v[t].double()
    return q_out, kc, vc


def rope_table(rows, rot, base=10000.0):
    a = torch.arange(rows, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([a.cos(), a.sin()], 1).float()
