"""The 4-bit cache written out from its definition, element by element, on the CPU: grids of groups, the bytes
of a block, and batches of attn_ref whose cache holds what the 4 bits stand for."""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np
import torch

import attn_ref as ref

LEAST = {"bf16": Fraction(1, 2 ** 100), "fp16": Fraction(1, 2 ** 20)}
MOST = {"bf16": Fraction(255 * 2 ** 120), "fp16": Fraction(65504)}


def grid(x, dtype):
    """(codes, scale, zero point) of a group's 64 numbers (floats that dtype holds); scale NaN if one is not finite."""
    if not all(math.isfinite(v) for v in x):
        return [0] * 64, math.nan, 0
    lo, hi = min(0.0, min(x)), max(0.0, max(x))
    with np.errstate(over="ignore", under="ignore"):
        span = Fraction(float(np.float32(hi / 16) - np.float32(lo / 16))) * 16
    need = span / 15
    s = LEAST[dtype]
    if need > s:
        e = math.floor(math.log2(need)) - 4
        while Fraction(2) ** e * 15 < need:
            e += 1
        s = Fraction(2) ** e * math.ceil(need / Fraction(2) ** e)  # 8 .. 15 steps of 2^e
        assert 15 * s >= span
    half = Fraction(1, 2)
    z = math.floor(-Fraction(lo) / s + half)
    most = math.floor(MOST[dtype] / s)
    codes = []
    for v in x:
        n = math.floor(Fraction(v) / s + half)
        codes.append(max(0, z - most, min(15, z + most, n + z)))
    return codes, float(s), z


def word(s, z):
    bits = int(np.float32(s).view(np.uint32))
    return 0x7ff0 if math.isnan(s) else (bits >> 16) | z


def value(s, z, c):
    return s * (c - z)


def store(row, dtype):
    """(bytes of codes, bytes of words, what they stand for) of a head's row (a 1-D tensor of the type)."""
    D = row.shape[0]
    G = D // 64
    codes, words, out = bytearray(D // 2), bytearray(), []
    for g in range(G):
        c, s, z = grid(row[64 * g:64 * g + 64].double().tolist(), dtype)
        for e, v in enumerate(c):
            w, j, odd = e // 8, e % 8 // 2, e % 2
            bit = 32 * (w * G + g) + 16 * odd + 4 * j
            codes[bit // 8] |= v << (bit % 8)
        words += int(word(s, z)).to_bytes(2, "little")
        out += [value(s, z, v) for v in c]
    return bytes(codes), bytes(words), torch.tensor(out, dtype=torch.float64)


class Blocks:
    """uint8 pools of keys and values for a ref.Batch, rows written from the batch's own cache, the others 0xff
    (a scale of NaN); the batch's cache becomes what they stand for."""

    def __init__(self, B):
        pages = B.k.shape[0]
        n, m = B.dim // 2, B.dim // 32
        self.B, self.code_bytes, self.word_bytes = B, n, m
        self.size = B.page * (n + m)
        self.pools = []
        for name in ("k", "v"):
            pool = np.full((pages, B.kv, self.size), 0xff, np.uint8)
            c = getattr(B, name).clone()
            for b, length in enumerate(B.lens):
                for j in range(max(0, length)):
                    page, row = int(B.table[b, j // B.page]), j % B.page
                    for h in range(B.kv):
                        self.write(pool[page, h], row, c, page, h)
            self.pools.append(torch.from_numpy(pool))
            setattr(B, name, c)

    def write(self, block, row, c, page, h):
        codes, words, stands = store(c[page, h, row], self.B.dtype)
        block[row * self.code_bytes:(row + 1) * self.code_bytes] = np.frombuffer(codes, np.uint8)
        at = self.B.page * self.code_bytes + row * self.word_bytes
        block[at:at + self.word_bytes] = np.frombuffer(words, np.uint8)
        c[page, h, row] = stands.to(c.dtype)

    def device(self, mc, cu=True, interleave=False):
        """(KVCache4, KVBatch) on the GPU."""
        B = self.B
        if interleave:  # keys and values of a page side by side, and a gap
            both = torch.cat([*self.pools, torch.zeros(B.k.shape[0], 1, self.size, dtype=torch.uint8)], 1).cuda()
            k, v = both[:, :B.kv], both[:, B.kv:2 * B.kv]
        else:
            k, v = (p.cuda() for p in self.pools)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
        cache = mc.KVCache4(k, v, B.page, B.dim, ref.DT[B.dtype])
        return cache, mc.KVBatch(i32(B.lens), B.table.cuda(), i32(B.cu) if cu else None, B.tokens if cu else None)


def fast_blocks(B):
    """Blocks with the rows of long batches quantised by vectorised 64-bit arithmetic (checked against grid() in
    the tests), finite caches only."""
    self = Blocks.__new__(Blocks)
    n, m = B.dim // 2, B.dim // 32
    self.B, self.code_bytes, self.word_bytes, self.size = B, n, m, B.page * (n + m)
    self.pools = []
    G = B.dim // 64
    for name in ("k", "v"):
        c = getattr(B, name)
        codes, s, z = grids(c.double().unflatten(-1, (G, 64)), B.dtype)
        stands = ((codes - z[..., None]) * s[..., None]).flatten(-2)
        w = codes.nan_to_num(15).to(torch.uint8).unflatten(-1, (8, 4, 2)).transpose(-1, -2).flatten(-2)
        w = (w[..., 0::2] | (w[..., 1::2] << 4)).transpose(-3, -2).flatten(-4)
        words = torch.where(s.isnan(), 0x7fff, (s.nan_to_num(1.0).float().view(torch.int32) >> 16) | z.nan_to_num(0).int()).to(torch.int16)
        self.pools.append(torch.cat([w, words.flatten(-2).contiguous().view(torch.uint8)], -1))
        setattr(B, name, stands.to(c.dtype))
    return self


def grids(x, dtype):
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    span = ((hi / 16).float() - (lo / 16).float()).double()
    m, e = np.frexp((span * 16 / 15).numpy())
    s = torch.from_numpy(np.ldexp(np.ceil(m * 16) / 16, e)).clamp(min=float(LEAST[dtype]))
    z = torch.floor(-lo / s + 0.5)
    most = torch.floor(float(MOST[dtype]) / s)
    c = torch.floor(x / s[..., None] + 0.5) + z[..., None]
    return torch.minimum(torch.maximum(c, (z - most).clamp(min=0.0)[..., None]), (z + most).clamp(max=15.0)[..., None]), s, z
