"""A small Mixtral-style decoder served end to end with this library: prompts of several users
prefilled in one ragged batch, then one token per user and step.

    python examples/decoder.py [--layers 2] [--steps 16]

Each layer is  h <- h + Wo attention(RMSNorm(h)),  h <- h + MoE(RMSNorm(h)):  kv_append norms and
rotates the new queries and keys and writes keys and values to the paged cache, attn_prefill or
attn_decode reads it, moe_forward is the compressed expert block.  The projections are plain
torch matrix products, weights are random.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_06270_gb300 as mc  # noqa: E402
import synth  # noqa: E402

HEADS, KV_HEADS, DIM, PAGE, VOCAB = 8, 2, 64, 16, 512


class Layer:
    """Weights of one layer, and its slice of the cache."""

    def __init__(self, seed, tokens, pages):
        g = torch.Generator(device="cuda").manual_seed(seed)
        L = synth.make_layer(tokens, 256, 512, 8, 64, [3, 2, 2, 1, 3, 2, 2, 3], seed)
        self.shape, self.bits, self.mu = mc.Shape(L.E, L.H, L.F, L.group), L.bits, 0.2
        flat = lambda a: [a[e][m] for e in range(L.E) for m in range(3)]  # noqa: E731
        self.experts = mc.pack_experts(self.shape, L.bits, flat(L.codes), flat(L.scale), flat(L.zero))
        self.gate = torch.from_numpy(L.gate.view(np.int16).copy()).view(torch.bfloat16).cuda()
        w = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[0] ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.qkv, self.out = w(L.H, (HEADS + 2 * KV_HEADS) * DIM), w(HEADS * DIM, L.H)
        self.norms = [torch.ones(n, dtype=torch.bfloat16, device="cuda") for n in (L.H, L.H, DIM, DIM)]
        pool = torch.empty(pages, 2, KV_HEADS, PAGE, DIM, dtype=torch.bfloat16, device="cuda")  # keys, values of a page
        self.cache = mc.KVCache(pool[:, 0], pool[:, 1])


class Decoder:
    """Layers, the page table of every user, and the buffers that calls reuse."""

    def __init__(self, layers, users, max_len, seed=0, max_tokens=512):
        width = -(-max_len // PAGE)
        self.layers = [Layer(seed + i, max_tokens, users * width) for i in range(layers)]
        self.hidden = self.layers[0].shape.H
        g = torch.Generator(device="cuda").manual_seed(seed + 1000)
        self.embed, self.head = (torch.randn(VOCAB, self.hidden, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        a = torch.arange(max_len, device="cuda", dtype=torch.float64)[:, None]
        a = a * 10000.0 ** (-torch.arange(0, DIM, 2, device="cuda", dtype=torch.float64) / DIM)
        self.rope = torch.cat([a.cos(), a.sin()], 1).float()
        # a user's pages, in an order of their own (a server would hand them out as sequences grow)
        self.table = torch.randperm(users * width, generator=torch.Generator().manual_seed(seed)).view(users, width).to(torch.int32).cuda()
        self.lens = torch.zeros(users, dtype=torch.int32, device="cuda")
        self.attn_ws = mc.attn_workspace(self.layers[0].cache, HEADS)
        self.moe_ws = mc.alloc_workspace(self.layers[0].shape, max_tokens)

    def forward(self, tokens, new=None):
        """Hidden states after the last layer of `tokens`: new[b] of user b, in order (None: one each)."""
        if new is None:
            self.lens += 1
            batch = mc.KVBatch(self.lens, self.table)
        else:
            new = torch.tensor(new, dtype=torch.int32)
            self.lens += new.cuda()
            cu = torch.cat([torch.zeros(1, dtype=torch.int32), new.cumsum(0, dtype=torch.int32)]).cuda()
            batch = mc.KVBatch(self.lens, self.table, cu, tokens.shape[0])
        h, T = self.embed[tokens], tokens.shape[0]
        for w in self.layers:
            x = (mc.rmsnorm(h, w.norms[0]) @ w.qkv).view(T, HEADS + 2 * KV_HEADS, DIM)
            q = mc.kv_append(w.cache, batch, x[:, :HEADS], x[:, HEADS:HEADS + KV_HEADS], x[:, HEADS + KV_HEADS:], rope=self.rope,
                             q_norm=w.norms[2], k_norm=w.norms[3], workspace=self.attn_ws)
            attend = mc.attn_decode if new is None else mc.attn_prefill
            o = attend(w.cache, batch, q, workspace=self.attn_ws)
            h = mc.add(h, o.view(T, -1) @ w.out)
            y = mc.moe_forward(mc.rmsnorm(h, w.norms[1]), w.gate, w.shape, w.bits, w.experts, w.mu, workspace=self.moe_ws)
            h = mc.add(h, y)
        return h

    def logits(self, h):
        return (h @ self.head.T).float()

    def check(self):
        mc.check_status(self.attn_ws)
        mc.check_status(self.moe_ws)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    prompts = [37, 5, 64, 1]
    d = Decoder(a.layers, len(prompts), max(prompts) + a.steps)
    tokens = torch.randint(VOCAB, (sum(prompts),), generator=torch.Generator().manual_seed(1)).cuda()
    h = d.forward(tokens, prompts)
    last = torch.tensor(prompts).cumsum(0).cuda() - 1
    nxt, made = d.logits(h[last]).argmax(-1), []
    for _ in range(a.steps):
        made.append(nxt)
        nxt = d.logits(d.forward(nxt)).argmax(-1)
    d.check()
    for user, row in enumerate(torch.stack(made, 1).tolist()):
        print("user %d, prompt of %d:" % (user, prompts[user]), row)


if __name__ == "__main__":
    main()
