"""A small Mixtral-style decoder served end to end with this library: prompts of several users
prefilled in one ragged batch, then one token per user and step.

    python examples/decoder.py [--layers 2] [--steps 16] [--bits4]

Each layer is  h <- h + Wo attention(RMSNorm(h)),  h <- h + MoE(RMSNorm(h)):  kv_append norms and
rotates the new queries and keys and writes keys and values to the paged cache, attn_prefill reads it,
moe_forward is the compressed expert block, and residual_norm is what lies between the
blocks.  kv_plan hands out the cache's pages as users grow, and takes them back; its batch says which users have a row
in the step, so one that it refuses (no page is left, or its table is full) is not in it.  (attn_decode, which takes a token
of every user, could not leave one out; with a token or a few of each, attn_prefill runs the same kernel.)  With --bits4
the cache holds 4 bits an element.  The projections are plain torch matrix products, weights are random.
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

    def __init__(self, seed, tokens, pages, bits4=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        L = synth.make_layer(tokens, 256, 512, 8, 64, [3, 2, 2, 1, 3, 2, 2, 3], seed)
        self.shape, self.bits, self.mu = mc.Shape(L.E, L.H, L.F, L.group), L.bits, 0.2
        flat = lambda a: [a[e][m] for e in range(L.E) for m in range(3)]  # noqa: E731
        self.experts = mc.pack_experts(self.shape, L.bits, flat(L.codes), flat(L.scale), flat(L.zero))
        self.gate = torch.from_numpy(L.gate.view(np.int16).copy()).view(torch.bfloat16).cuda()
        w = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[0] ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.qkv, self.out = w(L.H, (HEADS + 2 * KV_HEADS) * DIM), w(HEADS * DIM, L.H)
        self.norms = [torch.ones(n, dtype=torch.bfloat16, device="cuda") for n in (L.H, L.H, DIM, DIM)]
        if bits4:
            pool = torch.empty(pages, 2, KV_HEADS, mc.kv4_block_size(PAGE, DIM), dtype=torch.uint8, device="cuda")
            self.cache = mc.KVCache4(pool[:, 0], pool[:, 1], PAGE, DIM)
        else:
            pool = torch.empty(pages, 2, KV_HEADS, PAGE, DIM, dtype=torch.bfloat16, device="cuda")  # keys, values of a page
            self.cache = mc.KVCache(pool[:, 0], pool[:, 1])


class Decoder:
    """Layers, the page table of every user, the free pages, and the buffers that calls reuse."""

    def __init__(self, layers, users, max_len, seed=0, max_tokens=512, bits4=False):
        width = -(-max_len // PAGE)
        pages = (users + 1) * width  # (what a user gives back is free from the next step on)
        self.layers = [Layer(seed + i, max_tokens, pages, bits4) for i in range(layers)]
        self.append = mc.kv4_append if bits4 else mc.kv_append
        self.attend = mc.attn4_prefill if bits4 else mc.attn_prefill
        self.hidden = self.layers[0].shape.H
        g = torch.Generator(device="cuda").manual_seed(seed + 1000)
        self.embed, self.head = (torch.randn(VOCAB, self.hidden, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        a = torch.arange(max_len, device="cuda", dtype=torch.float64)[:, None]
        a = a * 10000.0 ** (-torch.arange(0, DIM, 2, device="cuda", dtype=torch.float64) / DIM)
        self.rope = torch.cat([a.cos(), a.sin()], 1).float()
        # free pages, in an order of their own
        ring = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()
        self.pool = mc.KVPool(pages, PAGE, ring=ring)
        self.table = torch.full((users, width), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(users, dtype=torch.int32, device="cuda")
        self.one = torch.ones(users, dtype=torch.int32, device="cuda")
        self.attn_ws = (mc.attn4_workspace if bits4 else mc.attn_workspace)(self.layers[0].cache, HEADS)
        self.plan_ws = mc.kv_plan_workspace(users)
        self.moe_ws = mc.alloc_workspace(self.layers[0].shape, max_tokens)

    def forward(self, tokens, new=None, over=None):
        """Hidden states after the last layer of `tokens`: new[b] of user b, in order (None: one each).  Users with
        over[b] are done: their pages go back, and what is new is another user's first text.  A user that there are no
        pages for stays as it is and may come again: its hidden states are zeros, and check() says so."""
        add = self.one if new is None else torch.tensor(new, dtype=torch.int32).cuda()
        over = None if over is None else torch.tensor(over, dtype=torch.uint8).cuda()
        plan = mc.kv_plan(self.pool, self.table, self.lens, add, done=over, tokens=tokens.shape[0], lens_out=self.lens,
                          positions=False, slots=False, workspace=self.plan_ws)
        # row t of the step holds the token `own[t]`: rows close up over the tokens of users that are refused, and as many
        # behind the last user's are padding
        T, first = tokens.shape[0], add.cumsum(0) - add
        row = torch.arange(T, dtype=torch.int32, device="cuda")
        user = (torch.searchsorted(plan.cu_q, row, right=True) - 1).clamp(max=add.shape[0] - 1)
        own = (first[user] + row - plan.cu_q[user]).clamp(max=T - 1)
        h = self.embed[tokens[own]]
        x = mc.rmsnorm(h, self.layers[0].norms[0])
        for i, w in enumerate(self.layers):
            x = (x @ w.qkv).view(T, HEADS + 2 * KV_HEADS, DIM)
            q = self.append(w.cache, plan.batch, x[:, :HEADS], x[:, HEADS:HEADS + KV_HEADS], x[:, HEADS + KV_HEADS:], rope=self.rope,
                            q_norm=w.norms[2], k_norm=w.norms[3], workspace=self.attn_ws)
            o = self.attend(w.cache, plan.batch, q, out=torch.zeros_like(q), workspace=self.attn_ws)  # (padding has no attention)
            h, x = mc.residual_norm(o.view(T, -1) @ w.out, h, pre_norm=w.norms[1])
            y = mc.moe_forward(x, w.gate, w.shape, w.bits, w.experts, w.mu, workspace=self.moe_ws)
            h, x = mc.residual_norm(y, h, pre_norm=self.layers[i + 1].norms[0] if i + 1 < len(self.layers) else None)
        out = h.new_zeros(T + 1, self.hidden)
        out[torch.where(row < plan.cu_q[-1], own, T)] = h
        return out[:T]

    def logits(self, h):
        return (h @ self.head.T).float()

    def check(self):
        mc.check_status(self.plan_ws)
        mc.check_status(self.attn_ws)
        mc.check_status(self.moe_ws)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--bits4", action="store_true", help="the cache in 4 bits")
    a = ap.parse_args()
    prompts = [37, 5, 64, 1]
    d = Decoder(a.layers, len(prompts), max(prompts) + a.steps, bits4=a.bits4)
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
