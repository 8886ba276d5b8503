"""One decoder layer's serving step around a key-value cache held in 4 bits: five operators.

  plan     ``kv_plan``: a step's block tables on the GPU, from the lengths of the requests: pages
           of finished ones go back to the pool, growing ones get theirs, and every new
           token gets its position and its slot in the cache
  append   ``kv4_append`` (and ``kv4_read``, which gives what was stored): per-head norms of
           queries and keys, the position rotation, and the keys and values of new tokens
           into the cache's pages, in 4 bits
  decode   ``attn4_decode``: attention of one new token per sequence over that cache
  prefill  ``attn4_prefill``: attention of many new tokens per sequence over it
  norm     ``residual_norm``: what lies between one block of the layer and the next: the
           block's norm, its gate and scale, the residual sum, the next block's norm

The cache holds a head's row in groups of 64 elements: codes c of 4 bits, a zero point z of
4 bits and a scale s of 4 significant bits, standing for s (c - z).  With x the elements
rounded to the cache's type, lo = min(x, 0), hi = max(x, 0):

  s = the smallest number of 4 significant bits with 15 s >= hi - lo (but at least 2^-100 in
      bf16, 2^-20 in fp16)
  z = floor(-lo / s + 1/2),  c = floor(x / s + 1/2) + z, at most 15

(and no code that stands for more than the type's largest number; a group with an infinite or NaN
element is NaN).  s (c - z) has at most 8 significant bits, so it is a number of the cache's type.
Of a page and head the codes of all rows come first, then a 16-bit word for each group: the scale's
float32 bits 30 .. 20 and z.  A 32-bit word of codes holds 8 elements, element 2i at bits 4i, 2i + 1
at 16 + 4i; a row's words alternate between its groups.

A case names its sizes; how the lengths of a ragged batch are spread follows from the
case alone, their order in the batch and every value from the seed.  Heads, head sizes and the
decode batch are the Mixtral block's (32 query heads on 8 key-value heads of 128, hidden
size 4096) or generic ones.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
SMALLEST = {"bf16": 2.0 ** -100, "fp16": 2.0 ** -20}
GOLDEN = 0.6180339887498949


def _case(op, seqs, new, ctx, heads=32, kv=8, dim=128, dtype="bf16", page=64, ragged=False, empty=False, softcap=0.0,
          window=0, bias=False, prefix=False, norm=False, rot=0, interleaved=False):
    return {"op": op, "seqs": seqs, "new": new, "ctx": ctx, "heads": heads, "kv": kv, "dim": dim, "dtype": dtype,
            "page": page, "ragged": ragged, "empty": empty, "softcap": softcap, "window": window, "bias": bias,
            "prefix": prefix, "norm": norm, "rot": rot, "interleaved": interleaved}


def _plan_case(seqs, ctx, prompts, prompt, page=16, short=False):
    """`prompts` of the sequences start with up to `prompt` tokens, the others take one each."""
    return {"op": "plan", "seqs": seqs, "ctx": ctx, "prompts": prompts, "prompt": prompt, "page": page, "short": short}


def _norm_case(tokens, hidden, dtype="bf16", post=True, pre=True, gate="channel", wide=0):
    """wide: columns by which the block's output is wider than what the call takes of it."""
    return {"op": "norm", "tokens": tokens, "hidden": hidden, "dtype": dtype, "post": post, "pre": pre, "gate": gate, "wide": wide}


def listed():
    return [
        # a decode step of a full server: one token each, some requests over: the smallest call, latency counts
        {"name": "plan_decode250", **_plan_case(250, 3000, 0, 1)},
        # prompts of new requests in chunks beside the running ones
        {"name": "plan_mixed1000", **_plan_case(1000, 6000, 40, 4096)},
        # a few prompts, normed heads of 64, half of each head rotated in interleaved pairs
        {"name": "append4_ragged7", **_case("append", 7, 301, 500, heads=20, kv=4, dim=64, dtype="fp16", page=48, ragged=True,
                                            norm=True, rot=32, interleaved=True)},
        # a long prompt of one user, norms and full rotation: bandwidth counts
        {"name": "append4_prompt8192", **_case("append", 1, 8192, 8192, norm=True, rot=128)},
        # one user, a short conversation: latency
        {"name": "decode4_1_777", **_case("decode", 1, 1, 777)},
        # many users with long contexts, what the small cache is for
        {"name": "decode4_64_8192", **_case("decode", 64, 1, 8192, page=128)},
        # capped scores, a window and the distance bias, ten query heads of 64 on a key head, idle slots
        {"name": "decode4_33_window", **_case("decode", 33, 1, 6001, heads=40, kv=4, dim=64, dtype="fp16", page=32,
                                              ragged=True, empty=True, softcap=50.0, window=1024, bias=True)},
        # the verification of five drafted tokens of sixteen users
        {"name": "prefill4_16_verify5", **_case("prefill", 16, 5, 2047, page=16, ragged=True)},
        # a chunk of a long prompt on what is already in the cache
        {"name": "prefill4_1_chunk509", **_case("prefill", 1, 509, 30000, page=128)},
        # a long prompt in one piece
        {"name": "prefill4_1_8192", **_case("prefill", 1, 8192, 8192)},
        # the benchmark's decode batch between attention and experts
        {"name": "norm_decode16", **_norm_case(16, 4096)},
        # a long prompt, gated element by element: bandwidth counts
        {"name": "norm_prompt8192", **_norm_case(8192, 4096, gate="element")},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "append", "decode", "decode", "prefill", "norm"])
    if op == "plan":
        seqs = _log_int(rng, 1, 4096)
        prompts = rng.choice([0, 0, _log_int(rng, 1, seqs)])
        return _plan_case(seqs, _log_int(rng, 1, 16384), prompts, _log_int(rng, 1, max(1, 200_000 // max(1, prompts))),
                          page=rng.choice([16, 32, 48, 64, 128, 256]), short=rng.random() < 0.2)
    if op == "norm":
        hidden = rng.choice([_log_int(rng, 16, 8192), 8 * _log_int(rng, 8, 1024), 256 * _log_int(rng, 1, 32)])
        return _norm_case(_log_int(rng, 1, min(16384, 33_000_000 // hidden)), hidden, rng.choice(["bf16", "bf16", "fp16"]),
                          rng.random() < 0.7, rng.random() < 0.8, rng.choice(["none", "channel", "token", "element"]),
                          rng.choice([0, 0, 0, 64, 5]))
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([g for g in (1, 2, 3, 4, 6, 8, 12, 16) if g * kv <= 48])
    kind = {"heads": heads, "kv": kv, "dim": rng.choice([64, 128, 128]), "dtype": rng.choice(["bf16", "bf16", "fp16"]),
            "page": rng.choice([16, 32, 48, 64, 128, 256]), "ragged": rng.random() < 0.7}
    if op == "append":
        seqs = _log_int(rng, 1, 64)
        new = rng.choice([1, _log_int(rng, 1, max(1, 8192 // seqs))])
        kind.update(norm=rng.random() < 0.5, rot=rng.choice([0, 16, kind["dim"] // 2, kind["dim"], kind["dim"]]),
                    interleaved=rng.random() < 0.4)
        return _case(op, seqs, new, new + _log_int(rng, 1, 300), **kind)
    kind.update(softcap=rng.choice([0.0, 0.0, 0.0, 30.0, 50.0]), bias=rng.random() < 0.25)
    if op == "decode":
        seqs = _log_int(rng, 1, 64)
        ctx = _log_int(rng, 1, 500_000 // seqs if seqs > 4 else 131071)
        kind.update(window=rng.choice([0, 0, 0, _log_int(rng, 1, 4096)]), empty=rng.random() < 0.3)
        return _case(op, seqs, 1, ctx, **kind)
    seqs = _log_int(rng, 1, 16)
    new = _log_int(rng, 1, 4096 // seqs)
    room = 1_000_000_000 // (heads * new * seqs)
    ctx = new + _log_int(rng, 1, max(1, min(32768, room) - new))
    kind.update(window=rng.choice([0, 0, 0, _log_int(rng, 1, 4096)]), prefix=rng.random() < 0.3)
    return _case(op, seqs, new, ctx, **kind)


def _spread(b, k=0):
    """A number in [0, 1) of sequence b, another one for each k."""
    return math.modf((b + 1) * GOLDEN * (1 + 0.37 * k) + 0.3 * k)[0]


def _lengths(case):
    """[(new tokens, length in the cache with them)] of the batch, spread by the case alone."""
    out = []
    for b in range(case["seqs"]):
        f = 1.0 if not case["ragged"] or b == 0 else _spread(b)
        g = 1.0 if not case["ragged"] or b == 0 else _spread(b, 1)
        n = 1 + int((case["new"] - 1) * g)
        length = max(n, 1 + int((case["ctx"] - 1) * f))
        if case["empty"] and b % 8 == 5:
            length = 0  # an idle slot of the batch
        out.append((n, length))
    return out


def _requests(case):
    """[(length, new tokens, over)] of a plan's sequences."""
    out = []
    for b in range(case["seqs"]):
        if b < case["prompts"]:
            new = 1 + int((case["prompt"] - 1) * (1.0 if b == 0 else _spread(b, 1)))
            # half of the prompts are at their first chunk
            out.append((0 if b % 2 else int(case["ctx"] * _spread(b) / 2), new, False))
        else:
            over = b % 11 == 7  # finished: its pages go back, nothing comes
            out.append((1 + int((case["ctx"] - 1) * _spread(b)), 0 if over else 1, over))
    return out


def _pages(tokens, page):
    return -(-tokens // page)


def _need(case):
    """Pages that the running sequences hold, that the new tokens ask for, and that finished ones give back."""
    page, held, asked, back = case["page"], 0, 0, 0
    for length, new, over in _requests(case):
        held += _pages(length, page)
        back += _pages(length, page) if over else 0
        asked += 0 if over else _pages(length + new, page) - _pages(length, page)
    return held, asked, back


def _visible(case, n, length, i):
    """(first, end) of the keys that the i-th of n new tokens sees."""
    p = length - n + i
    end = p + 1
    if case["prefix"]:
        end = max(end, _prefix(n, length))
    first = max(0, p - case["window"] + 1) if case["window"] else 0
    return first, max(first, min(end, length))


def _prefix(n, length):
    return length - n + (n + 1) // 2


def _slopes(heads):
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


# ------------------------------------------------------------- the 4-bit form --

def _power(e):
    """2^e in 64 bits, exactly."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _quantised(x, dtype):
    """(codes, scales, zero points) of x [..., groups, 64], which holds numbers of the cache's type, in 64 bits."""
    x = x.double()
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    span = (hi / 16).float().sub((lo / 16).float()).double()  # the difference rounded to 32 bits
    m, e = torch.frexp(span * 16 / 15)
    s = (torch.ceil(m * 16) / 16 * _power(e)).clamp(min=SMALLEST[dtype])
    z = torch.floor(-lo / s + 0.5)
    most = torch.floor(torch.finfo(DTYPES[dtype]).max / s)
    c = torch.floor(x / s[..., None] + 0.5) + z[..., None]
    c = torch.minimum(torch.maximum(c, (z - most).clamp(min=0.0)[..., None]), (z + most).clamp(max=15.0)[..., None])
    return c, s, z


def _scale_bits(s, z):
    return (s.float().view(torch.int32) >> 16) | z.int()  # (the low 20 bits of s are 0)


def _packed(c, s, z):
    """A page and head's block of bytes [..., page * 17 * dim / 32] of codes [..., page, groups, 64]."""
    w = c.to(torch.uint8).unflatten(-1, (8, 4, 2)).transpose(-1, -2).flatten(-2)  # nibbles of a word in order
    w = w[..., 0::2] | (w[..., 1::2] << 4)                                        # [..., page, groups, 8 words, 4 bytes]
    return torch.cat([w.transpose(-3, -2).flatten(-4), _scale_bits(s, z).to(torch.int16).flatten(-2).contiguous().view(torch.uint8)], -1)


def _block_rows(blocks, page, dim):
    """(codes [..., page, groups, 64], scales, zero points) of packed blocks."""
    G, n = dim // 64, page * dim // 2
    w = blocks[..., :n].unflatten(-1, (page, 8, G, 4)).transpose(-3, -2)
    nib = torch.stack([w & 15, w >> 4], -1).flatten(-2)             # [..., page, groups, 8 words, 8 nibbles]
    c = nib.unflatten(-1, (2, 4)).transpose(-1, -2).flatten(-3)
    words = blocks[..., n:].contiguous().view(torch.int16).unflatten(-1, (page, G)).int() & 0xffff
    return c, ((words & 0xfff0) << 16).view(torch.float32), words & 15


def _stands_for(c, s, z):
    return ((c.float() - z[..., None].float()) * s[..., None]).flatten(-2)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=torch.float32)  # noqa: E731
    if case["op"] == "plan":
        return _prepare_plan(case, g)
    if case["op"] == "norm":
        return _prepare_norm(case, randn)
    dtype, D, Hq, Hk, ps = DTYPES[case["dtype"]], case["dim"], case["heads"], case["kv"], case["page"]
    B = case["seqs"]
    pairs = _lengths(case)
    order = torch.randperm(B, generator=g, device=DEV).tolist()
    pairs = [pairs[b] for b in order]
    new, lens = [n for n, _ in pairs], [length for _, length in pairs]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    T = cu[-1]
    need = [-(-length // ps) for length in lens]
    width = max(1, max(need))
    pages = sum(need) + 2
    free = torch.randperm(pages, generator=g, device=DEV)
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b in range(B):
        table[b, :need[b]] = free[at:at + need[b]].to(torch.int32)
        at += need[b]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    block = ps * 17 * D // 32
    kc, vc = (torch.empty(pages, Hk, block, dtype=torch.uint8, device=DEV) for _ in range(2))
    s = {"case": case, "T": T, "max_new": max(new), "max_len": max(lens), "kc": kc, "vc": vc, "lens": i32(lens),
         "table": table, "cu": None if case["op"] == "decode" or case["new"] == 1 and case["op"] == "append" else i32(cu),
         "slopes": torch.tensor(_slopes(Hq), dtype=torch.float32, device=DEV) if case["bias"] else None,
         "prefix": i32([_prefix(n, length) for n, length in pairs]) if case["prefix"] else None}
    if case["op"] == "append":
        for c in (kc, vc):
            c.random_(0, 256, generator=g)
        s["qkv"] = randn(T, (Hq + 2 * Hk) * D).to(dtype)  # the projection's output: queries, keys, values of a token
        s["q_norm"], s["k_norm"] = ((1 + 0.1 * randn(D)).to(dtype) for _ in range(2)) if case["norm"] else (None, None)
        rot = case["rot"]
        if rot:
            f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
            a = torch.arange(case["ctx"], dtype=torch.float64, device=DEV)[:, None] * f
            s["rope"] = torch.cat([a.cos(), a.sin()], 1).float()  # [positions, cosines | sines]
        else:
            s["rope"] = None
    else:
        s["q"] = (1.5 * randn(T, Hq, D)).to(dtype)
        step = max(1, (1 << 26) // (Hk * ps * D))
        for c in (kc, vc):
            for p in range(0, pages, step):
                x = randn(min(step, pages - p), Hk, ps, D // 64, 64).to(dtype)
                c[p:p + step] = _packed(*_quantised(x, case["dtype"]))
        # rows of a page that no token was written to yet hold whatever memory held, scales of NaN among it
        for b in range(B):
            if lens[b] % ps:
                page, row = int(free[sum(need[:b]) + need[b] - 1]), lens[b] % ps
                for c in (kc, vc):
                    c[page, :, row * D // 2:ps * D // 2] = 0xff
                    c[page, :, ps * D // 2 + row * D // 32:] = 0xff
    if own:
        import paper_2410_06270_gb300 as mc
        s["cache"], s["batch"] = mc.KVCache4(kc, vc, ps, D, dtype), mc.KVBatch(s["lens"], table, s["cu"], tokens=T)
        s["ws"] = mc.attn4_workspace(s["cache"], Hq)
    return s


def _prepare_plan(case, g):
    page, held = case["page"], 0
    reqs = _requests(case)
    order = torch.randperm(case["seqs"], generator=g, device=DEV).tolist()
    reqs = [reqs[b] for b in order]
    held, asked, _ = _need(case)
    # enough pages, or too few for the last of the sequences
    spare = asked * 3 // 4 if case["short"] else asked + 64
    pages = max(1, held + spare)
    width = max(_pages(length + new, page) for length, new, _ in reqs)
    free = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    own_pages = [_pages(length, page) for length, _, _ in reqs]
    counts = torch.tensor(own_pages, device=DEV)
    starts = torch.cumsum(counts, 0) - counts
    j = torch.arange(width, device=DEV)
    table = torch.where(j < counts[:, None], free[(starts[:, None] + j).clamp(max=pages - 1)], -1).to(torch.int32).contiguous()
    # the ring of pages: those not held lie between the two counts
    taken = int(torch.randint(0, 1 << 34, (1,), generator=g, device=DEV))
    returned = taken + pages - held
    ring = torch.full((pages,), -1, dtype=torch.int32, device=DEV)
    ring[(taken + torch.arange(pages - held, device=DEV)) % pages] = free[held:]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    tokens = sum(new for _, new, _ in reqs)
    s = {"case": case, "T": (tokens + 63) // 64 * 64, "lens": i32([r[0] for r in reqs]), "add": i32([r[1] for r in reqs]),
         "over": torch.tensor([r[2] for r in reqs], dtype=torch.uint8, device=DEV), "table": table, "ring": ring,
         "state": torch.tensor([taken, returned], dtype=torch.int64, device=DEV)}
    if own:
        import paper_2410_06270_gb300 as mc
        s["pool"] = mc.KVPool(pages, page, ring=ring, state=s["state"])
        s["ws"] = mc.kv_plan_workspace(case["seqs"])
    return s


def _prepare_norm(case, randn):
    T, H, dtype = case["tokens"], case["hidden"], DTYPES[case["dtype"]]
    shape = {"channel": (1, H), "token": (T, 1), "element": (T, H)}.get(case["gate"])
    return {"case": case, "y": (1.5 * randn(T, H + case["wide"])).to(dtype)[:, :H], "h": (2.0 * randn(T, H)).to(dtype),
            "gate": torch.sigmoid(randn(*shape)).to(dtype) if shape else None,
            "post": (1 + 0.1 * randn(H)).to(dtype) if case["post"] else None,
            "pre": (1 + 0.1 * randn(H)).to(dtype) if case["pre"] else None}


SCALE, RESIDUAL_SCALE = 0.22, 0.9


def run(state):
    s, case = state, state["case"]
    if own:
        import paper_2410_06270_gb300 as mc
        if case["op"] == "plan":
            p = mc.kv_plan(s["pool"], s["table"], s["lens"], s["add"], done=s["over"], tokens=s["T"], commit=False, workspace=s["ws"])
            return {"lens": p.lens, "cu_q": p.cu_q, "positions": p.positions, "slots": p.slots, "table": s["table"],
                    "ring": s["ring"], "state": p.state}
        if case["op"] == "norm":
            h, x = mc.residual_norm(s["y"], s["h"], pre_norm=s["pre"], post_norm=s["post"], gate=s["gate"], scale=SCALE,
                                    residual_scale=RESIDUAL_SCALE, eps=EPS)
            return {"h": h, "x": x} if case["pre"] else {"h": h}
        D, Hq, Hk = case["dim"], case["heads"], case["kv"]
        if case["op"] == "append":
            x = s["qkv"].view(s["T"], Hq + 2 * Hk, D)
            q = mc.kv4_append(s["cache"], s["batch"], x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:], rope=s["rope"],
                              interleaved=case["interleaved"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS,
                              workspace=s["ws"])
            k, v = mc.kv4_read(s["cache"], s["batch"], workspace=s["ws"])
            return {"q": q, "k": k, "v": v}
        if case["op"] == "decode":
            out, lse = mc.attn4_decode(s["cache"], s["batch"], s["q"], softcap=case["softcap"], window=case["window"],
                                       slopes=s["slopes"], with_lse=True, workspace=s["ws"])
        else:
            out, lse = mc.attn4_prefill(s["cache"], s["batch"], s["q"], softcap=case["softcap"], window=case["window"],
                                        slopes=s["slopes"], prefix=s["prefix"], with_lse=True, workspace=s["ws"])
        return {"out": out, "lse": lse}
    plain = {"plan": _plain_plan, "norm": _plain_norm, "append": _plain_append}.get(case["op"], _plain_attention)
    return plain(s, case)


# ------------------------------------------------------------------ plain forms --

def _plain_plan(s, case):
    page, T, ring, table = case["page"], s["T"], s["ring"], s["table"]
    cap, width = ring.shape[0], table.shape[1]
    taken, returned = s["state"][0], s["state"][1]
    old, add, over = s["lens"].long().clamp(min=0), s["add"].long(), s["over"] != 0
    # finished sequences' pages, in order, behind those that were returned before
    back = torch.where(over, ((old + page - 1) // page).clamp(max=width), 0)
    first = torch.cumsum(back, 0) - back
    j = torch.arange(width, device=DEV)
    gives = j < back[:, None]
    ring[((returned + first[:, None] + j) % cap)[gives]] = table[gives]
    length = torch.where(over, 0, old)
    held = (length + page - 1) // page
    fits = (add >= 0) & (length + add <= width * page)
    need = torch.where(fits, (length + add + page - 1) // page - held, 0)
    upto = torch.cumsum(need, 0)
    rows = torch.cumsum(torch.where(fits, add, 0), 0)
    served = fits & ((need == 0) | (upto <= returned - taken)) & ((add == 0) | (rows <= T))
    n = torch.where(served, add, 0)
    cu = torch.cat([torch.zeros_like(n[:1]), torch.cumsum(n, 0)])
    t = torch.arange(T, device=DEV)
    real = t < cu[-1]
    b = (torch.searchsorted(cu, t, right=True) - 1).clamp(max=n.shape[0] - 1)
    pos = length[b] + t - cu[b]
    i = pos // page
    fresh = i >= held[b]
    got = ring[(taken + (upto - need)[b] + i - held[b]) % cap]
    p = torch.where(fresh, got, table[b, i.clamp(max=width - 1)])
    table[b[real & fresh], i[real & fresh]] = got[real & fresh]
    took = torch.where(served & (need > 0), upto, 0).amax()
    return {"lens": (length + n).int(), "cu_q": cu.int(), "positions": torch.where(real, pos, -1).int(),
            "slots": torch.where(real, p.long() * page + pos % page, -1), "table": table, "ring": ring,
            "state": torch.stack([taken + took, returned + back.sum()])}


def _plain_norm(s, case):
    u = s["y"].float()
    if case["post"]:
        u = u * torch.rsqrt((u * u).mean(-1, keepdim=True) + EPS) * s["post"].float()
    if s["gate"] is not None:
        u = u * s["gate"].float()
    h = (RESIDUAL_SCALE * s["h"].float() + SCALE * u).to(s["h"].dtype)
    if not case["pre"]:
        return {"h": h}
    x = h.float()  # what the next block's norm reads is the residual as it is stored
    return {"h": h, "x": (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["pre"].float()).to(h.dtype)}


def _places(s):
    """Sequence, index among its new tokens, and position of every token of the batch."""
    lens = s["lens"].long()
    if s["cu"] is None:
        b = torch.arange(s["T"], device=DEV)
        return b, torch.zeros_like(b), lens - 1, torch.ones_like(lens)
    cu = s["cu"].long()
    t = torch.arange(s["T"], device=DEV)
    b = torch.searchsorted(cu, t, right=True) - 1
    n = cu[1:] - cu[:-1]
    i = t - cu[b]
    return b, i, lens[b] - n[b] + i, n


def _plain_append(s, case):
    D, Hq, Hk, rot, ps = case["dim"], case["heads"], case["kv"], case["rot"], case["page"]
    b, _, pos, _ = _places(s)
    # keys in 64 bits: next to the border of two codes 32 lose which one it is
    x = s["qkv"].view(s["T"], Hq + 2 * Hk, D).double()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    if case["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + EPS) * s["q_norm"].double()
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + EPS) * s["k_norm"].double()
    if rot:
        c, sn = s["rope"][pos, None, :rot // 2].double(), s["rope"][pos, None, rot // 2:].double()
        q, k = _turn(q, c, sn, rot, case["interleaved"]), _turn(k, c, sn, rot, case["interleaved"])
    page, row = s["table"][b, pos // ps].long(), pos % ps
    out = {"q": q.to(s["qkv"].dtype)}
    for name, x, cache in (("k", k, s["kc"]), ("v", v, s["vc"])):
        codes, sc, z = _quantised(x.to(s["qkv"].dtype).unflatten(-1, (D // 64, 64)), case["dtype"])
        rows = _packed(codes[..., None, :, :], sc[..., None, :], z[..., None, :])  # each as a page of one row
        n, m = D // 2, D // 32
        j = torch.arange(n, device=DEV)
        cache[page[:, None], :, row[:, None] * n + j] = rows[..., :n].transpose(1, 2)
        j = torch.arange(m, device=DEV)
        cache[page[:, None], :, ps * n + row[:, None] * m + j] = rows[..., n:].transpose(1, 2)
        out[name] = _stands_for(codes, sc, z).to(s["qkv"].dtype)
    return out


def _turn(x, c, sn, rot, interleaved):
    y = x[..., :rot]
    if interleaved:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:]
        y = torch.cat([a * c - b * sn, b * c + a * sn], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_attention(s, case):
    D, Hq, Hk, B, T, ps = case["dim"], case["heads"], case["kv"], case["seqs"], s["T"], case["page"]
    G, N, L = Hq // Hk, s["max_new"], s["max_len"]
    b, i, pos, n = _places(s)
    lens = s["lens"].long()
    # rows of the batch, padded to the longest sequence's new tokens: [B, Hk, G, N, D]
    q = torch.zeros(B, N, Hk, G, D, device=DEV)
    q[b, i] = s["q"].float().view(T, Hk, G, D)
    q = q.permute(0, 2, 3, 1, 4).reshape(B, Hk, G * N, D)
    p = torch.full((B, N), -1, dtype=torch.long, device=DEV)
    p[b, i] = pos
    j = torch.arange(L, device=DEV)
    keys = []
    for cache in (s["kc"], s["vc"]):
        x = _stands_for(*_block_rows(cache, ps, D))  # [pages, Hk, ps, D]
        x = x[s["table"].clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(B, Hk, -1, D)[:, :, :L]
        keys.append(torch.where((j < lens[:, None])[:, None, :, None], x, 0.0))
    see = j <= p[..., None]
    if case["prefix"]:
        see = see | (j < s["prefix"].long()[:, None, None])
    if case["window"]:
        see = see & (j > p[..., None] - case["window"])
    see = (see & (j < lens[:, None, None]) & (p >= 0)[..., None])[:, None, None]
    x = (torch.matmul(q, keys[0].transpose(-1, -2)) * D ** -0.5).view(B, Hk, G, N, L)
    if case["softcap"]:
        x = case["softcap"] * torch.tanh(x / case["softcap"])
    if case["bias"]:
        x = x + s["slopes"].view(1, Hk, G, 1, 1) * (j - p[..., None])[:, None, None].float()
    x = torch.where(see, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(m.isinf(), 0.0, m))
    total = w.sum(-1, keepdim=True)
    lse = torch.where(total > 0, m + torch.log(total), -math.inf)[..., 0]
    o = torch.matmul(w.view(B, Hk, G * N, L), keys[1]).view(B, Hk, G, N, D) / torch.where(total > 0, total, 1.0)
    o, lse = o.permute(0, 3, 1, 2, 4)[b, i], lse.permute(0, 3, 1, 2)[b, i]
    return {"out": o.reshape(T, Hq, D).to(s["q"].dtype), "lse": lse.reshape(T, Hq).contiguous()}


def work(case):
    if case["op"] == "plan":
        reqs, page = _requests(case), case["page"]
        _, asked, back = _need(case)
        tokens = (sum(new for _, new, _ in reqs) + 63) // 64 * 64
        # lengths, new tokens, flags, the page that a sequence goes on in; its length and boundary; pages; tokens
        return {"bytes": len(reqs) * (9.0 + 4 + 8) + 8.0 * (asked + back) + 12.0 * tokens + 36, "flops": 10.0 * len(reqs) + 4.0 * tokens}
    if case["op"] == "norm":
        T, H = case["tokens"], case["hidden"]
        gate = {"channel": H, "token": T, "element": T * H}.get(case["gate"], 0)
        return {"bytes": 2.0 * (T * H * (3 + case["pre"]) + gate + H * (case["post"] + case["pre"])),
                "flops": T * H * (3.0 + 4 * case["post"] + 4 * case["pre"] + (gate > 0))}
    D, Hq, Hk = case["dim"], case["heads"], case["kv"]
    row = 17.0 * D / 32  # bytes of a key
    pairs = _lengths(case)
    T = sum(n for n, _ in pairs)
    if case["op"] == "append":
        # in and out in 16 bits, the cache's rows, and again as they are read back
        flops = T * (Hq + Hk) * (4.0 * D * case["norm"] + 3.0 * case["rot"]) + T * 2.0 * Hk * D * 6
        return {"bytes": T * ((2.0 * Hq + 2 * Hk) * D * 2 + 4 * Hk * row + 2 * Hk * D * 2 + case["rot"] * 4), "flops": flops}
    keys = visible = 0
    for n, length in pairs:
        spans = [_visible(case, n, length, i) for i in range(n)]
        visible += sum(e - f for f, e in spans)
        keys += max([e for f, e in spans if e > f], default=0) - min([f for f, e in spans if e > f], default=0)
    return {"bytes": keys * Hk * 2 * row + T * Hq * (D * 4.0 + 4), "flops": 4.0 * D * Hq * visible}


# ------------------------------------------------------------ definitions in 64 bits --

def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "norm": _exact_norm, "append": _exact_append}.get(case["op"], _exact_attention)(s, case)


def _exact_plan(s, case):
    page, T = case["page"], s["T"]
    ring, table = s["ring"].tolist(), s["table"].tolist()
    taken, returned = s["state"].tolist()
    cap, width, free = len(ring), len(table[0]), returned - taken
    lens, add, over = s["lens"].tolist(), s["add"].tolist(), s["over"].tolist()
    at, asked, rows, took = returned, 0, 0, 0
    for b, gone in enumerate(over):
        if gone:
            for p in table[b][:min(width, _pages(lens[b], page))]:
                ring[at % cap] = p
                at += 1
            lens[b] = 0
    cu, positions, slots = [0], [], []
    for b, n in enumerate(add):
        held, end = _pages(lens[b], page), lens[b] + n
        if end <= width * page:
            need = _pages(end, page) - held
            asked, rows = asked + need, rows + n
            if (need and asked > free) or (n and rows > T):
                n = 0
            else:
                for i in range(need):
                    table[b][held + i] = ring[(taken + asked - need + i) % cap]
                took = asked if need else took
        else:
            n = 0
        for pos in range(lens[b], lens[b] + n):
            positions.append(pos)
            slots.append(table[b][pos // page] * page + pos % page)
        lens[b] += n
        cu.append(cu[-1] + n)
    pad = [-1] * (T - len(slots))
    t = lambda v, dt: torch.tensor(v, dtype=dt, device=DEV)  # noqa: E731
    return {"lens": t(lens, torch.int32), "cu_q": t(cu, torch.int32), "positions": t(positions + pad, torch.int32),
            "slots": t(slots + pad, torch.int64), "table": t(table, torch.int32), "ring": t(ring, torch.int32),
            "state": t([taken + took, at], torch.int64)}


def _exact_norm(s, case):
    def unit(x, gain):
        return x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / x.shape[-1] + EPS) * gain.double()

    u = unit(s["y"].double(), s["post"]) if case["post"] else s["y"].double()
    h = s["h"].double() * RESIDUAL_SCALE + (u if s["gate"] is None else s["gate"].double() * u) * SCALE
    return {"h": h, "x": unit(h.to(s["h"].dtype).double(), s["pre"])} if case["pre"] else {"h": h}


def _exact_append(s, case):
    D, Hq, Hk, ps = case["dim"], case["heads"], case["kv"], case["page"]
    lens, dtype = s["lens"].tolist(), s["qkv"].dtype
    cu = list(range(case["seqs"] + 1)) if s["cu"] is None else s["cu"].tolist()
    outs = [torch.empty(s["T"], n, D, dtype=torch.float64, device=DEV) for n in (Hq, Hk, Hk)]
    for b, length in enumerate(lens):
        x = s["qkv"][cu[b]:cu[b + 1]].double().view(-1, Hq + 2 * Hk, D)
        pos = torch.arange(length - x.shape[0], length, device=DEV)
        for i, (part, gain) in enumerate(((x[:, :Hq], s["q_norm"]), (x[:, Hq:Hq + Hk], s["k_norm"]), (x[:, Hq + Hk:], None))):
            if case["norm"] and i < 2:
                part = part / torch.sqrt(torch.linalg.vector_norm(part, dim=-1, keepdim=True) ** 2 / D + EPS) * gain.double()
            if case["rot"] and i < 2:
                half = case["rot"] // 2
                w = torch.complex(*(s["rope"][pos].double()[:, None, k * half:(k + 1) * half].contiguous() for k in (0, 1)))
                part = part.clone()
                lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))
                z = torch.complex(part[..., lo].contiguous(), part[..., hi].contiguous()) * w
                part[..., lo], part[..., hi] = z.real, z.imag
            if i:  # stored: the grid of the group, element by element
                y = part.to(dtype).double().reshape(-1, Hk, D // 64, 64)
                span = (y.amax(-1, keepdim=True).clamp(min=0) / 16).float() - (y.amin(-1, keepdim=True).clamp(max=0) / 16).float()
                need = span.double() * 16 / 15
                e = torch.floor(torch.log2(need.clamp(min=1e-60)))
                step = torch.full_like(need, math.inf)
                for d in (-1, 0, 1, 2):  # the numbers of four significant bits around it
                    for m in range(8, 16):
                        v = m * _power(e + d - 3)
                        step = torch.where((v >= need) & (v < step), v, step)
                step = step.clamp(min=SMALLEST[case["dtype"]])
                zero = torch.floor(0.5 - y.amin(-1, keepdim=True).clamp(max=0) / step)
                most = torch.floor(torch.finfo(dtype).max / step)
                n = torch.floor(y / step + 0.5)
                n = torch.minimum(torch.maximum(n, torch.maximum(-zero, -most)), torch.minimum(15 - zero, most))
                part = (n * step).reshape(-1, Hk, D)
            outs[i][cu[b]:cu[b + 1]] = part
    return {"q": outs[0], "k": outs[1], "v": outs[2]}


def _exact_attention(s, case):
    D, Hq, Hk, ps = case["dim"], case["heads"], case["kv"], case["page"]
    G, lens, table = Hq // Hk, s["lens"].tolist(), s["table"].long()
    cu = list(range(case["seqs"] + 1)) if s["cu"] is None else s["cu"].tolist()
    out = torch.zeros(s["T"], Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.full((s["T"], Hq), -math.inf, dtype=torch.float64, device=DEV)
    # where an element's code and its group's word lie in a block
    d = torch.arange(D, device=DEV)
    group, e = d // 64, d % 64
    byte = ((e // 8) * (D // 64) + group) * 4 + (e % 2) * 2 + (e % 8) // 4
    shift = (e % 8) // 2 % 2 * 4
    rows = 2048

    def read(cache, b, h, j):
        blocks = cache[table[b, j // ps], h]
        r = (j % ps)[:, None]
        code = torch.gather(blocks, 1, r * (D // 2) + byte).int() >> shift & 15
        at = ps * (D // 2) + r * (D // 32) + 2 * group
        word = torch.gather(blocks, 1, at).int() | torch.gather(blocks, 1, at + 1).int() << 8
        return (code - (word & 15)).double() * (1 + (word >> 4 & 7).double() / 8) * _power((word >> 7 & 255) - 127)

    for b, length in enumerate(lens):
        n = cu[b + 1] - cu[b]
        if length == 0:
            continue
        j = torch.arange(length, device=DEV)
        for h in range(Hk):
            k, v = read(s["kc"], b, h, j), read(s["vc"], b, h, j)
            for head in range(h * G, (h + 1) * G):
                for i0 in range(0, n, rows):
                    i = torch.arange(i0, min(n, i0 + rows), device=DEV)
                    p = (length - n + i)[:, None]
                    x = s["q"][cu[b] + i, head].double() @ k.T / math.sqrt(D)
                    if case["softcap"]:
                        x = torch.tanh(x / case["softcap"]) * case["softcap"]
                    if case["bias"]:
                        x = x - (p - j) * float(s["slopes"][head])
                    hide = j > p
                    if case["prefix"]:
                        hide &= j >= int(s["prefix"][b])
                    if case["window"]:
                        hide |= j <= p - case["window"]
                    x = x.masked_fill(hide, -math.inf)
                    lse[cu[b] + i, head] = torch.logsumexp(x, -1)
                    out[cu[b] + i, head] = torch.softmax(x, -1) @ v
    return {"out": out, "lse": lse}
