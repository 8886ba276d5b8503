"""The attention half of a decoder layer over a paged key-value cache: three operators.

  append   ``kv_append``: per-head norms of queries and keys, the position rotation, and
           the keys and values of new tokens written into the cache's pages, in one pass
  decode   ``attn_decode``: attention of one new token per sequence over the cache
  prefill  ``attn_prefill``: attention of many new tokens per sequence (a ragged batch)
           over the cache, causal, with a prefix that every query sees

Both attentions take a tanh cap on the scores, a sliding window and a bias that is
linear in the distance.  Token i of a sequence's n new ones sits at position
p = len - n + i and sees the keys j <= p, and j < prefix, that have j > p - window.

A case names its sizes; how the lengths of a ragged batch are spread follows from the
case alone, their order in the batch and every value from the seed.  Heads, head sizes
and the decode batch are the Mixtral block's (32 query heads on 8 key-value heads of
128) or generic ones.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
GOLDEN = 0.6180339887498949


def _case(op, seqs, new, ctx, heads=32, kv=8, dim=128, dtype="bf16", page=64, ragged=False, empty=False, softcap=0.0,
          window=0, bias=False, prefix=False, norm=False, rot=0, interleaved=False):
    return {"op": op, "seqs": seqs, "new": new, "ctx": ctx, "heads": heads, "kv": kv, "dim": dim, "dtype": dtype,
            "page": page, "ragged": ragged, "empty": empty, "softcap": softcap, "window": window, "bias": bias,
            "prefix": prefix, "norm": norm, "rot": rot, "interleaved": interleaved}


def listed():
    return [
        # the new tokens of a decode batch: latency counts
        {"name": "append_decode48", **_case("append", 48, 1, 700, page=16, ragged=True, rot=128)},
        # a few prompts, normed heads of 64, half of each head rotated in interleaved pairs
        {"name": "append_ragged7", **_case("append", 7, 301, 500, heads=24, dim=64, dtype="fp16", page=48, ragged=True,
                                           norm=True, rot=32, interleaved=True)},
        # a long prompt of one user, norms and full rotation: bandwidth counts
        {"name": "append_prompt8192", **_case("append", 1, 8192, 8192, norm=True, rot=128)},
        # one user, a short conversation: the smallest call
        {"name": "decode1_777", **_case("decode", 1, 1, 777)},
        # the benchmark's decode batch, lengths of every size, idle slots among them
        {"name": "decode16_ragged", **_case("decode", 16, 1, 4099, page=16, ragged=True, empty=True)},
        # many users with long contexts
        {"name": "decode64_8192", **_case("decode", 64, 1, 8192, page=128)},
        # one user with a very long document
        {"name": "decode1_131071", **_case("decode", 1, 1, 131071, page=256)},
        # capped scores, a window and the distance bias, twelve query heads of 64 on a key head
        {"name": "decode33_window", **_case("decode", 33, 1, 6001, heads=48, kv=4, dim=64, dtype="fp16", page=32,
                                            ragged=True, softcap=50.0, window=1024, bias=True)},
        # the verification of five drafted tokens of sixteen users, capped scores
        {"name": "prefill16_verify5", **_case("prefill", 16, 5, 2047, page=16, ragged=True, softcap=30.0)},
        # a batch of odd prompts, heads of 64, a bidirectional prefix and the distance bias
        {"name": "prefill9_ragged", **_case("prefill", 9, 777, 1013, heads=12, kv=4, dim=64, dtype="fp16", page=48,
                                            ragged=True, bias=True, prefix=True)},
        # a chunk of a long prompt on what is already in the cache
        {"name": "prefill1_chunk509", **_case("prefill", 1, 509, 30000, page=128)},
        # a long prompt in one piece
        {"name": "prefill1_8192", **_case("prefill", 1, 8192, 8192)},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "prefill", "prefill"])
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


def _lengths(case):
    """[(new tokens, length in the cache with them)] of the batch, spread by the case alone."""
    out = []
    for b in range(case["seqs"]):
        f = 1.0 if not case["ragged"] or b == 0 else math.modf((b + 1) * GOLDEN)[0]
        g = 1.0 if not case["ragged"] or b == 0 else math.modf((b + 1) * GOLDEN * GOLDEN + 0.3)[0]
        n = 1 + int((case["new"] - 1) * g)
        length = max(n, 1 + int((case["ctx"] - 1) * f))
        if case["empty"] and b % 8 == 5:
            length = 0  # an idle slot of the batch
        out.append((n, length))
    return out


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


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
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
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=torch.float32)  # noqa: E731
    kc, vc = (torch.empty(pages, Hk, ps, D, dtype=dtype, device=DEV) for _ in range(2))
    for c in (kc, vc):
        c.normal_(generator=g)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s = {"case": case, "T": T, "max_new": max(new), "max_len": max(lens), "kc": kc, "vc": vc, "lens": i32(lens),
         "table": table, "cu": None if case["op"] == "decode" or case["new"] == 1 and case["op"] == "append" else i32(cu),
         "slopes": torch.tensor(_slopes(Hq), dtype=torch.float32, device=DEV) if case["bias"] else None,
         "prefix": i32([_prefix(n, length) for n, length in pairs]) if case["prefix"] else None}
    if case["op"] == "append":
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
        # rows of a page that no token was written to yet hold whatever memory held
        last = [(int(free[sum(need[:b]) + need[b] - 1]), lens[b] % ps) for b in range(B) if lens[b] % ps]
        for page, row in last:
            kc[page, :, row:] = float("nan")
            vc[page, :, row:] = float("nan")
    if own:
        import paper_2410_06270_gb300 as mc
        s["cache"], s["batch"] = mc.KVCache(kc, vc), mc.KVBatch(s["lens"], table, s["cu"], tokens=T)
        s["ws"] = mc.attn_workspace(s["cache"], Hq)
    return s


def run(state):
    s, case = state, state["case"]
    D, Hq, Hk = case["dim"], case["heads"], case["kv"]
    scale = D ** -0.5
    if own:
        import paper_2410_06270_gb300 as mc
        if case["op"] == "append":
            x = s["qkv"].view(s["T"], Hq + 2 * Hk, D)
            q = mc.kv_append(s["cache"], s["batch"], x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:], rope=s["rope"],
                             interleaved=case["interleaved"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS,
                             workspace=s["ws"])
            return {"q": q, "k_cache": s["kc"], "v_cache": s["vc"]}
        if case["op"] == "decode":
            out, lse = mc.attn_decode(s["cache"], s["batch"], s["q"], scale=scale, softcap=case["softcap"],
                                      window=case["window"], slopes=s["slopes"], with_lse=True, workspace=s["ws"])
        else:
            out, lse = mc.attn_prefill(s["cache"], s["batch"], s["q"], scale=scale, softcap=case["softcap"],
                                       window=case["window"], slopes=s["slopes"], prefix=s["prefix"], with_lse=True,
                                       workspace=s["ws"])
        return {"out": out, "lse": lse}
    if case["op"] == "append":
        return _plain_append(s, case)
    return _plain_attention(s, case, scale)


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
    x = s["qkv"].view(s["T"], Hq + 2 * Hk, D).float()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    if case["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + EPS) * s["q_norm"].float()
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + EPS) * s["k_norm"].float()
    if rot:
        c, sn = s["rope"][pos, None, :rot // 2], s["rope"][pos, None, rot // 2:]
        q, k = _turn(q, c, sn, rot, case["interleaved"]), _turn(k, c, sn, rot, case["interleaved"])
    page, row = s["table"][b, pos // ps].long(), pos % ps
    s["kc"][page, :, row] = k.to(s["kc"].dtype)
    s["vc"][page, :, row] = v.to(s["vc"].dtype)
    return {"q": q.to(s["qkv"].dtype), "k_cache": s["kc"], "v_cache": s["vc"]}


def _turn(x, c, sn, rot, interleaved):
    y = x[..., :rot]
    if interleaved:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:]
        y = torch.cat([a * c - b * sn, b * c + a * sn], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_attention(s, case, scale):
    D, Hq, Hk, B, T = case["dim"], case["heads"], case["kv"], case["seqs"], s["T"]
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
    keys = [c[s["table"].clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(B, Hk, -1, D)[:, :, :L].float()
            for c in (s["kc"], s["vc"])]
    v = torch.where((j < lens[:, None])[:, None, :, None], keys[1], 0.0)
    see = j <= p[..., None]
    if case["prefix"]:
        see = see | (j < s["prefix"].long()[:, None, None])
    if case["window"]:
        see = see & (j > p[..., None] - case["window"])
    see = (see & (j < lens[:, None, None]) & (p >= 0)[..., None])[:, None, None]
    x = (torch.matmul(q, keys[0].transpose(-1, -2)) * scale).view(B, Hk, G, N, L)
    if case["softcap"]:
        x = case["softcap"] * torch.tanh(x / case["softcap"])
    if case["bias"]:
        x = x + s["slopes"].view(1, Hk, G, 1, 1) * (j - p[..., None])[:, None, None].float()
    x = torch.where(see, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(m.isinf(), 0.0, m))
    total = w.sum(-1, keepdim=True)
    lse = torch.where(total > 0, m + torch.log(total), -math.inf)[..., 0]
    o = torch.matmul(w.view(B, Hk, G * N, L), v).view(B, Hk, G, N, D) / torch.where(total > 0, total, 1.0)
    o, lse = o.permute(0, 3, 1, 2, 4)[b, i], lse.permute(0, 3, 1, 2)[b, i]
    return {"out": o.reshape(T, Hq, D).to(s["q"].dtype), "lse": lse.reshape(T, Hq).contiguous()}


def work(case):
    D, Hq, Hk = case["dim"], case["heads"], case["kv"]
    pairs = _lengths(case)
    T = sum(n for n, _ in pairs)
    if case["op"] == "append":
        heads = Hq + 2 * Hk
        flops = T * (Hq + Hk) * (4.0 * D * case["norm"] + 3.0 * case["rot"])
        return {"bytes": T * (2.0 * heads * D * 2 + case["rot"] * 4), "flops": flops}
    keys = visible = 0
    for n, length in pairs:
        spans = [_visible(case, n, length, i) for i in range(n)]
        visible += sum(e - f for f, e in spans)
        keys += max([e for f, e in spans if e > f], default=0) - min([f for f, e in spans if e > f], default=0)
    return {"bytes": keys * Hk * D * 4.0 + T * Hq * (D * 4.0 + 4), "flops": 4.0 * D * Hq * visible}


def exact(case, seed):
    s = prepare(case, seed)
    kc, vc, lens, table = s["kc"], s["vc"], s["lens"].tolist(), s["table"].long()
    D, Hq, Hk, ps = case["dim"], case["heads"], case["kv"], case["page"]
    G = Hq // Hk
    cu = list(range(case["seqs"] + 1)) if s["cu"] is None else s["cu"].tolist()
    if case["op"] == "append":
        q_out = torch.empty(s["T"], Hq, D, dtype=torch.float64, device=DEV)
        new_k, new_v = kc.double(), vc.double()
        for b, length in enumerate(lens):
            x = s["qkv"][cu[b]:cu[b + 1]].double().view(-1, Hq + 2 * Hk, D)
            pos = torch.arange(length - x.shape[0], length, device=DEV)
            sides = []
            for part, gain in ((x[:, :Hq], s["q_norm"]), (x[:, Hq:Hq + Hk], s["k_norm"])):
                if case["norm"]:
                    part = part / torch.sqrt(torch.linalg.vector_norm(part, dim=-1, keepdim=True) ** 2 / D + EPS) * gain.double()
                if case["rot"]:
                    half = case["rot"] // 2
                    w = torch.complex(*(s["rope"][pos].double()[:, None, k * half:(k + 1) * half].contiguous() for k in (0, 1)))
                    part = part.clone()
                    lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))
                    z = torch.complex(part[..., lo].contiguous(), part[..., hi].contiguous()) * w
                    part[..., lo], part[..., hi] = z.real, z.imag
                sides.append(part)
            q_out[cu[b]:cu[b + 1]] = sides[0]
            for h in range(Hk):
                new_k[table[b, pos // ps], h, pos % ps] = sides[1][:, h]
                new_v[table[b, pos // ps], h, pos % ps] = x[:, Hq + Hk + h]
        return {"q": q_out, "k_cache": new_k, "v_cache": new_v}
    out = torch.zeros(s["T"], Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.full((s["T"], Hq), -math.inf, dtype=torch.float64, device=DEV)
    rows = 2048
    for b, length in enumerate(lens):
        n = cu[b + 1] - cu[b]
        if length == 0:
            continue
        j = torch.arange(length, device=DEV)
        for h in range(Hk):
            k, v = (c[table[b, j // ps], h, j % ps].double() for c in (kc, vc))
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
