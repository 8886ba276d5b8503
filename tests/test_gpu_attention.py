"""The paged cache's append and the two attentions over it against their definitions in
64 bits: head layouts, types, page sizes, lengths around every tile's edges, empty rows,
masks, strides, NaN where nothing was written, streams, graphs and repeated calls."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import attn_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2410_06270_gb300 import build
    build.build()
    import paper_2410_06270_gb300 as m
    m.load()
    m.set_debug(0, 1_000_000_000)
    return m


EDGES = [0, 1, 2, 15, 16, 17, 31, 63, 64, 65, 100, 127, 128, 129, 255, 257, 700]


# ---------------------------------------------------------------- append --

@pytest.mark.parametrize("heads,kv,dim,dtype,page,rot,interleaved,norm,ragged", [
    (32, 8, 128, "bf16", 16, 128, False, False, False),
    (12, 4, 64, "fp16", 48, 32, True, True, True),
    (5, 1, 128, "bf16", 64, 64, False, True, True),
    (3, 3, 64, "bf16", 16, 64, False, False, True),
    (7, 7, 128, "fp16", 32, 16, True, False, False),
    (16, 2, 128, "fp16", 128, 0, False, True, True),
    (1, 1, 64, "bf16", 16, 16, False, True, False),
])
def test_append_matches_its_definition(mc, heads, kv, dim, dtype, page, rot, interleaved, norm, ragged):
    lens = [0, 1, page, page + 1, 100, 5 * page - 1, 3]
    new = [0, 1, page, 2, 100, 33, 5] if ragged else [1] * len(lens)  # the last: more new tokens than its length
    B = ref.Batch(lens, new, kv, page, dim, dtype, 11, pad_tokens=3 if ragged else 0)
    qkv = B.randn(B.tokens, (heads + 2 * kv) * dim + 8)  # a row's tail is not the call's
    cut = lambda x, a, n: x[:, a * dim:(a + n) * dim].unflatten(1, (n, dim))  # noqa: E731
    qn, kn = ((1 + 0.1 * B.randn(dim)).to(ref.DT[dtype]) for _ in range(2)) if norm else (None, None)
    rope = ref.rope_table(600, rot) if rot else None
    parts = [cut(qkv, 0, heads), cut(qkv, heads, kv), cut(qkv, heads + kv, kv)]
    want = ref.append(B, *parts, rope, interleaved, qn, kn)
    cache, batch = B.device(mc, cu=ragged)
    ws = mc.attn_workspace(cache, heads)
    dev = qkv.cuda()
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    q_out = torch.full((B.tokens, heads, dim), 7.0, dtype=ref.DT[dtype], device="cuda")
    q = mc.kv_append(cache, batch, cut(dev, 0, heads), cut(dev, heads, kv), cut(dev, heads + kv, kv), rope=up(rope),
                     interleaved=interleaved, q_norm=up(qn), k_norm=up(kn), q_out=q_out, workspace=ws)
    mc.check_status(ws)
    assert q.data_ptr() == q_out.data_ptr()
    n = B.cu[-1]
    assert (q[n:] == 7).all()  # padding is left alone
    # one rounding of a value formed in fp32 (a few units of 2^-24 of the pair's larger member)
    for got, ex in ((q[:n], want[0][:n]), (cache.k, want[1]), (cache.v, want[2])):
        got = got.double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(ex))
        ok = ~torch.isnan(ex)
        assert ((got - ex)[ok].abs() <= ref.HALF_ULP[dtype] * ex[ok].abs() + 2.0 ** -20 * 8 + (2.0 ** -24 if dtype == "fp16" else 0)).all()
    assert torch.equal(torch.nan_to_num(cache.v.cpu()), torch.nan_to_num(want[2].to(ref.DT[dtype])))  # copied bits


def test_append_in_place_and_long_offsets(mc):
    """q_out may be q; a page far into a strided pool lies past 2^31 elements."""
    B = ref.Batch([70], [70], 2, 64, 64, "bf16", 3, spare=0)
    big = torch.zeros((1 << 31) // 4 * 5 // 4 + (1 << 20), dtype=torch.int64, device="cuda").view(torch.bfloat16)
    stride = (1 << 31) + 1024
    k = big.as_strided((2, 2, 64, 64), (stride, 64 * 64, 64, 1))
    v = big.as_strided((2, 2, 64, 64), (stride, 64 * 64, 64, 1), 64 * 64 * 2)
    cache = mc.KVCache(k, v)
    batch = mc.KVBatch(torch.tensor([70], dtype=torch.int32).cuda(), B.table.cuda(),
                       torch.tensor([0, 70], dtype=torch.int32).cuda(), 70)
    x = B.randn(3, 70, 2, 64)
    rope = ref.rope_table(70, 64)
    want = ref.append(B, x[0], x[1], x[2], rope)
    q = x[0].cuda()
    got = mc.kv_append(cache, batch, q, x[1].cuda(), x[2].cuda(), rope=rope.cuda(), q_out=q)
    assert got.data_ptr() == q.data_ptr()
    assert (got.double().cpu() - want[0]).abs().max() <= 2.0 ** -8 * want[0].abs().max() + 1e-5
    for c, w in ((k, want[1]), (v, want[2])):
        ok = ~torch.isnan(w)
        assert ((c.double().cpu() - w)[ok].abs() <= 2.0 ** -8 * w[ok].abs() + 1e-5).all()
    q2 = x[0].cuda()
    out = mc.attn_prefill(cache, batch, q2)
    att = ref.Batch([70], [70], 2, 64, 64, "bf16", 3, spare=0)
    att.k, att.v = k.cpu(), v.cpu()
    w = ref.attention(att, x[0], 64 ** -0.5)
    ref.assert_attention(out, None, w, "bf16", 70, 5.0)


# ---------------------------------------------------------------- decode --

DECODE = [
    # heads, kv, dim, dtype, page, softcap, window, bias
    (32, 8, 128, "bf16", 16, 0.0, 0, False),
    (8, 8, 64, "fp16", 48, 0.0, 0, False),
    (6, 2, 128, "fp16", 64, 30.0, 0, True),
    (48, 4, 64, "bf16", 32, 0.0, 50, False),
    (16, 1, 128, "bf16", 128, 50.0, 129, True),
    (40, 2, 128, "bf16", 16, 0.0, 1, False),
    (33, 1, 64, "fp16", 16, 0.0, 0, True),
    (1, 1, 128, "bf16", 256, 0.0, 0, False),
]


def _slopes(heads):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)])


@pytest.mark.parametrize("heads,kv,dim,dtype,page,softcap,window,bias", DECODE)
def test_decode_matches_its_definition(mc, heads, kv, dim, dtype, page, softcap, window, bias):
    B = ref.Batch(EDGES, [1] * len(EDGES), kv, page, dim, dtype, 5, interleave=True)
    q = 1.5 * B.randn(len(EDGES), heads, dim)
    sl = _slopes(heads) if bias else None
    want = ref.attention(B, q, dim ** -0.5, softcap, window, sl)
    cache, batch = B.device(mc, cu=False, interleave=True)
    ws = mc.attn_workspace(cache, heads)
    out, lse = mc.attn_decode(cache, batch, q.cuda(), softcap=softcap, window=window,
                              slopes=None if sl is None else sl.cuda(), with_lse=True, workspace=ws)
    mc.check_status(ws)
    ref.assert_attention(out, lse, want, dtype, max(EDGES), 5.0)


@pytest.mark.parametrize("seqs,length,kv,heads", [(1, 5000, 1, 8), (1, 20011, 2, 8), (3, 2049, 8, 32), (300, 40, 1, 2), (1, 1, 1, 1),
                                                   (70, 900, 2, 8), (128, 129, 1, 16)])
def test_decode_splits_and_joins(mc, seqs, length, kv, heads):
    lens = [max(1, length - 37 * b) if seqs < 100 else (b * 7) % length for b in range(seqs)]
    B = ref.Batch(lens, [1] * seqs, kv, 32, 128, "bf16", 8)
    q = B.randn(seqs, heads, 128)
    want = ref.attention(B, q, 0.1)
    cache, batch = B.device(mc, cu=False)
    out, lse = mc.attn_decode(cache, batch, q.cuda(), scale=0.1, with_lse=True)
    ref.assert_attention(out, lse, want, "bf16", length, 5.0)
    again, _ = mc.attn_decode(cache, batch, q.cuda(), scale=0.1, with_lse=True)
    assert torch.equal(out, again)  # the same sums in the same order


def test_decode_large_scores(mc):
    """One key far above the others, early or late: running maxima have to move."""
    for at in (0, 300, 999):
        B = ref.Batch([1000], [1], 1, 16, 64, "bf16", 9)
        q = B.randn(1, 4, 64)
        B.k[B.table[0, at // 16], 0, at % 16] = (q[0, 1] * 20).to(torch.bfloat16)
        want = ref.attention(B, q, 1.0)
        cache, batch = B.device(mc, cu=False)
        out, lse = mc.attn_decode(cache, batch, q.cuda(), scale=1.0, with_lse=True)
        assert (out.double().cpu() - want[0]).abs().max() <= 2.0 ** -8 * 5 + 2e-2  # scores of hundreds: 1e-5 of them in fp32
        assert ((lse.double().cpu() - want[1]).abs() <= 1e-5 * want[1].abs() + 1e-4).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("below", [9.0, 14.0, 17.0, 17.40625])  # (fp16 and, but for the last, bf16 hold them)
@pytest.mark.parametrize("new,group", [(1, 1), (32, 8)])  # each kernel
def test_small_weights_keep_their_sum(mc, dtype, below, new, group):
    """8191 equal keys far below one: each weighs little, in fp16 less than the type's normal numbers,
    together they weigh what they should.  A weight of the largest one's 2^-21 or more is rounded to
    half an ulp, a smaller one to 2^-25 of 2^7."""
    if dtype == "bf16" and below == 17.40625:
        below = 17.375
    seqs, kv, length, dim = 40, 8, 8192, 64
    k, v = (torch.zeros(length // 128, kv, 128, dim, dtype=ref.DT[dtype], device="cuda") for _ in range(2))
    v[:] = torch.linspace(1, 64, dim, device="cuda").to(v.dtype)
    k[0, :, 0, 0], v[0, :, 0] = below, 0.0
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    table = torch.arange(length // 128, dtype=torch.int32, device="cuda").repeat(seqs, 1)  # (one cache for all)
    cache = mc.KVCache(k, v)
    batch = mc.KVBatch(i32([length] * seqs), table, i32([new * b for b in range(seqs + 1)]), new * seqs)
    q = torch.zeros(new * seqs, kv * group, dim, dtype=ref.DT[dtype], device="cuda")
    q[..., 0] = 1.0
    out, lse = mc.attn_prefill(cache, batch, q, scale=1.0, with_lse=True)
    others = torch.arange(length - new, length, dtype=torch.float64)  # keys after the first one, of each new token
    w = others * np.exp(-below)
    want = (w / (1 + w))[:, None] * v[0, 0, 1].double().cpu()
    h = ref.HALF_ULP[dtype]
    tol = (2 * h + 1e-4) * want + (2.0 ** -24 + length * 2.0 ** -32 * 64 if dtype == "fp16" else 0)
    assert ((out.view(seqs, new, kv * group, dim).double().cpu() - want[:, None]).abs() <= tol[:, None]).all()
    assert ((lse.view(seqs, new, kv * group).double().cpu() - (below + torch.log1p(w))[:, None]).abs() <= 1e-4).all()


# --------------------------------------------------------------- prefill --

PREFILL = [
    # heads, kv, dim, dtype, page, softcap, window, bias, prefix
    (8, 2, 128, "bf16", 16, 0.0, 0, False, False),
    (4, 4, 64, "fp16", 48, 0.0, 0, False, True),
    (6, 2, 128, "fp16", 64, 30.0, 0, True, False),
    (12, 1, 64, "bf16", 32, 0.0, 50, False, False),
    (5, 1, 128, "bf16", 128, 50.0, 129, True, True),
    (8, 8, 64, "bf16", 16, 0.0, 1, False, False),
    (2, 1, 128, "fp16", 256, 0.0, 300, False, True),
]


@pytest.mark.parametrize("heads,kv,dim,dtype,page,softcap,window,bias,prefix", PREFILL)
def test_prefill_matches_its_definition(mc, heads, kv, dim, dtype, page, softcap, window, bias, prefix):
    lens = [0, 1, 17, 64, 130, 300, 511, 9, 257]
    new = [2, 1, 17, 3, 130, 1, 129, 12, 64]  # sequences 0 and 7: more new tokens than their length
    B = ref.Batch(lens, new, kv, page, dim, dtype, 6, pad_tokens=2)
    q = 1.5 * B.randn(B.tokens, heads, dim)
    sl = _slopes(heads) if bias else None
    pre = [0, 1, 9, 64, 70, 299, 1000, 4, 250] if prefix else None
    want = ref.attention(B, q, dim ** -0.5, softcap, window, sl, pre)
    cache, batch = B.device(mc)
    ws = mc.attn_workspace(cache, heads)
    out = torch.full((B.tokens, heads + 1, dim), 3.0, dtype=ref.DT[dtype], device="cuda")
    got, lse = mc.attn_prefill(cache, batch, q.cuda(), softcap=softcap, window=window,
                               slopes=None if sl is None else sl.cuda(),
                               prefix=None if pre is None else torch.tensor(pre, dtype=torch.int32).cuda(),
                               out=out[:, :heads], with_lse=True, workspace=ws)
    mc.check_status(ws)
    n = B.cu[-1]
    assert (out[:, heads] == 3).all() and (out[n:] == 3).all()  # other heads' columns and padding rows
    ref.assert_attention(got, lse, want, dtype, 512, 5.0, rows=slice(0, n))


@pytest.mark.parametrize("heads,kv,dim,dtype,page,softcap,window,bias,prefix", [
    # few rows a sequence: slices of 8, 16 and 32 rows, some sequences with more than one
    (4, 4, 128, "bf16", 16, 0.0, 0, False, False),
    (3, 1, 64, "fp16", 48, 0.0, 20, True, False),
    (8, 2, 128, "bf16", 32, 30.0, 0, False, True),
    (12, 2, 64, "bf16", 16, 50.0, 3, True, True),
    (6, 1, 128, "fp16", 128, 0.0, 100, False, False),
    (4, 1, 64, "fp16", 16, 0.0, 0, True, True),
])
def test_prefill_of_few_tokens_matches_its_definition(mc, heads, kv, dim, dtype, page, softcap, window, bias, prefix):
    lens, new = [0, 5, 17, 64, 130, 300, 511, 3, 1025], [2, 5, 3, 1, 8, 4, 6, 7, 5]
    B = ref.Batch(lens, new, kv, page, dim, dtype, 16, pad_tokens=2)
    q = 1.5 * B.randn(B.tokens, heads, dim)
    sl = _slopes(heads) if bias else None
    pre = [1, 3, 17, 60, 125, 0, 600, 2, 1022] if prefix else None
    want = ref.attention(B, q, dim ** -0.5, softcap, window, sl, pre)
    cache, batch = B.device(mc)
    ws = mc.attn_workspace(cache, heads)
    out = torch.full((B.tokens, heads, dim), 3.0, dtype=ref.DT[dtype], device="cuda")
    got, lse = mc.attn_prefill(cache, batch, q.cuda(), softcap=softcap, window=window,
                               slopes=None if sl is None else sl.cuda(),
                               prefix=None if pre is None else torch.tensor(pre, dtype=torch.int32).cuda(),
                               out=out, with_lse=True, workspace=ws)
    mc.check_status(ws)
    n = B.cu[-1]
    assert (out[n:] == 3).all()
    ref.assert_attention(got, lse, want, dtype, 1025, 5.0, rows=slice(0, n))


@pytest.mark.parametrize("new,length,kv,heads,dim", [(1, 4000, 1, 4, 128), (5, 9000, 1, 5, 128), (40, 6000, 2, 4, 64), (700, 700, 1, 1, 128),
                                                     (515, 2100, 2, 6, 128), (1, 1, 1, 1, 64)])
def test_prefill_splits_and_joins(mc, new, length, kv, heads, dim):
    B = ref.Batch([length], [new], kv, 64, dim, "bf16", 8)
    q = B.randn(new, heads, dim)
    want = ref.attention(B, q, dim ** -0.5)
    cache, batch = B.device(mc)
    out, lse = mc.attn_prefill(cache, batch, q.cuda(), with_lse=True)
    ref.assert_attention(out, lse, want, "bf16", length, 5.0)
    again, _ = mc.attn_prefill(cache, batch, q.cuda(), with_lse=True)
    assert torch.equal(out, again)


@pytest.mark.parametrize("softcap,window", [(0.0, 0), (20.0, 60000)])
def test_prefill_of_a_chunk_over_a_cache_beyond_l2(mc, softcap, window):
    """A cache of 80 MB, read by several row tiles a head: the units are taken in another order."""
    B = ref.Batch([80000], [200], 2, 256, 128, "bf16", 17)
    q = B.randn(200, 8, 128)
    cache, batch = B.device(mc)
    out, lse = mc.attn_prefill(cache, batch, q.cuda(), softcap=softcap, window=window, with_lse=True)
    some = [0, 1, 63, 64, 130, 199]  # rows of every tile
    C = ref.Batch([80000], [200], 2, 256, 128, "bf16", 17)
    C.new, C.cu, want = [1], [0, 1], []
    for i in some:
        C.lens = [80000 - 200 + i + 1]
        want.append(ref.attention(C, q[i:i + 1], 128 ** -0.5, softcap, window))
    want = tuple(torch.cat(x) for x in zip(*want))
    ref.assert_attention(out[some], lse[some], want, "bf16", 80000, 5.0)


@pytest.mark.parametrize("seqs,heads,kv", [(45, 16, 1), (70, 40, 1)])
def test_prefill_of_many_sequences(mc, seqs, heads, kv):
    """More sequences than a warp has lanes, some without tokens, some without keys."""
    new = [(5 * b) % 23 for b in range(seqs)]
    lens = [0 if b % 11 == 4 else new[b] + (37 * b) % 300 for b in range(seqs)]
    B = ref.Batch(lens, new, kv, 16, 64, "bf16", 61, pad_tokens=1)
    q = B.randn(B.tokens, heads, 64)
    want = ref.attention(B, q, 0.125)
    cache, batch = B.device(mc)
    ws = mc.attn_workspace(cache, heads)
    out, lse = mc.attn_prefill(cache, batch, q.cuda(), with_lse=True, workspace=ws)
    mc.check_status(ws)
    ref.assert_attention(out, lse, want, "bf16", 400, 5.0, rows=slice(0, B.cu[-1]))
    # and the append of as many, then the same attention over what it wrote
    x = B.randn(3, B.tokens, kv, 64)
    full = ref.append(B, q, x[0], x[1])
    mc.kv_append(cache, batch, q.cuda(), x[0].cuda(), x[1].cuda(), workspace=ws)
    mc.check_status(ws)
    assert torch.equal(torch.nan_to_num(cache.k.double().cpu()), torch.nan_to_num(full[1]))
    assert torch.equal(torch.nan_to_num(cache.v.double().cpu()), torch.nan_to_num(full[2]))


@pytest.mark.parametrize("lens,new,heads,kv,dim,dtype,window,cap", [
    ([4096], [4096], 32, 8, 128, "bf16", 0, 0.0),
    ([3001, 40, 0, 2500, 3700, 1], [3001, 9, 0, 2300, 3600, 1], 12, 4, 64, "fp16", 0, 20.0),  # items of five sequences
    ([5000] + [700] * 31, [5000] + [300] * 31, 16, 4, 64, "bf16", 900, 0.0),                 # as many as a queue takes
    ([4000] + [100] * 32, [4000] + [100] * 32, 16, 4, 64, "bf16", 0, 0.0),                   # one more: runs
])
def test_prefill_of_long_prompts(mc, lens, new, heads, kv, dim, dtype, window, cap):
    """Batches of many items, a part of the rows against the definition; twice over, bit for bit."""
    B = ref.Batch(lens, new, kv, 64, dim, dtype, 61, pad_tokens=2)
    q = B.randn(B.tokens, heads, dim)
    cache, batch = B.device(mc)
    ws = mc.attn_workspace(cache, heads)
    slopes = -torch.linspace(0.1, 0.01, heads) if cap else None
    kw = dict(softcap=cap, window=window, slopes=None if slopes is None else slopes.cuda(), workspace=ws)
    got, lse = mc.attn_prefill(cache, batch, q.cuda(), with_lse=True, **kw)
    again = torch.full_like(got, 3.0)
    mc.attn_prefill(cache, batch, q.cuda(), out=again, **kw)
    mc.check_status(ws)
    assert torch.equal(got[:B.cu[-1]], again[:B.cu[-1]])
    g = torch.Generator().manual_seed(62)
    for b, (n, length) in enumerate(zip(new, lens)):
        if not n or (4 < b < len(lens) - 2):
            continue
        toks = sorted({0, n - 1, n // 2} | {int(i) for i in torch.randint(0, n, (6,), generator=g)})
        for i in toks:  # one new token at the end of a shorter sequence, the same cache
            p = length - n + i
            one = ref.Batch.__new__(ref.Batch)
            one.__dict__.update(B.__dict__, lens=[p + 1], new=[1], cu=[0, 1], table=B.table[b:b + 1], tokens=1)
            t = B.cu[b] + i
            want = ref.attention(one, q[t:t + 1], dim ** -0.5, cap, window, slopes)
            ref.assert_attention(got[t:t + 1], lse[t:t + 1], want, dtype, length, 5.0)


def test_prefill_of_one_token_each_is_decode(mc):
    """The same rows through both entry points, each within its bound of the other's sums."""
    B = ref.Batch(EDGES, [1] * len(EDGES), 2, 16, 128, "bf16", 15)
    q = B.randn(len(EDGES), 8, 128)
    cache, batch = B.device(mc, cu=False)
    d, dl = mc.attn_decode(cache, batch, q.cuda(), with_lse=True)
    p, pl = mc.attn_prefill(cache, batch, q.cuda(), with_lse=True)
    assert (d.float() - p.float()).abs().max() <= 4 * 2.0 ** -9 * 5
    assert torch.allclose(dl, pl, rtol=1e-4, atol=1e-4)


@pytest.mark.parametrize("dim,dtype,cap,lens,new,window", [(128, "bf16", 50.0, [900, 2, 1, 3000], [1] * 4, 2), (64, "fp16", 50.0, [1, 2, 3, 5, 8, 64], [1] * 6, 0),
                                                           (128, "bf16", 30.0, [4, 3, 70], [4, 2, 3], 3)])
def test_caps_over_few_keys(mc, dim, dtype, cap, lens, new, window):
    """With few keys the errors of their scores do not average out: lse to 8 roundings of fp32 (2^-24) of itself or
    of the largest uncapped term, scores of a few units (products of 128 terms: 16 roundings of those)."""
    B = ref.Batch(lens, new, 2, 16, dim, dtype, 71)
    q = B.randn(B.tokens, 6, dim)
    want = ref.attention(B, q, dim ** -0.5, cap, window)
    cache, batch = B.device(mc)
    out, lse = mc.attn_prefill(cache, batch, q.cuda(), softcap=cap, window=window, with_lse=True)
    ref.assert_attention(out, lse, want, dtype, 3000, 5.0)
    assert ((lse.double().cpu() - want[1]).abs() <= 24 * 2.0 ** -24 * (1 + want[1].abs())).all()


@pytest.mark.parametrize("dim,dtype,cap,spread", [(128, "bf16", 2.0, 1.0), (64, "fp16", 0.5, 3.0), (128, "fp16", 40.0, 1.5), (64, "bf16", 8.0, 2.0)])
def test_caps_far_below_and_around_the_scores(mc, dim, dtype, cap, spread):
    """Scores from a fraction of the cap to many times it: both of the cap's forms, in every kernel."""
    for lens, new in (([200, 515], [1, 1]), ([200, 515], [7, 3]), ([260, 300], [260, 130])):
        B = ref.Batch(lens, new, 2, 32, dim, dtype, 31)
        q = spread * B.randn(B.tokens, 8, dim)
        q[0] *= 0.01
        want = ref.attention(B, q, dim ** -0.5, cap)
        cache, batch = B.device(mc)
        out, lse = mc.attn_prefill(cache, batch, q.cuda(), softcap=cap, with_lse=True)
        ref.assert_attention(out, lse, want, dtype, 520, 5.0)


@pytest.mark.parametrize("cap", [50.0, 1e3, 1e5, 1e8, 1e18])
@pytest.mark.parametrize("dim,dtype,lens,new", [(128, "bf16", [500, 2, 131], [1, 1, 1]), (64, "fp16", [300, 90], [4, 2]),  # few rows a sequence
                                                (128, "fp16", [150, 400], [150, 60]), (64, "bf16", [140, 300], [140, 80])])
def test_caps_far_above_the_scores(mc, dim, dtype, cap, lens, new):
    """A cap far above the scores leaves them as they are, whatever its size, in either kernel and
    for rows of few keys and of many.  Bound on lse: its sums and products as in the caps over few
    keys, 24 roundings of fp32, and 8 more for the cap of each score (its form's error)."""
    B = ref.Batch(lens, new, 2, 16, dim, dtype, 91)
    q = B.randn(B.tokens, 12, dim)
    want = ref.attention(B, q, dim ** -0.5, cap)
    cache, batch = B.device(mc)
    ws = mc.attn_workspace(cache, 12)
    out, lse = mc.attn_prefill(cache, batch, q.cuda(), softcap=cap, with_lse=True, workspace=ws)
    mc.check_status(ws)
    ref.assert_attention(out, lse, want, dtype, 500, 5.0)
    assert ((lse.double().cpu() - want[1]).abs() <= 32 * 2.0 ** -24 * (1 + want[1].abs())).all()


@pytest.mark.parametrize("dim,dtype,lens,new,heads,kv,window", [
    (128, "bf16", [40, 300], [6, 3], 4, 2, 0),         # few rows: decode kernel
    (64, "fp16", [9000], [5], 2, 1, 100),              # the same, over pages that a window has left behind
    (64, "bf16", [9000], [5], 2, 1, 0),                # the same, split and joined
    (128, "bf16", [300, 130], [200, 130], 4, 2, 0),    # many rows
    (64, "fp16", [300, 700], [300, 64], 3, 1, 40),
    (128, "fp16", [5000], [100], 2, 1, 0),             # many rows, split and joined
])
def test_hidden_infinities_and_nan_stay_hidden(mc, dim, dtype, lens, new, heads, kv, window):
    """NaN and infinities in keys and values that some queries see and others do not: rows that
    do not see them are as if they were zero, rows that do are what the definition makes of them."""
    B = ref.Batch(lens, new, kv, 16, dim, dtype, 41)
    q = B.randn(B.tokens, heads, dim)
    planted = []
    for b, (n, length) in enumerate(zip(new, lens)):
        for at, what, col in ((length - 1, float("nan"), 3), (length - 2, float("inf"), 7)):
            B.v[B.table[b, at // 16], :, at % 16, col] = what
            planted.append((b, at, col, what))
        if window:  # a key that the window has left behind (the batch that starts at 0: seen by its first queries)
            B.v[B.table[b, 0], :, 0, :] = float("nan")
            B.k[B.table[b, 0], :, 0, :] = float("nan")
    want = ref.attention(B, q, dim ** -0.5, window=window)
    cache, batch = B.device(mc)
    ws = mc.attn_workspace(cache, heads)
    got, lse = mc.attn_prefill(cache, batch, q.cuda(), window=window, with_lse=True, workspace=ws)
    mc.check_status(ws)
    got = got.double().cpu()
    odd = ~torch.isfinite(want[0])
    assert odd.any() and torch.equal(torch.isnan(got), torch.isnan(want[0]))
    assert torch.equal(got[odd & ~torch.isnan(got)], want[0][odd & ~torch.isnan(got)])
    h = ref.HALF_ULP[dtype]
    tol = (2 * h + 1e-4) * torch.nan_to_num(want[2], posinf=0) + 1e-30 + (2.0 ** -24 + max(lens) * 2.0 ** -25 * 5 if dtype == "fp16" else 0)
    assert ((got - want[0]).abs() <= tol)[~odd].all()
    assert torch.allclose(lse.double().cpu(), want[1], rtol=1e-4, atol=1e-4, equal_nan=True)


@pytest.mark.parametrize("dim,dtype,length,new,heads,window", [(128, "bf16", 300, 3, 2, 0), (64, "fp16", 9000, 5, 2, 0), (128, "fp16", 300, 100, 4, 0),
                                                               (64, "bf16", 6000, 100, 2, 5950)])
def test_a_visible_score_of_minus_infinity_weighs_nothing(mc, dim, dtype, length, new, heads, window):
    """The first keys that a row sees score -inf, and a key that all but the last row do not see
    has an infinite value."""
    B = ref.Batch([length], [new], 1, 16, dim, dtype, 43)
    first = max(0, length - new - window + 1) if window else 0
    for j in range(first, first + 2):
        B.k[B.table[0, j // 16], 0, j % 16, 0] = -float("inf")
    B.v[B.table[0, (length - 1) // 16], 0, (length - 1) % 16, 5] = float("inf")
    q = B.randn(new, heads, dim)
    q[:, :, 0] = q[:, :, 0].abs() + 0.25
    want = ref.attention(B, q, dim ** -0.5, window=window)
    cache, batch = B.device(mc)
    got, lse = mc.attn_prefill(cache, batch, q.cuda(), window=window, with_lse=True)
    rows = torch.arange(new - 1)
    ref.assert_attention(got, lse, want, dtype, length, 5.0, rows=rows)


# ------------------------------------------- both kernels, by the mean of rows --
# A sequence's new tokens times its group are its rows; with a mean of up to 16 (32 under a cap) the
# batch takes the kernel for few rows, beyond that the tensor-memory one.

@pytest.mark.parametrize("heads,kv,dim,dtype,cap", [(8, 2, 128, "bf16", 0.0), (6, 2, 64, "fp16", 0.0), (8, 2, 128, "bf16", 30.0)])
def test_one_token_each_through_either_kernel(mc, heads, kv, dim, dtype, cap):
    """The same single tokens alone and beside a prompt that takes the batch over the limit."""
    B = ref.Batch(EDGES + [900], [1] * len(EDGES) + [900], kv, 16, dim, dtype, 101)
    n = len(EDGES)
    q = B.randn(B.tokens, heads, dim)
    want = ref.attention(B, q, dim ** -0.5, cap)
    cache, batch = B.device(mc)
    mixed, mixed_lse = mc.attn_prefill(cache, batch, q.cuda(), softcap=cap, with_lse=True)
    assert (n + 900) * (heads // kv) / (n + 1) > 32
    ref.assert_attention(mixed, mixed_lse, want, dtype, 900, 5.0)
    one = mc.KVBatch(batch._keep[0][:n].contiguous(), batch._keep[1][:n].contiguous())
    for call in (mc.attn_decode, mc.attn_prefill):
        alone, lse = call(cache, one, q[:n].cuda(), softcap=cap, with_lse=True)
        ref.assert_attention(alone, lse, tuple(w[:n] for w in want), dtype, 900, 5.0)


@pytest.mark.parametrize("dtype,window,prefix", [("bf16", 0, False), ("fp16", 90, False), ("bf16", 0, True)])
def test_a_long_prompt_through_the_kernel_for_few_rows(mc, dtype, window, prefix):
    """Many slots with a token or none bring the mean down: the prompt's rows are many slices."""
    lens, new = [650] + [0, 40, 7] * 20, [600] + [0, 1, 1] * 20
    B = ref.Batch(lens, new, 1, 32, 64, dtype, 103, pad_tokens=1)
    assert B.tokens / len(lens) <= 16
    q = B.randn(B.tokens, 1, 64)
    pre = [300] + [0] * 60 if prefix else None
    want = ref.attention(B, q, 0.125, window=window, prefix=pre)
    cache, batch = B.device(mc)
    ws = mc.attn_workspace(cache, 1)
    out, lse = mc.attn_prefill(cache, batch, q.cuda(), window=window, with_lse=True, workspace=ws,
                               prefix=None if pre is None else torch.tensor(pre, dtype=torch.int32).cuda())
    mc.check_status(ws)
    ref.assert_attention(out, lse, want, dtype, 650, 5.0, rows=slice(0, B.cu[-1]))


@pytest.mark.parametrize("new", [[2, 3, 1], [200, 131, 60]])  # few rows, many rows
@pytest.mark.parametrize("heads,kv,dim,dtype", [(4, 1, 128, "bf16"), (3, 1, 64, "fp16"), (10, 2, 128, "fp16"), (14, 2, 64, "bf16"),
                                                (24, 1, 128, "bf16"), (17, 1, 64, "bf16")])
def test_queries_and_outputs_with_a_token_stride(mc, new, heads, kv, dim, dtype):
    """Queries as a slice of the projection's output, for groups that divide a tile and others; outputs
    whose rows start at multiples of 16 bytes but not of 32."""
    B = ref.Batch([260, 400, 61], new, kv, 16, dim, dtype, 107, pad_tokens=1)
    wide = B.randn(B.tokens, (heads + 2 * kv) * dim + 8)
    q = wide[:, 8:8 + heads * dim].unflatten(1, (heads, dim))
    want = ref.attention(B, q, dim ** -0.5)
    cache, batch = B.device(mc)
    ws = mc.attn_workspace(cache, heads)
    dev = wide.cuda()[:, 8:8 + heads * dim].unflatten(1, (heads, dim))
    buf = torch.full((B.tokens, heads * dim + 8), 3.0, dtype=ref.DT[dtype], device="cuda")
    out = buf[:, :heads * dim].unflatten(1, (heads, dim))
    got, lse = mc.attn_prefill(cache, batch, dev, out=out, with_lse=True, workspace=ws)
    mc.check_status(ws)
    assert (buf[:, heads * dim:] == 3).all() and (buf[B.cu[-1]:] == 3).all()
    ref.assert_attention(got, lse, want, dtype, 400, 5.0, rows=slice(0, B.cu[-1]))


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("new", [[2, 1, 3], [50, 70, 130]])  # few rows, many rows
def test_pages_lengths_and_boundaries_that_are_not_sound(mc, new, cap):
    """In either kernel: a page outside the pool reads as zeros, a length is cut to the table's rows, a
    sequence whose boundaries are not sound has no tokens; each is recorded, and the other sequences
    are right."""
    lens, heads, kv, dim = [96, 160, 144], 8, 2, 64
    ok = ref.Batch(lens, new, kv, 16, dim, "bf16", 109)
    q = ok.randn(ok.tokens, heads, dim)
    cache, batch = ok.device(mc)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731

    def attend(b):
        ws = mc.attn_workspace(cache, heads)
        out = torch.full((ok.tokens, heads, dim), 3.0, dtype=torch.bfloat16, device="cuda")
        _, lse = mc.attn_prefill(cache, b, q.cuda(), softcap=cap, out=out, with_lse=True, workspace=ws)
        return out, lse, ws

    def reported(ws):
        with pytest.raises(mc.MCError) as e:
            mc.check_status(ws)
        assert e.value.code == mc.ERR_RANGE

    want = ref.attention(ok, q, dim ** -0.5, cap)
    good, good_lse, ws = attend(batch)
    mc.check_status(ws)
    ref.assert_attention(good, good_lse, want, "bf16", 160, 5.0)

    for page in (ok.k.shape[0], -1, 2 ** 31 - 1, -2 ** 31):  # of sequence 1's keys 32 .. 47
        table = ok.table.clone()
        table[1, 2] = page
        out, lse, ws = attend(mc.KVBatch(batch._keep[0], table.cuda(), batch._keep[2], ok.tokens))
        reported(ws)
        zero = ref.Batch(lens, new, kv, 16, dim, "bf16", 109)
        zero.k[zero.table[1, 2].long()] = 0
        zero.v[zero.table[1, 2].long()] = 0
        ref.assert_attention(out, lse, ref.attention(zero, q, dim ** -0.5, cap), "bf16", 160, 5.0)
        others = [t for t in range(ok.tokens) if not ok.cu[1] <= t < ok.cu[2]]
        assert torch.equal(out[others], good[others])

    for length in (161, 1 << 20, 2 ** 31 - 1):
        out, lse, ws = attend(mc.KVBatch(i32([96, length, 144]), batch._keep[1], batch._keep[2], ok.tokens))
        reported(ws)
        ref.assert_attention(out, lse, want, "bf16", 160, 5.0)  # (the table has pages for 160 rows)

    # (in the first, sequence 2 claims every row, those of sequence 0 too: none is anybody's alone)
    for cu, sound in (([0, ok.cu[1], 0, ok.cu[3]], []), ([0, ok.cu[1], ok.tokens + 1, ok.tokens + 1], [0]),
                      ([-1, ok.cu[1], ok.cu[2], ok.cu[3]], [1, 2]), ([0, ok.cu[1], ok.cu[2], ok.cu[2] - 1], [0, 1])):
        out, lse, ws = attend(mc.KVBatch(batch._keep[0], batch._keep[1], i32(cu), ok.tokens))
        reported(ws)
        for b in sound:
            t = slice(ok.cu[b], ok.cu[b + 1])
            ref.assert_attention(out[t], lse[t], tuple(w[t] for w in want), "bf16", 160, 5.0)
        if sound == [1, 2]:
            assert (out[:ok.cu[1]] == 3).all()


# ----------------------------------------------------------- streams, status --

def test_on_another_stream_and_in_a_graph(mc):
    B = ref.Batch([40, 130, 7], [1] * 3, 2, 16, 64, "bf16", 21)
    cache, batch = B.device(mc, cu=False)
    q, k, v = (B.randn(3, n, 64).cuda() for n in (8, 2, 2))
    rope = ref.rope_table(200, 64).cuda()
    ws = mc.attn_workspace(cache, 8)

    def step():
        return mc.attn_decode(cache, batch, mc.kv_append(cache, batch, q, k, v, rope=rope, workspace=ws), workspace=ws)

    want = step().clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = step()
    s.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        res = step()
    res.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(res, want)


def test_pages_behind_the_window_may_be_gone(mc):
    """Their table entries are not read and their rows not looked at."""
    for new, heads, cap in ((1, 4, 0.0), (4, 4, 0.0), (1, 32, 0.0), (150, 4, 0.0), (150, 4, 20.0)):
        B = ref.Batch([700, 333], [new, new], 2, 16, 64, "bf16", 51)
        q = B.randn(B.tokens, heads, 64)
        want = ref.attention(B, q, 0.125, cap, 100)
        for b, length in enumerate(B.lens):
            gone = max(0, length - new - 100 + 1) // 16
            B.v[B.table[b, :gone].long()] = float("nan")
            B.k[B.table[b, :gone].long()] = float("nan")
            B.table[b, :gone] = -1
        cache, batch = B.device(mc)
        ws = mc.attn_workspace(cache, heads)
        out, lse = mc.attn_prefill(cache, batch, q.cuda(), softcap=cap, window=100, with_lse=True, workspace=ws)
        mc.check_status(ws)
        ref.assert_attention(out, lse, want, "bf16", 700, 5.0)


def test_bad_pages_lengths_and_positions_are_reported(mc):
    """What only the device can see is bounded there and reported, and the next call works."""
    B = ref.Batch([40, 64], [1, 1], 2, 16, 64, "bf16", 22)
    cache, batch = B.device(mc, cu=False)
    q, k, v = (B.randn(2, n, 64).cuda() for n in (4, 2, 2))
    ws = mc.attn_workspace(cache, 4)
    good = mc.attn_decode(cache, batch, q, workspace=ws)
    mc.check_status(ws)
    bad = B.table.clone()
    bad[0, 1] = cache.k.shape[0]
    cases = [mc.KVBatch(batch._keep[0], bad.cuda()), mc.KVBatch(torch.tensor([40, 1 << 20], dtype=torch.int32).cuda(), B.table.cuda())]
    for other in cases:
        for call in (mc.attn_decode, mc.attn_prefill):
            out = call(cache, other, q, workspace=ws)
            with pytest.raises(mc.MCError) as e:
                mc.check_status(ws)
            assert e.value.code == mc.ERR_RANGE
            assert torch.equal(out[1], good[1]) or other is cases[1] or call is mc.attn_prefill
    before = cache.k.clone()
    bad[0, 2] = -1  # the page of the new token of sequence 0
    mc.kv_append(cache, mc.KVBatch(batch._keep[0], bad.cuda()), q, k, v, workspace=ws)
    with pytest.raises(mc.MCError):
        mc.check_status(ws)
    changed = (torch.nan_to_num(cache.k.float()) != torch.nan_to_num(before.float())).flatten(1).any(1).nonzero().flatten()
    assert changed.tolist() == [int(B.table[1, 3])]
    mc.kv_append(cache, batch, q, k, v, rope=ref.rope_table(10, 64).cuda(), workspace=ws)  # positions past the table
    with pytest.raises(mc.MCError):
        mc.check_status(ws)
    cu = torch.tensor([0, 3, 2], dtype=torch.int32).cuda()
    mc.attn_prefill(cache, mc.KVBatch(batch._keep[0], batch._keep[1], cu, 2), q, workspace=ws)
    with pytest.raises(mc.MCError):
        mc.check_status(ws)
    mc.attn_decode(cache, batch, q, workspace=ws)
    mc.check_status(ws)


@pytest.mark.parametrize("many", [False, True])
def test_a_descending_cu_q_stays_within_the_tables(mc, many):
    """A token that no sequence's rows hold is appended nowhere: not past its sequence's
    length either, which the row after the last one's page list would be read for."""
    seqs = 40 if many else 3
    B = ref.Batch([32] * seqs, [1] * seqs, 2, 16, 64, "fp16", 24)
    table = torch.cat([B.table, B.table[:1]])  # (what lies behind the last row here names a page)
    table[seqs] = min(set(range(len(B.k))) - {int(i) for i in B.table.flatten()})
    cu = torch.tensor([0, 9, 1, 2] + [2] * (seqs - 3), dtype=torch.int32).cuda()
    B.k.zero_(), B.v.zero_()
    cache, _ = B.device(mc)
    batch = mc.KVBatch(torch.tensor(B.lens, dtype=torch.int32).cuda(), table.cuda()[:seqs], cu, 9)
    q, k, v = (B.randn(9, n, 64).cuda() for n in (4, 2, 2))
    ws = mc.attn_workspace(cache, 4)
    mc.kv_append(cache, batch, q, k, v, workspace=ws)
    with pytest.raises(mc.MCError):
        mc.check_status(ws)
    written = {int(i) for i in (cache.k.flatten(1) != 0).any(1).nonzero().flatten()}
    assert written <= {int(i) for i in B.table.flatten()}


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("new,over", [([1, 1], 1), ([1, 1], 40), ([5, 3], 2), ([5, 3], 30)])
def test_an_overlong_length_moves_no_token(mc, new, over, many):
    """A length past the page table's rows: the tokens that its pages hold go where that length
    puts them, the others nowhere, and no row of another token is touched."""
    fill = 40 if many else 0  # (idle slots: more sequences than a warp looks at at once)
    B = ref.Batch([64, 40] + [0] * fill, new + [0 if sum(new) > 2 else 1] * fill, 2, 16, 64, "bf16", 26)
    cache, _ = B.device(mc)
    ragged = sum(new) > 2
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    batch = mc.KVBatch(i32([64 + over, 40] + [0] * fill), B.table.cuda(), i32(B.cu) if ragged else None, B.tokens if ragged else None)
    q, k, v = (B.randn(B.tokens, n, 64) for n in (4, 2, 2))
    ws = mc.attn_workspace(cache, 4)
    got = mc.kv_append(cache, batch, q.cuda(), k.cuda(), v.cuda(), workspace=ws)
    with pytest.raises(mc.MCError) as e:
        mc.check_status(ws)
    assert e.value.code == mc.ERR_RANGE
    want_k, want_v, want_q = B.k.clone(), B.v.clone(), torch.zeros_like(q)
    for b, (n, length) in enumerate(zip(B.new, [64 + over, 40] + [0] * fill)):
        for i in range(n):
            pos, t = length - n + i, B.cu[b] + i
            if 0 <= pos < 64:
                page, row = int(B.table[b, pos // 16]), pos % 16
                want_k[page, :, row], want_v[page, :, row], want_q[t] = k[t], v[t], q[t]
    for a, w in ((cache.k, want_k), (cache.v, want_v), (got, want_q)):
        assert torch.equal(a.cpu().view(torch.int16), w.view(torch.int16))


@pytest.mark.parametrize("seqs,new,length,kv,heads", [(90, 64, 2000, 2, 8), (2, 3000, 3000, 8, 16)])  # runs, and a queue
def test_rows_redone_do_not_hold_the_others_up(mc, seqs, new, length, kv, heads):
    """A value that only a sequence's last token sees is infinite: the rows that share its units are
    redone, which takes far longer than a wait of the pipeline may last, here 3 ms.  Against the same
    batch with a zero there: each side is within 2 * 2^-8 + 1e-4 of the mean |v|, which is below 5, and
    lse within 1e-4."""
    B = ref.Batch([length] * seqs, [new] * seqs, kv, 64, 64, "bf16", 81)
    q = B.randn(B.tokens, heads, 64).cuda()
    ws = None
    got = []
    for what in (0.0, float("inf")):
        for b in range(0, seqs, 2):
            B.v[B.table[b, (length - 1) // 64], :, (length - 1) % 64, 9] = what
        cache, batch = B.device(mc)
        ws = mc.attn_workspace(cache, heads) if ws is None else ws
        mc.set_debug(0, 3_000_000)
        try:
            out, lse = mc.attn_prefill(cache, batch, q, out=torch.full_like(q, 100.0), with_lse=True, workspace=ws)
            mc.check_status(ws)
        finally:
            mc.set_debug(0, 1_000_000_000)
        got.append((out.float().view(seqs, new, heads, 64), lse.view(seqs, new, heads)))
    (want, want_lse), (out, lse) = got
    assert torch.isposinf(out[0::2, -1, :, 9]).all()
    out[0::2, -1, :, 9] = want[0::2, -1, :, 9] = 0
    assert torch.isfinite(out).all()
    assert ((out - want).abs() <= 2 * (2 * 2.0 ** -8 + 1e-4) * 5).all()
    assert torch.allclose(lse, want_lse, rtol=2e-4, atol=2e-4)


@pytest.mark.parametrize("seqs,new,length,heads,kv", [(1, 4096, 4096, 16, 4),   # whole items
                                                      (1, 300, 9000, 8, 2),     # split and joined
                                                      (16, 4, 4000, 16, 4)])    # few rows a sequence
def test_a_visible_nan_costs_little(mc, seqs, new, length, heads, kv):
    """A NaN that every row sees: their results are NaN there as they come, none is redone key by
    key.  (Ten times a finite call's time; redone, it is a hundred times and more.)"""
    B = ref.Batch([length] * seqs, [new] * seqs, kv, 64, 128, "bf16", 83)
    q = B.randn(B.tokens, heads, 128).cuda()
    ws, took, got = None, [], []
    for what in (0.0, float("nan")):
        for b in range(seqs):
            B.v[B.table[b, 0], :, 0, 3] = what
        cache, batch = B.device(mc)
        ws = mc.attn_workspace(cache, heads) if ws is None else ws
        out = torch.full_like(q, 100.0)
        call = lambda: mc.attn_prefill(cache, batch, q, out=out, workspace=ws)  # noqa: E731
        for _ in range(3):
            call()
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        for _ in range(10):
            call()
        end.record()
        mc.check_status(ws)
        torch.cuda.synchronize()
        took.append(start.elapsed_time(end) / 10)
        got.append(out)
    assert torch.isnan(got[1][..., 3]).all()
    got[1][..., 3] = got[0][..., 3]
    assert torch.equal(got[0], got[1])
    assert took[1] <= 10 * took[0], took


def test_prefill_waits_expire_and_the_context_lives(mc):
    """With the copies switched off every wait of the kernel reaches its bound."""
    B = ref.Batch([300], [300], 1, 16, 64, "bf16", 23)
    cache, batch = B.device(mc)
    q = B.randn(300, 4, 64).cuda()
    ws = mc.attn_workspace(cache, 4)
    want = mc.attn_prefill(cache, batch, q, workspace=ws)
    mc.check_status(ws)
    mc.set_debug(1, 20_000_000)
    try:
        mc.attn_prefill(cache, batch, q, workspace=ws)
        with pytest.raises(mc.MCError) as e:
            mc.check_status(ws)
        assert e.value.code == mc.ERR_TIMEOUT
    finally:
        mc.set_debug(0, 1_000_000_000)
    assert torch.equal(mc.attn_prefill(cache, batch, q, workspace=ws), want)
    mc.check_status(ws)
