"""The 4-bit cache's append, its rows read back and the two attentions over it against their definitions: bytes
of blocks, head layouts, types, page sizes, lengths around every tile's edges, masks, groups of NaN, unsound pages,
strides, streams and graphs.  What the cache stands for is exact in its type, so the attentions' bounds are those of
the 16-bit cache's."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import attn_ref as ref  # noqa: E402
import kv4_ref as ref4  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=["room for prompts", "no room"])
def mc(request):
    """Every test with a workspace in which long prompts' keys are unpacked, and with one without."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2410_06270_gb300 import build
    build.build()
    import paper_2410_06270_gb300 as m
    m.load()
    m.set_debug(0, 1_000_000_000)
    patch = pytest.MonkeyPatch()
    whole = m.attn4_workspace
    patch.setattr(m, "attn4_workspace", lambda cache, heads, prompts=request.param == "room for prompts": whole(cache, heads, prompts))
    yield m
    patch.undo()


EDGES = [0, 1, 2, 15, 16, 17, 31, 63, 64, 65, 100, 127, 128, 129, 255, 257, 700]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _slopes(heads):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)])


def _reported(mc, ws):
    with pytest.raises(mc.MCError) as e:
        mc.check_status(ws)
    assert e.value.code == mc.ERR_RANGE


# ---------------------------------------------------------------- append --

APPEND = [
    # heads, kv, dim, dtype, page, rot, interleaved, norm, ragged
    (9, 3, 128, "bf16", 16, 128, False, False, False),
    (12, 4, 64, "fp16", 48, 32, True, True, True),
    (5, 1, 128, "bf16", 64, 64, False, True, True),
    (3, 3, 64, "bf16", 16, 64, False, False, True),
    (7, 7, 128, "fp16", 32, 96, False, False, False),
    (4, 2, 128, "fp16", 128, 0, False, True, True),
    (1, 1, 64, "bf16", 16, 16, False, True, False),
    (9, 9, 128, "bf16", 16, 0, False, False, True),
    (2, 2, 64, "fp16", 16, 0, False, False, False),
    (2, 1, 128, "bf16", 32, 128, True, True, True),
]


@pytest.mark.parametrize("heads,kv,dim,dtype,page,rot,interleaved,norm,ragged", APPEND)
def test_append_stores_what_the_definition_says(mc, heads, kv, dim, dtype, page, rot, interleaved, norm, ragged):
    """The queries are kv_append's; a stored row is, byte for byte, the grid of the row that kv_append
    writes (rounded to the type); every other byte is left alone; and what is read back stands for it."""
    lens = [0, 1, page, page + 1, 100, 5 * page - 1, 3]
    new = [0, 1, page, 2, 60, 33, 5] if ragged else [1] * len(lens)  # the last: more new tokens than its length
    B = ref.Batch(lens, new, kv, page, dim, dtype, 11, pad_tokens=3 if ragged else 0)
    T = ref.DT[dtype]
    wide = B.randn(B.tokens, (heads + 2 * kv) * dim + 8)  # a row's tail is not the call's
    wide[:, (heads + kv) * dim:] *= 3
    cut = lambda x, a, n: x[:, a * dim:(a + n) * dim].unflatten(1, (n, dim))  # noqa: E731
    qn, kn = ((1 + 0.1 * B.randn(dim)).to(T).cuda() for _ in range(2)) if norm else (None, None)
    rope = ref.rope_table(600, rot).cuda() if rot else None
    dev = wide.cuda()
    parts = [cut(dev, 0, heads), cut(dev, heads, kv), cut(dev, heads + kv, kv)]
    kw = dict(rope=rope, interleaved=interleaved, q_norm=qn, k_norm=kn)
    cache16, batch = B.device(mc, cu=ragged)
    q16 = mc.kv_append(cache16, batch, *parts, **kw)

    size = mc.kv4_block_size(page, dim)
    assert size == page * 17 * dim // 32
    before = torch.randint(0, 256, (2, B.k.shape[0], kv, size), generator=B.g, dtype=torch.uint8)
    pools = before.cuda()
    cache = mc.KVCache4(pools[0], pools[1], page, dim, T)
    ws = mc.attn4_workspace(cache, heads)
    q_out = torch.full((B.tokens, heads, dim), 7.0, dtype=T, device="cuda")
    q = mc.kv4_append(cache, batch, *parts, q_out=q_out, workspace=ws, **kw)
    mc.check_status(ws)
    n = B.cu[-1]
    assert q.data_ptr() == q_out.data_ptr() and (q[n:] == 7).all()
    assert torch.equal(q[:n], q16[:n])
    want = before.numpy().copy()
    stands = torch.zeros(2, B.tokens, kv, dim, dtype=torch.float64)
    for side, c in enumerate((cache16.k.cpu(), cache16.v.cpu())):
        for b, (m, length) in enumerate(zip(B.new, B.lens)):
            for i in range(m):
                pos = length - m + i
                if pos < 0:
                    continue
                p, row = int(B.table[b, pos // page]), pos % page
                for h in range(kv):
                    codes, words, x = ref4.store(c[p, h, row], dtype)
                    want[side, p, h, row * dim // 2:(row + 1) * dim // 2] = np.frombuffer(codes, np.uint8)
                    at = page * dim // 2 + row * dim // 32
                    want[side, p, h, at:at + dim // 32] = np.frombuffer(words, np.uint8)
                    stands[side, B.cu[b] + i, h] = x
    assert np.array_equal(pools.cpu().numpy(), want)
    k, v = (torch.full((B.tokens, kv, dim), 5.0, dtype=T, device="cuda") for _ in range(2))
    k2, v2 = mc.kv4_read(cache, batch, k=k, v=v, workspace=ws)
    mc.check_status(ws)
    assert k2.data_ptr() == k.data_ptr() and (k[n:] == 5).all() and (v[n:] == 5).all()
    assert torch.equal(k[:n].double().cpu(), stands[0, :n]) and torch.equal(v[:n].double().cpu(), stands[1, :n])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_at_the_ends_of_the_type(mc, dtype):
    """Groups of zeros, of the largest and the smallest numbers, constants, outliers, halves between codes, and
    groups that are not finite: byte for byte, and read back."""
    T = ref.DT[dtype]
    top = torch.finfo(T).max
    g = torch.Generator().manual_seed(5)
    rows = [torch.zeros(64), torch.full((64,), top), torch.full((64,), -top), torch.cat([torch.full((32,), top), torch.full((32,), -top)]),
            torch.cat([torch.full((32,), top * 0.992), torch.full((32,), -top * 0.12)]), torch.full((64,), 2.0 ** -24), torch.full((64,), -0.0),
            torch.full((64,), 1.0), torch.full((64,), -7.5), torch.arange(64) - 20.0, (torch.arange(64) % 16) * 0.5,
            (torch.arange(64) % 31) * 0.25 - 3.75]
    for e in range(-30 if dtype == "bf16" else -18, 14, 1):
        x = torch.randn(64, generator=g)
        x[e % 64] *= 50
        rows.append((x * 2.0 ** e).clamp(-top, top))
    for bad in (float("inf"), -float("inf"), float("nan")):
        x = torch.randn(64, generator=g)
        x[9] = bad
        rows.append(x)
    while len(rows) % 8:
        rows.append(torch.randn(64, generator=g))
    x = torch.stack(rows).to(T)  # a group each; two heads of 128 a token
    tokens = x.shape[0] // 4
    kv = x.view(tokens, 2, 128)
    page, pages = 16, -(-tokens // 16)
    pools = torch.zeros(2, pages, 2, mc.kv4_block_size(page, 128), dtype=torch.uint8, device="cuda")
    cache = mc.KVCache4(pools[0], pools[1], page, 128, T)
    batch = mc.KVBatch(_i32([tokens]), torch.arange(pages, dtype=torch.int32).cuda()[None], _i32([0, tokens]), tokens)
    dev = kv.cuda()
    mc.kv4_append(cache, batch, dev, dev, -dev)
    k, v = mc.kv4_read(cache, batch)
    for side, src, got in ((0, kv, k), (1, -kv, v)):
        for t in range(tokens):
            for h in range(2):
                codes, words, stands = ref4.store(src[t, h], dtype)
                block = pools[side, t // page, h].cpu().numpy()
                r = t % page
                finite = np.isfinite(stands.numpy())
                have = block[page * 64 + r * 4:page * 64 + r * 4 + 4].tobytes()
                for grp in range(2):
                    if finite[64 * grp]:
                        assert have[2 * grp:2 * grp + 2] == words[2 * grp:2 * grp + 2]
                assert torch.equal(got[t, h].double().cpu().nan_to_num(1e30), stands.nan_to_num(1e30))
                if finite.all():
                    assert block[r * 64:r * 64 + 64].tobytes() == codes


def test_append_in_place_and_long_offsets(mc):
    """q_out may be q; pages far into a strided pool lie past 2^32 bytes."""
    B = ref.Batch([70], [70], 2, 64, 64, "bf16", 3, spare=0)
    stride, size = (1 << 32) + 4096, 64 * 34
    big = torch.zeros(stride + (1 << 20), dtype=torch.uint8, device="cuda")
    k = big.as_strided((2, 2, size), (stride, size, 1))
    v = big.as_strided((2, 2, size), (stride, size, 1), 1 << 16)
    cache = mc.KVCache4(k, v, 64, 64)
    batch = mc.KVBatch(_i32([70]), B.table.cuda(), _i32([0, 70]), 70)
    x = B.randn(3, 70, 2, 64)
    q = x[0].cuda()
    got = mc.kv4_append(cache, batch, q, x[1].cuda(), x[2].cuda(), q_out=q)
    assert got.data_ptr() == q.data_ptr() and torch.equal(q.cpu(), x[0])
    kr, vr = mc.kv4_read(cache, batch)
    for t in (0, 1, 63, 64, 69):
        for h in range(2):
            assert torch.equal(kr[t, h].double().cpu(), ref4.store(x[1][t, h], "bf16")[2])
            assert torch.equal(vr[t, h].double().cpu(), ref4.store(x[2][t, h], "bf16")[2])
    j = torch.arange(70)
    B.k[B.table[0, j // 64].long(), :, j % 64] = kr.cpu()
    B.v[B.table[0, j // 64].long(), :, j % 64] = vr.cpu()
    want = ref.attention(B, x[0], 0.125)
    ref.assert_attention(mc.attn4_prefill(cache, batch, q), None, want, "bf16", 70, 5.0)
    one = mc.KVBatch(_i32([70]), B.table.cuda())
    out = mc.attn4_decode(cache, one, q[69:])
    ref.assert_attention(out, None, tuple(w[69:] for w in want), "bf16", 70, 5.0)


# ---------------------------------------------------------------- decode --

DECODE = [
    # heads, kv, dim, dtype, page, softcap, window, bias
    (32, 8, 128, "bf16", 16, 0.0, 0, False),
    (8, 8, 64, "fp16", 48, 0.0, 0, False),
    (6, 2, 128, "fp16", 64, 30.0, 0, True),
    (40, 4, 64, "bf16", 32, 0.0, 50, False),
    (16, 1, 128, "bf16", 128, 50.0, 129, True),
    (40, 2, 128, "bf16", 16, 0.0, 1, False),
    (33, 1, 64, "fp16", 16, 0.0, 0, True),
    (1, 1, 128, "fp16", 256, 0.0, 0, False),
]


@pytest.mark.parametrize("heads,kv,dim,dtype,page,softcap,window,bias", DECODE)
def test_decode_matches_its_definition(mc, heads, kv, dim, dtype, page, softcap, window, bias):
    B = ref.Batch(EDGES, [1] * len(EDGES), kv, page, dim, dtype, 5)
    blocks = ref4.fast_blocks(B)
    q = 1.5 * B.randn(len(EDGES), heads, dim)
    sl = _slopes(heads) if bias else None
    want = ref.attention(B, q, dim ** -0.5, softcap, window, sl)
    cache, batch = blocks.device(mc, cu=False, interleave=True)
    ws = mc.attn4_workspace(cache, heads)
    out, lse = mc.attn4_decode(cache, batch, q.cuda(), softcap=softcap, window=window,
                               slopes=None if sl is None else sl.cuda(), with_lse=True, workspace=ws)
    mc.check_status(ws)
    ref.assert_attention(out, lse, want, dtype, max(EDGES), 5.0)


@pytest.mark.parametrize("seqs,length,kv,heads,dim", [(1, 5000, 1, 8, 128), (1, 20011, 2, 8, 64), (3, 2049, 8, 32, 128), (300, 40, 1, 2, 128),
                                                       (1, 1, 1, 1, 64), (70, 900, 2, 8, 64), (128, 129, 1, 16, 128)])
def test_decode_splits_and_joins(mc, seqs, length, kv, heads, dim):
    lens = [max(1, length - 37 * b) if seqs < 100 else (b * 7) % length for b in range(seqs)]
    B = ref.Batch(lens, [1] * seqs, kv, 32, dim, "bf16", 8)
    blocks = ref4.fast_blocks(B)
    q = B.randn(seqs, heads, dim)
    want = ref.attention(B, q, 0.1)
    cache, batch = blocks.device(mc, cu=False)
    out, lse = mc.attn4_decode(cache, batch, q.cuda(), scale=0.1, with_lse=True)
    ref.assert_attention(out, lse, want, "bf16", length, 5.0)
    again, _ = mc.attn4_decode(cache, batch, q.cuda(), scale=0.1, with_lse=True)
    assert torch.equal(out, again)  # the same sums in the same order


def test_groups_far_apart_in_scale(mc):
    """Neighbouring groups and neighbouring keys with scales from 2^-10 to 2^10: no scale reaches another's group."""
    for dtype in ("bf16", "fp16"):
        B = ref.Batch([300, 77], [1, 1], 2, 16, 128, dtype, 12)
        f = 2.0 ** ((torch.arange(16)[:, None] * 7 + torch.arange(2) * 5) % 11 - 8.0)
        B.k = (B.k.unflatten(-1, (2, 64)).float() * f[..., None] * 0.25).flatten(-2).to(B.k.dtype)
        B.v = (B.v.unflatten(-1, (2, 64)).float() * f.flip(0)[..., None] * 64).flatten(-2).to(B.v.dtype)
        blocks = ref4.fast_blocks(B)
        q = B.randn(2, 6, 128)
        want = ref.attention(B, q, 128 ** -0.5)
        cache, batch = blocks.device(mc, cu=False)
        out, lse = mc.attn4_decode(cache, batch, q.cuda(), with_lse=True)
        ref.assert_attention(out, lse, want, dtype, 300, 600.0)
        pre, pl = mc.attn4_prefill(cache, mc.KVBatch(batch._keep[0], batch._keep[1], _i32([0, 1, 2]), 2), q.cuda(), with_lse=True)
        ref.assert_attention(pre, pl, want, dtype, 300, 600.0)


@pytest.mark.parametrize("dim,dtype", [(128, "bf16"), (64, "bf16"), (128, "fp16"), (64, "fp16")])
@pytest.mark.parametrize("heads", [8, 40])  # queries in registers and in shared memory
def test_queries_of_any_size(mc, dim, dtype, heads):
    """Rows whose largest element is 2^-40 to 2^40 (fp16: 2^-12 to 2^12), some elements far below it, a row of zeros: the
    scale makes up for it, and lse is off by 48 roundings of a score of ten at most."""
    B = ref.Batch([300, 77, 5, 130], [1] * 4, 1, 16, dim, dtype, 14)
    blocks = ref4.fast_blocks(B)
    base = B.randn(4, heads, dim).float()
    base[:, :, 3::7] *= 2.0 ** -9
    base[1, 0] = 0
    span = 40 if dtype == "bf16" else 12
    for e in (-span, -10, 0, 11, span):
        q = (base * 2.0 ** e).to(ref.DT[dtype])
        scale = 0.1 * 2.0 ** -e
        want = ref.attention(B, q, scale)
        cache, batch = blocks.device(mc, cu=False)
        out, lse = mc.attn4_decode(cache, batch, q.cuda(), scale=scale, with_lse=True)
        ref.assert_attention(out, lse, want, dtype, 300, 5.0)
        assert ((lse.double().cpu() - want[1]).abs() <= 48 * 2.0 ** -24 * 10).all()


@pytest.mark.parametrize("heads,new", [(8, 1), (20, 1), (32, 1), (40, 1), (8, 3)])  # queries in registers, in shared memory, many rows, few tokens
@pytest.mark.parametrize("dtype,queries,keys", [
    ("bf16", (0, -30), (0, 30)), ("bf16", (-24, 3), (24, -3)), ("bf16", (0, -60), (-20, 40)), ("bf16", (50, -50), (-50, 50)),
    ("bf16", (-100, -100), (118, 118)), ("bf16", (112, 112), (-94, -94)), ("bf16", (-100, 100), (118, -82)),
    ("fp16", (0, -12), (0, 12)), ("fp16", (-10, 10), (12, -8))])
def test_queries_and_keys_far_apart_in_scale(mc, heads, new, dtype, queries, keys):
    """Groups of small queries against groups of large keys and the other way round, as powers of two for each group: what
    they add to a score is of the same size.  Scores are those of 128 products of a few units (their sizes 30 at most in
    sum after the scale), whose fp32 sums are off by 128 * 2^-24 * 30 in the worst case."""
    B = ref.Batch([300, 77, 5, 130], [new] * 4, 1, 16, 128, dtype, 15)
    size = lambda e: 2.0 ** torch.tensor(e, dtype=torch.float64).repeat_interleave(64)  # noqa: E731
    B.k = (B.k.double() * size(keys)).to(B.k.dtype)
    blocks = ref4.fast_blocks(B)
    q = (B.randn(4 * new, heads, 128).double() * size(queries)).to(ref.DT[dtype])
    scale = 0.1 * 2.0 ** -max(a + b for a, b in zip(queries, keys))
    want = ref.attention(B, q, scale)
    cache, batch = blocks.device(mc, cu=new > 1)
    call = mc.attn4_prefill if new > 1 else mc.attn4_decode
    out, lse = call(cache, batch, q.cuda(), scale=scale, with_lse=True)
    ref.assert_attention(out, lse, want, dtype, 300, 5.0)
    assert ((lse.double().cpu() - want[1]).abs() <= 128 * 2.0 ** -24 * 30).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("below", [9.0, 14.0, 17.0])
@pytest.mark.parametrize("new,group", [(1, 1), (32, 8)])  # each kernel
def test_small_weights_keep_their_sum(mc, dtype, below, new, group):
    """8191 equal keys far below one: each weighs little, together they weigh what they should."""
    seqs, kv, length, dim, page = 40, 8, 8192, 64, 128
    T = ref.DT[dtype]
    pages = length // page
    k, v = (torch.zeros(pages, kv, page, dim, dtype=T) for _ in range(2))
    v[:] = (torch.arange(dim) % 16).to(T)  # on the grid of step 1
    k[0, :, 0, 0], v[0, :, 0] = below, 0.0
    B = ref.Batch.__new__(ref.Batch)
    B.__dict__.update(k=k, v=v, kv=kv, page=page, dim=dim, dtype=dtype, lens=[length] * seqs, new=[new] * seqs, table=torch.arange(pages, dtype=torch.int32).repeat(seqs, 1),
                      cu=[new * b for b in range(seqs + 1)], tokens=new * seqs)
    blocks = ref4.fast_blocks(B)
    assert torch.equal(B.v[0, 0, 1], v[0, 0, 1])
    below = float(B.k[0, 0, 0, 0])
    cache, batch = blocks.device(mc)
    q = torch.zeros(new * seqs, kv * group, dim, dtype=T, device="cuda")
    q[..., 0] = 1.0
    out, lse = mc.attn4_prefill(cache, batch, q, scale=1.0, with_lse=True)
    others = torch.arange(length - new, length, dtype=torch.float64)  # keys after the first one, of each new token
    w = others * np.exp(-below)
    want = (w / (1 + w))[:, None] * v[0, 0, 1].double()
    h = ref.HALF_ULP[dtype]
    tol = (2 * h + 1e-4) * want + (2.0 ** -24 + length * 2.0 ** -32 * 64 if dtype == "fp16" else 0) + 1e-30
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
MANY = ([0, 1, 17, 64, 130, 300, 511, 9, 257], [2, 1, 17, 3, 130, 1, 129, 12, 64], [0, 1, 9, 64, 70, 299, 1000, 4, 250])
FEW = ([0, 5, 17, 64, 130, 300, 511, 3, 1025], [2, 5, 3, 1, 8, 4, 6, 7, 5], [1, 3, 17, 60, 125, 0, 600, 2, 1022])


@pytest.mark.parametrize("few", [False, True])
@pytest.mark.parametrize("heads,kv,dim,dtype,page,softcap,window,bias,prefix", PREFILL)
def test_prefill_matches_its_definition(mc, heads, kv, dim, dtype, page, softcap, window, bias, prefix, few):
    """Many rows a sequence and few (slices of 8 to 32 rows), sequences with more new tokens than their length."""
    lens, new, pre = FEW if few else MANY
    B = ref.Batch(lens, new, kv, page, dim, dtype, 6, pad_tokens=2)
    blocks = ref4.fast_blocks(B)
    q = 1.5 * B.randn(B.tokens, heads, dim)
    sl = _slopes(heads) if bias else None
    pre = pre if prefix else None
    want = ref.attention(B, q, dim ** -0.5, softcap, window, sl, pre)
    cache, batch = blocks.device(mc)
    ws = mc.attn4_workspace(cache, heads)
    out = torch.full((B.tokens, heads + 1, dim), 3.0, dtype=ref.DT[dtype], device="cuda")
    got, lse = mc.attn4_prefill(cache, batch, q.cuda(), softcap=softcap, window=window,
                                slopes=None if sl is None else sl.cuda(), prefix=None if pre is None else _i32(pre),
                                out=out[:, :heads], with_lse=True, workspace=ws)
    mc.check_status(ws)
    n = B.cu[-1]
    assert (out[:, heads] == 3).all() and (out[n:] == 3).all()  # other heads' columns and padding rows
    ref.assert_attention(got, lse, want, dtype, 1025, 5.0, rows=slice(0, n))


def _far(mc, blocks, **kw):
    """(cache, batch) with tables of 12288 keys and more, their last entries no pages."""
    cache, batch = blocks.device(mc, **kw)
    B = blocks.B
    table = torch.full((len(B.lens), -(-12288 // B.page)), -7, dtype=torch.int32)
    table[:, :B.table.shape[1]] = B.table
    assert B.cu[-1] * 1.0 * table.shape[1] * B.page / 256 / 128 > 4096 / 20
    return cache, mc.KVBatch(batch._keep[0], table.cuda(), batch._keep[2], B.tokens)


@pytest.mark.parametrize("page_of", [0, 17])
def test_a_long_prompt_with_a_page_outside_the_pool(mc, page_of):
    """It reads as zeros and is recorded, and what the workspace holds from before does not show."""
    lens, new, heads, kv = [600, 300], [400, 300], 48, 2
    ok = ref.Batch(lens, new, kv, 16, 64, "bf16", 111)
    blocks = ref4.fast_blocks(ok)
    q = ok.randn(ok.tokens, heads, 64)
    cache, batch = _far(mc, blocks)
    ws = mc.attn4_workspace(cache, heads)
    got, lse = mc.attn4_prefill(cache, batch, q.cuda(), with_lse=True, workspace=ws)
    mc.check_status(ws)
    ref.assert_attention(got, lse, ref.attention(ok, q, 0.125), "bf16", 600, 5.0)
    for bad in (ok.k.shape[0], -1, 2 ** 31 - 1, -2 ** 31):
        table = batch._keep[1].clone()
        table[0, page_of] = bad
        out, out_lse = mc.attn4_prefill(cache, mc.KVBatch(batch._keep[0], table, batch._keep[2], ok.tokens), q.cuda(), with_lse=True, workspace=ws)
        _reported(mc, ws)
        assert torch.equal(out[400:], got[400:])
    zero = ref.Batch(lens, new, kv, 16, 64, "bf16", 111)
    ref4.fast_blocks(zero)
    zero.k[zero.table[0, page_of].long()] = 0
    zero.v[zero.table[0, page_of].long()] = 0
    ref.assert_attention(out, out_lse, ref.attention(zero, q, 0.125), "bf16", 600, 5.0)


@pytest.mark.parametrize("heads,kv,dim,dtype,page,softcap,window,bias,prefix,nan", [
    (32, 2, 128, "bf16", 16, 0.0, 0, False, False, False),
    (24, 1, 64, "fp16", 48, 0.0, 0, False, True, False),
    (20, 1, 128, "fp16", 64, 30.0, 0, True, False, False),
    (40, 2, 64, "bf16", 32, 0.0, 50, False, False, True),
    (17, 1, 128, "bf16", 128, 50.0, 129, True, True, False),
    (32, 2, 128, "bf16", 16, 0.0, 0, False, False, True),
    (20, 1, 64, "fp16", 16, 20.0, 100, False, False, False),
])
def test_prompts_of_many_rows(mc, heads, kv, dim, dtype, page, softcap, window, bias, prefix, nan):
    """1024 rows a sequence and more, with tables that reach far, which is where a workspace with room for prompts has
    their keys unpacked first: strided queries and outputs, more new tokens than the length, sequences without tokens or keys, hidden groups of
    NaN, pages that a window has left behind; and again over what the call before left in the workspace."""
    lens, new, pre = [0, 3, 130, 300, 511, 9, 700, 64], [2, 3, 130, 1, 129, 12, 400, 0], [0, 1, 64, 70, 299, 4, 650, 64]
    B = ref.Batch(lens, new, kv, page, dim, dtype, 6, pad_tokens=2)
    assert -(-B.tokens // len(lens)) * (heads // kv) >= 1024
    if nan:
        for b, length in enumerate(lens):
            if new[b] > 1 and length:
                B.v[B.table[b, (length - 1) // page], :, (length - 1) % page, 3] = float("nan")
    blocks = ref4.fast_blocks(B)
    wide = 1.5 * B.randn(B.tokens, heads * dim + 8)
    q = wide[:, 8:].unflatten(1, (heads, dim))
    sl = _slopes(heads) if bias else None
    pre = pre if prefix else None
    want = ref.attention(B, q, dim ** -0.5, softcap, window, sl, pre)
    if window:
        for b, (n, length) in enumerate(zip(new, lens)):
            gone = max(0, length - n - window + 1) // page
            for p in blocks.pools:
                p[B.table[b, :gone].long()] = 0xff
            B.table[b, :gone] = -1
    cache, batch = _far(mc, blocks, interleave=True)
    ws = mc.attn4_workspace(cache, heads)
    ws[256 + (1 << 20):] = 0xff  # (what a call leaves there is any bits)
    dev = wide.cuda()[:, 8:].unflatten(1, (heads, dim))
    for _ in range(2):
        buf = torch.full((B.tokens, heads * dim + 8), 3.0, dtype=ref.DT[dtype], device="cuda")
        got, lse = mc.attn4_prefill(cache, batch, dev, softcap=softcap, window=window, slopes=None if sl is None else sl.cuda(),
                                    prefix=None if pre is None else _i32(pre), out=buf[:, :heads * dim].unflatten(1, (heads, dim)),
                                    with_lse=True, workspace=ws)
        mc.check_status(ws)
        n = B.cu[-1]
        assert (buf[:, heads * dim:] == 3).all() and (buf[n:] == 3).all()
        if nan:
            assert torch.equal(torch.isnan(got[:n].cpu()), torch.isnan(want[0][:n]))
            seen = torch.isnan(want[0][:n]).flatten(1).any(1).nonzero().flatten().tolist()
            assert seen
            rows = [t for t in range(n) if t not in seen]
        else:
            rows = slice(0, n)
        ref.assert_attention(got, lse, want, dtype, 700, 5.0, rows=rows)


@pytest.mark.parametrize("new,length,kv,heads,dim", [(1, 4000, 1, 4, 128), (5, 9000, 1, 5, 128), (40, 6000, 2, 4, 64), (700, 700, 1, 1, 128),
                                                     (515, 2100, 2, 6, 128), (1, 1, 1, 1, 64)])
def test_prefill_splits_and_joins(mc, new, length, kv, heads, dim):
    B = ref.Batch([length], [new], kv, 64, dim, "bf16", 8)
    blocks = ref4.fast_blocks(B)
    q = B.randn(new, heads, dim)
    want = ref.attention(B, q, dim ** -0.5)
    cache, batch = blocks.device(mc)
    out, lse = mc.attn4_prefill(cache, batch, q.cuda(), with_lse=True)
    ref.assert_attention(out, lse, want, "bf16", length, 5.0)
    again, _ = mc.attn4_prefill(cache, batch, q.cuda(), with_lse=True)
    assert torch.equal(out, again)


@pytest.mark.parametrize("seqs,heads,kv", [(45, 16, 1), (70, 40, 1)])
def test_prefill_of_many_sequences(mc, seqs, heads, kv):
    """More sequences than a warp has lanes, some without tokens, some without keys."""
    new = [(5 * b) % 23 for b in range(seqs)]
    lens = [0 if b % 11 == 4 else new[b] + (37 * b) % 300 for b in range(seqs)]
    B = ref.Batch(lens, new, kv, 16, 64, "bf16", 61, pad_tokens=1)
    blocks = ref4.fast_blocks(B)
    q = B.randn(B.tokens, heads, 64)
    want = ref.attention(B, q, 0.125)
    cache, batch = blocks.device(mc)
    ws = mc.attn4_workspace(cache, heads)
    out, lse = mc.attn4_prefill(cache, batch, q.cuda(), with_lse=True, workspace=ws)
    mc.check_status(ws)
    ref.assert_attention(out, lse, want, "bf16", 400, 5.0, rows=slice(0, B.cu[-1]))


@pytest.mark.parametrize("lens,new,heads,kv,dim,dtype,window,cap", [
    ([4096], [4096], 32, 8, 128, "bf16", 0, 0.0),
    ([3001, 40, 0, 2500, 3700, 1], [3001, 9, 0, 2300, 3600, 1], 12, 4, 64, "fp16", 0, 20.0),  # items of five sequences
    ([5000] + [700] * 31, [5000] + [300] * 31, 16, 4, 64, "bf16", 900, 0.0),                 # as many as a queue takes
    ([4000] + [100] * 32, [4000] + [100] * 32, 16, 4, 64, "bf16", 0, 0.0),                   # one more: runs
    ([80000], [200], 8, 2, 128, "bf16", 60000, 0.0),                                         # a chunk of a long one
])
def test_prefill_is_that_of_the_16_bit_cache(mc, lens, new, heads, kv, dim, dtype, window, cap):
    """Large batches against attn_prefill over a 16-bit cache that holds the same numbers: the kernels
    multiply the same operands, so each is within its bound of the other; twice over, bit for bit."""
    B = ref.Batch(lens, new, kv, 64, dim, dtype, 61, pad_tokens=2)
    blocks = ref4.fast_blocks(B)
    q = B.randn(B.tokens, heads, dim).cuda()
    cache16, batch = B.device(mc)
    cache, _ = blocks.device(mc)
    ws, ws16 = mc.attn4_workspace(cache, heads), mc.attn_workspace(cache16, heads)
    slopes = (-torch.linspace(0.1, 0.01, heads)).cuda() if cap else None
    kw = dict(softcap=cap, window=window, slopes=slopes, with_lse=True)
    want, want_lse = mc.attn_prefill(cache16, batch, q, workspace=ws16, **kw)
    got, lse = mc.attn4_prefill(cache, batch, q, workspace=ws, **kw)
    again, _ = mc.attn4_prefill(cache, batch, q, workspace=ws, **kw)
    mc.check_status(ws)
    n = B.cu[-1]
    assert torch.equal(got[:n], again[:n])
    h = ref.HALF_ULP[dtype]
    assert ((got[:n].float() - want[:n].float()).abs() <= 2 * (2 * h + 1e-4) * 5).all()
    fin = torch.isfinite(want_lse[:n])
    assert torch.equal(torch.isfinite(lse[:n]), fin)
    assert ((lse[:n] - want_lse[:n])[fin].abs() <= 1e-4).all()


@pytest.mark.parametrize("cap", [50.0, 1e5])
@pytest.mark.parametrize("dim,dtype,lens,new", [(128, "bf16", [900, 2, 1, 3000], [1] * 4), (64, "fp16", [1, 2, 3, 5, 8, 64], [1] * 6),
                                                (128, "bf16", [4, 3, 70], [4, 2, 3]), (64, "bf16", [140, 300], [140, 80])])
def test_caps_over_few_keys(mc, dim, dtype, cap, lens, new):
    """lse to 32 roundings of fp32 (2^-24) of itself or of a score of one: products of 128 terms, 16, their
    groups' scales, sums and logarithm, 8, and 8 for the cap's form."""
    B = ref.Batch(lens, new, 2, 16, dim, dtype, 71)
    blocks = ref4.fast_blocks(B)
    q = B.randn(B.tokens, 6, dim)
    want = ref.attention(B, q, dim ** -0.5, cap)
    cache, batch = blocks.device(mc)
    out, lse = mc.attn4_prefill(cache, batch, q.cuda(), softcap=cap, with_lse=True)
    ref.assert_attention(out, lse, want, dtype, 3000, 5.0)
    assert ((lse.double().cpu() - want[1]).abs() <= 32 * 2.0 ** -24 * (1 + want[1].abs())).all()


@pytest.mark.parametrize("dim,dtype,lens,new,heads,kv,window,cap", [
    (128, "bf16", [40, 300], [6, 3], 4, 2, 0, 0.0),         # few rows
    (64, "fp16", [9000], [5], 2, 1, 100, 0.0),              # the same, over pages that a window has left behind
    (64, "bf16", [9000], [5], 2, 1, 0, 0.0),                # the same, split and joined
    (128, "bf16", [300, 130], [200, 130], 4, 2, 0, 0.0),    # many rows
    (64, "fp16", [300, 700], [300, 64], 3, 1, 40, 0.0),
    (128, "fp16", [5000], [100], 2, 1, 0, 0.0),             # many rows, split and joined
])
def test_hidden_groups_of_nan_stay_hidden(mc, dim, dtype, lens, new, heads, kv, window, cap):
    """Groups that are NaN in keys and values that some queries see and others do not."""
    B = ref.Batch(lens, new, kv, 16, dim, dtype, 41)
    q = B.randn(B.tokens, heads, dim)
    for b, (n, length) in enumerate(zip(new, lens)):
        for at, what, col in ((length - 1, float("nan"), 3), (length - 2, float("inf"), dim - 7)):
            B.v[B.table[b, at // 16], :, at % 16, col] = what
        if window:  # a key that the window has left behind (the batch that starts at 0: seen by its first queries)
            B.v[B.table[b, 0], :, 0, :] = float("nan")
            B.k[B.table[b, 0], :, 0, :] = float("nan")
    blocks = ref4.Blocks(B) if sum(lens) < 2000 else ref4.fast_blocks(_groups_of_nan(B))
    want = ref.attention(B, q, dim ** -0.5, cap, window=window)
    cache, batch = blocks.device(mc)
    ws = mc.attn4_workspace(cache, heads)
    got, lse = mc.attn4_prefill(cache, batch, q.cuda(), softcap=cap, window=window, with_lse=True, workspace=ws)
    mc.check_status(ws)
    got = got.double().cpu()
    odd = torch.isnan(want[0])
    assert odd.any() and not odd.all() and torch.equal(torch.isnan(got), odd)
    h = ref.HALF_ULP[dtype]
    tol = (2 * h + 1e-4) * want[2] + 1e-30 + (2.0 ** -24 + max(lens) * 2.0 ** -25 * 5 if dtype == "fp16" else 0)
    assert ((got - want[0]).abs() <= tol)[~odd].all()
    assert torch.allclose(lse.double().cpu(), want[1], rtol=1e-4, atol=1e-4, equal_nan=True)


def _groups_of_nan(B):
    """(grids() takes a group's NaN for its scale, but an infinity for a span)"""
    for c in (B.k, B.v):
        c[torch.isinf(c)] = float("nan")
    return B


def test_a_sequence_of_nan_leaves_the_others_alone(mc):
    """One token each: a NaN key, a NaN value, and unwritten rows behind every length."""
    B = ref.Batch([33, 50, 18, 700], [1] * 4, 1, 16, 128, "bf16", 42)
    B.k[B.table[1, 2], 0, 3, 5] = float("nan")
    B.v[B.table[2, 0], 0, 7, 100] = float("nan")
    blocks = ref4.Blocks(B)
    q = B.randn(4, 4, 128)
    want = ref.attention(B, q, 0.1, 30.0)
    cache, batch = blocks.device(mc, cu=False)
    for call in (mc.attn4_decode, mc.attn4_prefill):
        out, lse = call(cache, batch, q.cuda(), scale=0.1, softcap=30.0, with_lse=True)
        assert torch.equal(torch.isnan(out.cpu()), torch.isnan(want[0]))
        assert torch.isnan(out[1]).all() and torch.isnan(out[2, :, 64:]).all() and torch.isfinite(out[2, :, :64]).all()
        ref.assert_attention(out, lse, want, "bf16", 700, 5.0, rows=[0, 3])


@pytest.mark.parametrize("new", [[2, 3, 1], [200, 131, 60]])  # few rows, many rows
@pytest.mark.parametrize("heads,kv,dim,dtype", [(4, 1, 128, "bf16"), (3, 1, 64, "fp16"), (10, 2, 128, "fp16"), (17, 1, 64, "bf16")])
def test_queries_and_outputs_with_a_token_stride(mc, new, heads, kv, dim, dtype):
    B = ref.Batch([260, 400, 61], new, kv, 16, dim, dtype, 107, pad_tokens=1)
    blocks = ref4.fast_blocks(B)
    wide = B.randn(B.tokens, (heads + 2 * kv) * dim + 8)
    q = wide[:, 8:8 + heads * dim].unflatten(1, (heads, dim))
    want = ref.attention(B, q, dim ** -0.5)
    cache, batch = blocks.device(mc)
    ws = mc.attn4_workspace(cache, heads)
    dev = wide.cuda()[:, 8:8 + heads * dim].unflatten(1, (heads, dim))
    buf = torch.full((B.tokens, heads * dim + 8), 3.0, dtype=ref.DT[dtype], device="cuda")
    out = buf[:, :heads * dim].unflatten(1, (heads, dim))
    got, lse = mc.attn4_prefill(cache, batch, dev, out=out, with_lse=True, workspace=ws)
    mc.check_status(ws)
    assert (buf[:, heads * dim:] == 3).all() and (buf[B.cu[-1]:] == 3).all()
    ref.assert_attention(got, lse, want, dtype, 400, 5.0, rows=slice(0, B.cu[-1]))


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("new,heads", [([1, 1, 1], 8), ([2, 1, 3], 8), ([50, 70, 130], 8), ([50, 70, 130], 40)])  # one, few and many rows
def test_pages_lengths_and_boundaries_that_are_not_sound(mc, new, heads, cap):
    """A page outside the pool reads as zeros, a length is cut to the table's rows, a sequence whose
    boundaries are not sound has no tokens; each is recorded, and the other sequences are right."""
    lens, kv, dim = [96, 160, 144], 2, 64
    ok = ref.Batch(lens, new, kv, 16, dim, "bf16", 109)
    blocks = ref4.fast_blocks(ok)
    q = ok.randn(ok.tokens, heads, dim)
    cache, batch = blocks.device(mc)

    def attend(b):
        ws = mc.attn4_workspace(cache, heads)
        out = torch.full((ok.tokens, heads, dim), 3.0, dtype=torch.bfloat16, device="cuda")
        _, lse = mc.attn4_prefill(cache, b, q.cuda(), softcap=cap, out=out, with_lse=True, workspace=ws)
        return out, lse, ws

    want = ref.attention(ok, q, dim ** -0.5, cap)
    good, good_lse, ws = attend(batch)
    mc.check_status(ws)
    ref.assert_attention(good, good_lse, want, "bf16", 160, 5.0)
    for page in (ok.k.shape[0], -1, 2 ** 31 - 1, -2 ** 31):  # of sequence 1's keys 32 .. 47
        table = ok.table.clone()
        table[1, 2] = page
        out, lse, ws = attend(mc.KVBatch(batch._keep[0], table.cuda(), batch._keep[2], ok.tokens))
        _reported(mc, ws)
        zero = ref.Batch(lens, new, kv, 16, dim, "bf16", 109)
        ref4.fast_blocks(zero)
        zero.k[zero.table[1, 2].long()] = 0
        zero.v[zero.table[1, 2].long()] = 0
        ref.assert_attention(out, lse, ref.attention(zero, q, dim ** -0.5, cap), "bf16", 160, 5.0)
        others = [t for t in range(ok.tokens) if not ok.cu[1] <= t < ok.cu[2]]
        assert torch.equal(out[others], good[others])
        k, v = mc.kv4_read(cache, mc.KVBatch(_i32([96, 48, 144]), table.cuda(), _i32([0, 0, 16, 16]), 16))
        assert (k == 0).all() and (v == 0).all()
    for length in (161, 1 << 20, 2 ** 31 - 1):
        out, lse, ws = attend(mc.KVBatch(_i32([96, length, 144]), batch._keep[1], batch._keep[2], ok.tokens))
        _reported(mc, ws)
        ref.assert_attention(out, lse, want, "bf16", 160, 5.0)  # (the table has pages for 160 rows)
    for cu, sound in (([0, ok.cu[1], ok.tokens + 1, ok.tokens + 1], [0]), ([-1, ok.cu[1], ok.cu[2], ok.cu[3]], [1, 2])):
        out, lse, ws = attend(mc.KVBatch(batch._keep[0], batch._keep[1], _i32(cu), ok.tokens))
        _reported(mc, ws)
        for b in sound:
            t = slice(ok.cu[b], ok.cu[b + 1])
            ref.assert_attention(out[t], lse[t], tuple(w[t] for w in want), "bf16", 160, 5.0)


def test_pages_behind_the_window_may_be_gone(mc):
    """Their table entries are not read and their rows not looked at."""
    for new, heads, cap in ((1, 4, 0.0), (4, 4, 0.0), (1, 32, 0.0), (150, 4, 0.0), (150, 4, 20.0)):
        B = ref.Batch([700, 333], [new, new], 2, 16, 64, "bf16", 51)
        q = B.randn(B.tokens, heads, 64)
        blocks = ref4.fast_blocks(B)
        want = ref.attention(B, q, 0.125, cap, 100)
        for b, length in enumerate(B.lens):
            gone = max(0, length - new - 100 + 1) // 16
            for p in blocks.pools:
                p[B.table[b, :gone].long()] = 0xff
            B.table[b, :gone] = -1
        cache, batch = blocks.device(mc)
        ws = mc.attn4_workspace(cache, heads)
        out, lse = mc.attn4_prefill(cache, batch, q.cuda(), softcap=cap, window=100, with_lse=True, workspace=ws)
        mc.check_status(ws)
        ref.assert_attention(out, lse, want, "bf16", 700, 5.0)


@pytest.mark.parametrize("seqs,new,length,heads,kv", [(1, 4096, 4096, 16, 4),   # whole items
                                                      (1, 300, 9000, 8, 2),     # split and joined
                                                      (16, 4, 4000, 16, 4)])    # few rows a sequence
def test_a_visible_nan_costs_little(mc, seqs, new, length, heads, kv):
    """A NaN that every row sees: none is redone key by key."""
    B = ref.Batch([length] * seqs, [new] * seqs, kv, 64, 128, "bf16", 83)
    q = B.randn(B.tokens, heads, 128).cuda()
    k0, v0 = B.k.clone(), B.v.clone()
    took, got = [], []
    for what in (None, float("nan")):
        B.k, B.v = k0.clone(), v0.clone()
        if what is not None:
            for b in range(seqs):
                B.v[B.table[b, 0], :, 0, 3] = what
        cache, batch = ref4.fast_blocks(B).device(mc)
        ws = mc.attn4_workspace(cache, heads)
        out = torch.full_like(q, 100.0)
        call = lambda: mc.attn4_prefill(cache, batch, q, out=out, workspace=ws)  # noqa: E731
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
    assert torch.isnan(got[1][..., :64]).all()
    assert torch.equal(got[0][..., 64:], got[1][..., 64:])
    assert took[1] <= 10 * took[0], took


# ----------------------------------------------------------- streams, status --

def test_on_another_stream_and_in_graphs_that_share_a_workspace(mc):
    B = ref.Batch([40, 130, 7], [1] * 3, 2, 16, 64, "bf16", 21)
    cache, batch = ref4.fast_blocks(B).device(mc, cu=False)
    q, k, v = (B.randn(3, n, 64).cuda() for n in (8, 2, 2))
    rope = ref.rope_table(200, 64).cuda()
    ws = mc.attn4_workspace(cache, 8)

    def step():
        return mc.attn4_decode(cache, batch, mc.kv4_append(cache, batch, q, k, v, rope=rope, workspace=ws), workspace=ws)

    def chunk():
        return mc.attn4_prefill(cache, batch, q.repeat(1, 8, 1), workspace=ws)  # 64 heads: the kernel for many rows

    want, want2 = step().clone(), chunk().clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got, got2 = step(), chunk()
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(got2, want2)
    graphs, res = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g, f in zip(graphs, (step, chunk)):
        with torch.cuda.graph(g):
            res.append(f())
    for _ in range(3):
        for r in res:
            r.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(res[0], want) and torch.equal(res[1], want2)
    mc.check_status(ws)


def test_an_append_without_a_page_or_position_is_reported(mc):
    B = ref.Batch([40, 64], [1, 1], 2, 16, 64, "bf16", 22)
    cache, batch = ref4.fast_blocks(B).device(mc, cu=False)
    q, k, v = (B.randn(2, n, 64).cuda() for n in (4, 2, 2))
    ws = mc.attn4_workspace(cache, 4)
    before = cache.k.clone()
    bad = B.table.clone()
    bad[0, 2] = -1  # the page of the new token of sequence 0
    mc.kv4_append(cache, mc.KVBatch(batch._keep[0], bad.cuda()), q, k, v, workspace=ws)
    _reported(mc, ws)
    changed = (cache.k != before).flatten(1).any(1).nonzero().flatten()
    assert changed.tolist() == [int(B.table[1, 3])]
    mc.kv4_append(cache, batch, q, k, v, rope=ref.rope_table(10, 64).cuda(), workspace=ws)  # positions past the table
    _reported(mc, ws)
    mc.kv4_append(cache, mc.KVBatch(_i32([200, 64]), B.table.cuda()), q, k, v, workspace=ws)  # a length past the pages
    _reported(mc, ws)


@pytest.mark.parametrize("lens,new,heads", [([300], [300], 4), ([300, 40], [200, 40], 3)])
def test_waits_expire_and_the_context_lives(mc, lens, new, heads):
    """With the copies switched off every wait of the kernel for many rows reaches its bound."""
    B = ref.Batch(lens, new, 1, 16, 64, "bf16", 23)
    cache, batch = ref4.fast_blocks(B).device(mc)
    q = B.randn(B.tokens, heads, 64).cuda()
    ws = mc.attn4_workspace(cache, heads)
    want = mc.attn4_prefill(cache, batch, q, workspace=ws)
    mc.check_status(ws)
    mc.set_debug(1, 20_000_000)
    try:
        mc.attn4_prefill(cache, batch, q, workspace=ws)
        with pytest.raises(mc.MCError) as e:
            mc.check_status(ws)
        assert e.value.code == mc.ERR_TIMEOUT
    finally:
        mc.set_debug(0, 1_000_000_000)
    assert torch.equal(mc.attn4_prefill(cache, batch, q, workspace=ws), want)
    mc.check_status(ws)
