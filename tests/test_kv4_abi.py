"""What the 4-bit cache's, the plan's and the residual norm's entry points refuse, on the host, before any device
work."""
import ctypes

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def mc():
    from paper_2410_06270_gb300 import build
    build.build()
    import paper_2410_06270_gb300 as m
    m.load()
    return m


def _cpu(mc, pages=4, kv=2, page=16, dim=64, dtype=torch.bfloat16, seqs=3, width=2):
    k, v = (torch.zeros(pages, kv, mc.kv4_block_size(page, dim), dtype=torch.uint8) for _ in range(2))
    return mc.KVCache4(k, v, page, dim, dtype), mc.KVBatch(torch.ones(seqs, dtype=torch.int32), torch.zeros(seqs, width, dtype=torch.int32))


def _code(mc, fn, *a, **k):
    with pytest.raises(mc.MCError) as e:
        fn(*a, **k)
    assert str(e.value)
    return e.value.code


def test_block_sizes(mc):
    assert mc.kv4_block_size(16, 64) == 16 * 34 and mc.kv4_block_size(48, 128) == 48 * 68
    for page, dim in ((8, 64), (24, 64), (0, 128), (65536, 64), (16, 96), (16, 0)):
        assert _code(mc, mc.kv4_block_size, page, dim) == mc.ERR_INVALID_ARG


@pytest.mark.parametrize("field,value,code", [
    ("head_dim", 96, -2), ("dtype", 2, -2), ("page_size", 8, -1), ("page_size", 24, -1), ("page_size", 1 << 16, -1),
    ("num_pages", 0, -1), ("kv_heads", 0, -1), ("kv_heads", 3, -1), ("page_stride", 2 * 16 * 34 - 16, -1),
    ("page_stride", 2 * 16 * 34 + 8, -1), ("page_stride", 1 << 40, -1)])
def test_bad_caches(mc, field, value, code):
    cache, batch = _cpu(mc)
    setattr(cache._c, field, value)
    lib, fake = mc.load(), 0x100000  # never dereferenced: every call below is refused
    assert lib.mc_attn4_workspace_size(cache._ref, 4, 1) == 0 and mc.last_error()
    opts = mc._AttnOptsC(0.1, 0.0, 0, None, None)
    for fn in (lib.mc_attn4_decode, lib.mc_attn4_prefill):
        assert fn(cache._ref, batch._ref, fake, 256, 4, ctypes.addressof(opts), fake, 256, None, fake, 1 << 30, None) == code
    assert lib.mc_kv4_append(cache._ref, batch._ref, fake, 256, fake, 128, fake, 128, 4, None, None, 1e-6, None, 0, 0, 0, fake, None, None) == code
    if field != "kv_heads" or value == 0:
        assert lib.mc_kv4_read(cache._ref, batch._ref, fake, fake, None, None) == code


def test_binding_refuses_what_c_cannot_see(mc):
    cache, batch = _cpu(mc)
    q, kv = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    u8 = cache.k
    assert _code(mc, mc.KVCache4, u8, u8, 16, 64, torch.float32) == mc.ERR_UNSUPPORTED
    for k, v in ((u8, u8[:3]), (u8.view(torch.int8), u8.view(torch.int8)), (u8[..., :-16], u8[..., :-16]), (u8.transpose(1, 2), u8.transpose(1, 2)),
                 (u8[0], u8[0]), (torch.cat([u8, u8], 2)[..., :u8.shape[2]],) * 2):
        assert _code(mc, mc.KVCache4, k, v, 16, 64) == -1
    assert _code(mc, mc.KVCache4, u8, u8, 32, 64) == -1
    for bad in (q.half(), q[:2], q[:, :, :32], q.transpose(0, 1), q.flatten(1)):
        assert _code(mc, mc.attn4_decode, cache, batch, bad, workspace=ws) == -1
        assert _code(mc, mc.kv4_append, cache, batch, bad, kv, kv, workspace=ws) == -1
    assert _code(mc, mc.kv4_append, cache, batch, q, q, kv) == -1
    assert _code(mc, mc.kv4_append, cache, batch, q, kv, kv, q_norm=torch.ones(32, dtype=torch.bfloat16)) == -1
    assert _code(mc, mc.kv4_read, cache, batch, k=q) == -1
    # either cache with the other's calls
    plain = mc.KVCache(*(torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16) for _ in range(2)))
    for fn in (mc.attn4_decode, mc.attn4_prefill):
        assert _code(mc, fn, plain, batch, q, workspace=ws) == -1
    for fn in (mc.attn_decode, mc.attn_prefill):
        assert _code(mc, fn, cache, batch, q, workspace=ws) == -1
    assert _code(mc, mc.kv4_append, plain, batch, q, kv, kv) == -1
    assert _code(mc, mc.kv_append, cache, batch, q, kv, kv) == -1
    assert _code(mc, mc.kv4_read, plain, batch) == -1
    assert _code(mc, mc.attn4_workspace, plain, 4) == -1
    assert _code(mc, mc.attn_workspace, cache, 4) == -1


def test_a_users_own_kind_of_cache_is_what_it_derives_from(mc):
    """A class derived from KVCache4 holds bytes: the 16-bit calls, which would take its strides for elements, refuse it."""
    class Four(mc.KVCache4):
        pass

    class Sixteen(mc.KVCache):
        pass

    k, v = (torch.zeros(4, 2, mc.kv4_block_size(16, 64), dtype=torch.uint8) for _ in range(2))
    four, sixteen = Four(k, v, 16, 64), Sixteen(*(torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16) for _ in range(2)))
    batch = _cpu(mc)[1]
    q, kv = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: mc.kv_append(four, batch, q, kv, kv), lambda: mc.attn_decode(four, batch, q), lambda: mc.attn_prefill(four, batch, q),
                 lambda: mc.attn_workspace(four, 4), lambda: mc.kv4_append(sixteen, batch, q, kv, kv), lambda: mc.attn4_decode(sixteen, batch, q),
                 lambda: mc.attn4_prefill(sixteen, batch, q), lambda: mc.kv4_read(sixteen, batch), lambda: mc.attn4_workspace(sixteen, 4)):
        with pytest.raises(mc.MCError, match="is taken") as e:
            call()
        assert e.value.code == mc.ERR_INVALID_ARG
    assert mc.attn4_workspace(four, 4, prompts=False).numel() == mc.attn4_workspace(_cpu(mc)[0], 4, prompts=False).numel()
    assert mc.attn_workspace(sixteen, 4).numel() > 0


def test_host_tensors_are_refused(mc):
    """Before anything is launched: the answer is an argument error, not a launch's."""
    cache, batch = _cpu(mc)
    q, kv = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    ws = torch.zeros(mc.load().mc_attn4_workspace_size(cache._ref, 4, 0) + 256, dtype=torch.uint8)
    ws = ws[-ws.data_ptr() % 256:]
    for call in (lambda: mc.kv4_append(cache, batch, q, kv, kv), lambda: mc.kv4_read(cache, batch),
                 lambda: mc.attn4_decode(cache, batch, q, workspace=ws), lambda: mc.attn4_prefill(cache, batch, q, workspace=ws)):
        assert _code(mc, call) == mc.ERR_INVALID_ARG
    pool = mc.KVPool(4, 16, device="cpu")
    i32 = torch.zeros(3, dtype=torch.int32)
    assert _code(mc, mc.kv_plan, pool, torch.zeros(3, 2, dtype=torch.int32), i32, i32) == mc.ERR_INVALID_ARG
    assert _code(mc, mc.residual_norm, q[0], q[0]) == mc.ERR_INVALID_ARG


def test_bad_pointers(mc):
    cache, batch = _cpu(mc)
    lib, fake, odd = mc.load(), 0x100000, 0x100008
    need = lib.mc_attn4_workspace_size(cache._ref, 4, 0)
    assert 0 < need == lib.mc_attn4_workspace_size(cache._ref, 4, 1) - (256 << 20)

    def attn(fn, q=fake, qs=256, heads=4, out=fake, os=256, lse=None, ws=fake, nbytes=need, scale=0.1, cap=0.0, window=0, prefix=None):
        opts = mc._AttnOptsC(scale, cap, window, None, prefix)
        return fn(cache._ref, batch._ref, q, qs, heads, ctypes.addressof(opts), out, os, lse, ws, nbytes, None)

    for bad in ({"q": None}, {"q": odd}, {"qs": 248}, {"heads": 3}, {"out": None}, {"out": odd}, {"os": 255}, {"lse": 0x100002}, {"ws": None},
                {"ws": 0x100010}, {"nbytes": need - 1}, {"scale": 0.0}, {"cap": -1.0}, {"window": -1}):
        for fn in (lib.mc_attn4_decode, lib.mc_attn4_prefill):
            assert attn(fn, **bad) == mc.ERR_INVALID_ARG, bad
    assert attn(lib.mc_attn4_decode, prefix=fake) == mc.ERR_INVALID_ARG
    for k, v, ws in ((odd, fake, None), (fake, odd, None), (fake, fake, 0x100001)):
        assert lib.mc_kv4_read(cache._ref, batch._ref, k, v, ws, None) == mc.ERR_INVALID_ARG
    assert lib.mc_kv4_read(None, batch._ref, fake, fake, None, None) == mc.ERR_INVALID_ARG
    assert lib.mc_kv4_read(cache._ref, None, fake, fake, None, None) == mc.ERR_INVALID_ARG
    _, none = _cpu(mc, seqs=0)
    assert lib.mc_kv4_read(cache._ref, none._ref, None, None, None, None) == mc.OK


def test_plans(mc):
    pool = mc.KVPool(8, 16, device="cpu")
    lib, fake = mc.load(), 0x100000
    need = lib.mc_kv_plan_workspace_size(5)
    assert need >= 256 + 20 and lib.mc_kv_plan_workspace_size(-1) == 0

    def call(lens=fake, add=fake, done=None, seqs=5, tokens=9, table=fake, width=3, out=fake, cu=fake, pos=fake, slots=fake, state=fake, ws=fake,
             nbytes=need, pool=pool):
        return lib.mc_kv_plan(pool._ref, lens, add, done, seqs, tokens, table, width, out, cu, pos, slots, state, ws, nbytes, None)

    for bad in ({"lens": None}, {"add": None}, {"table": None}, {"out": None}, {"cu": None}, {"state": None}, {"ws": None}, {"lens": 0x100002},
                {"slots": 0x100004}, {"state": 0x100004}, {"ws": 0x100010}, {"nbytes": need - 1}, {"seqs": -1}, {"tokens": -1}, {"width": 0},
                {"seqs": 0}, {"pos": 0x100001}):
        assert call(**bad) == mc.ERR_INVALID_ARG, bad
        assert mc.last_error()
    assert call(tokens=(1 << 30) + 1) == mc.ERR_UNSUPPORTED
    assert call(seqs=0, tokens=0) == mc.OK
    for field, value in (("num_pages", 0), ("page_size", 0), ("page_size", 32769), ("ring", None), ("state", None), ("state", 0x100004)):
        p = mc.KVPool(8, 16, device="cpu")
        setattr(p._c, field, value)
        assert call(pool=p) == mc.ERR_INVALID_ARG, field
    assert lib.mc_kv_plan(None, fake, fake, None, 5, 9, fake, 3, fake, fake, None, None, fake, fake, need, None) == mc.ERR_INVALID_ARG
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    for a in ((i32(5, 3), i32(4), i32(4)), (i32(5, 3), i32(5), i32(4)), (i32(5, 3).float(), i32(5), i32(5)), (i32(5), i32(5), i32(5)),
              (i32(3, 5).T, i32(5), i32(5)), (i32(5, 3), i32(5).long(), i32(5))):
        assert _code(mc, mc.kv_plan, pool, *a) == mc.ERR_INVALID_ARG
    assert _code(mc, mc.kv_plan, pool, i32(5, 3), i32(5), i32(5), done=i32(5)) == mc.ERR_INVALID_ARG
    for kw in ({"ring": i32(7)}, {"ring": torch.zeros(8)}, {"state": i32(2)}, {"state": torch.zeros(3, dtype=torch.int64)}):
        assert _code(mc, mc.KVPool, 8, 16, device="cpu", **kw) == mc.ERR_INVALID_ARG


def test_residual_norms(mc):
    fake, nan, inf = 0x100000, float("nan"), float("inf")

    def call(T=3, H=64, dtype=0, y=fake, h=fake + 4096, ys=64, hs=64, post=fake, pre=fake, gate=None, grow=0, gcol=0, scale=1.0, rs=1.0, eps=1e-5,
             out=fake + 8192, x=fake + 16384, os=64, xs=64):
        a = mc._ResidualC(T, H, dtype, y, h, ys, hs, post, pre, gate, grow, gcol, scale, rs, eps, out, x, os, xs)
        return mc.load().mc_residual_norm(ctypes.addressof(a), None)

    for bad in ({"T": -1}, {"H": 0}, {"eps": nan}, {"eps": -1.0}, {"eps": inf}, {"y": None}, {"h": None}, {"out": None}, {"x": None}, {"y": fake + 1},
                {"pre": fake + 1}, {"ys": 63}, {"hs": 0}, {"os": 63}, {"xs": 63}, {"scale": nan}, {"rs": inf}, {"gate": fake, "gcol": 2},
                {"gate": fake, "grow": -1}, {"gate": fake + 1}, {"x": fake + 8192}, {"x": fake + 4096}):
        assert call(**bad) == mc.ERR_INVALID_ARG, bad
        assert mc.last_error()
    assert call(dtype=2) == mc.ERR_UNSUPPORTED and call(H=65537, ys=65537, hs=65537, os=65537, xs=65537) == mc.ERR_UNSUPPORTED
    assert mc.load().mc_residual_norm(None, None) == mc.ERR_INVALID_ARG
    assert call(T=0, y=None) == mc.OK


def test_residual_rows_in_place_keep_their_stride(mc):
    """Over another operand with another row stride, a row would lie over rows that other blocks still read."""
    y, h, out, x = 0x100000, 0x110000, 0x120000, 0x130000

    def call(T=3, y=y, h=h, out=out, x=x, ys=64, hs=64, os=64, xs=64, pre=y + 0x8000):
        a = mc._ResidualC(T, 64, 0, y, h, ys, hs, None, pre, None, 0, 0, 1.0, 1.0, 1e-5, out, x, os, xs)
        return mc.load().mc_residual_norm(ctypes.addressof(a), None)

    for bad in ({"out": h, "os": 72}, {"out": h, "hs": 72}, {"out": y, "os": 128}, {"out": y, "ys": 65}, {"x": y, "xs": 65}, {"x": y, "ys": 128}):
        assert call(**bad) == mc.ERR_INVALID_ARG, bad
        assert "stride" in mc.last_error()
