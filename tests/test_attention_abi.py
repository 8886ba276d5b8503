"""What the paged cache's entry points refuse, on the host, before any device work."""
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
    k, v = (torch.zeros(pages, kv, page, dim, dtype=dtype) for _ in range(2))
    cache = mc.KVCache(k, v)
    batch = mc.KVBatch(torch.ones(seqs, dtype=torch.int32), torch.zeros(seqs, width, dtype=torch.int32))
    return cache, batch


def _code(mc, fn, *a, **k):
    with pytest.raises(mc.MCError) as e:
        fn(*a, **k)
    assert str(e.value)
    return e.value.code


@pytest.mark.parametrize("field,value,code", [
    ("head_dim", 96, -2), ("dtype", 2, -2), ("page_size", 8, -1), ("page_size", 24, -1), ("page_size", 1 << 16, -1),
    ("num_pages", 0, -1), ("kv_heads", 0, -1), ("kv_heads", 3, -1), ("page_stride", 2 * 16 * 64 - 8, -1),
    ("page_stride", 2 * 16 * 64 + 4, -1)])
def test_bad_caches(mc, field, value, code):
    cache, batch = _cpu(mc)
    setattr(cache._c, field, value)
    assert mc.load().mc_attn_workspace_size(cache._ref, 4) == 0
    assert mc.last_error()
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    lib = mc.load()
    opts = mc._AttnOptsC(0.1, 0.0, 0, None, None)
    for fn in (lib.mc_attn_decode, lib.mc_attn_prefill):
        assert fn(cache._ref, batch._ref, q.data_ptr(), 256, 4, ctypes.addressof(opts), q.data_ptr(), 256, None,
                  q.data_ptr(), 1 << 30, None) == code
    assert lib.mc_kv_append(cache._ref, batch._ref, q.data_ptr(), 256, q.data_ptr(), 256, q.data_ptr(), 256, 4, None,
                            None, 1e-6, None, 0, 0, 0, q.data_ptr(), None, None) == code


def test_binding_refuses_what_c_cannot_see(mc):
    cache, batch = _cpu(mc)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    kv = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    assert _code(mc, mc.KVCache, cache.k.float(), cache.v.float()) == mc.ERR_UNSUPPORTED
    assert _code(mc, mc.KVCache, cache.k, cache.v[:3]) == -1
    assert _code(mc, mc.KVCache, cache.k.transpose(1, 2), cache.v.transpose(1, 2)) == -1
    assert _code(mc, mc.KVBatch, torch.ones(3), torch.zeros(3, 2, dtype=torch.int32)) == -1
    assert _code(mc, mc.KVBatch, torch.ones(3, dtype=torch.int64), torch.zeros(3, 2, dtype=torch.int32)) == -1
    assert _code(mc, mc.KVBatch, torch.ones(3, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32)) == -1
    assert _code(mc, mc.KVBatch, torch.ones(3, dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32),
                 torch.zeros(3, dtype=torch.int32), 3) == -1
    assert _code(mc, mc.KVBatch, torch.ones(3, dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32),
                 torch.zeros(4, dtype=torch.int32)) == -1
    for bad in (q.half(), q[:2], q[:, :, :32], q.transpose(0, 1), q.flatten(1),
                torch.zeros(3, 64, 4, dtype=torch.bfloat16).transpose(1, 2)):
        assert _code(mc, mc.attn_decode, cache, batch, bad, workspace=ws) == -1
        assert _code(mc, mc.kv_append, cache, batch, bad, kv, kv, workspace=ws) == -1
    assert _code(mc, mc.kv_append, cache, batch, q, q, kv) == -1       # four heads of keys
    assert _code(mc, mc.kv_append, cache, batch, q, kv, kv, q_norm=torch.ones(32, dtype=torch.bfloat16)) == -1
    assert _code(mc, mc.kv_append, cache, batch, q, kv, kv, k_norm=torch.ones(64)) == -1
    assert _code(mc, mc.kv_append, cache, batch, q, kv, kv, rope=torch.zeros(10, 64, dtype=torch.float64)) == -1
    assert _code(mc, mc.kv_append, cache, batch, q, kv, kv, workspace=torch.zeros(2, dtype=torch.uint8)) == -1
    assert _code(mc, mc.attn_decode, cache, batch, q, slopes=torch.zeros(3), workspace=ws) == -1
    assert _code(mc, mc.attn_prefill, cache, batch, q, prefix=torch.zeros(3), workspace=ws) == -1


def _aligned(n):
    t = torch.zeros(n + 256, dtype=torch.uint8)
    return t[-t.data_ptr() % 256:][:n]


def test_host_tensors_and_other_devices_are_refused(mc, monkeypatch):
    """Before anything is launched: the answer is an argument error, not a launch's."""
    cache, batch = _cpu(mc)
    q, kv = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    ws = _aligned(mc.load().mc_attn_workspace_size(cache._ref, 4))
    assert _code(mc, mc.kv_append, cache, batch, q, kv, kv) == mc.ERR_INVALID_ARG
    assert _code(mc, mc.kv_append, cache, batch, q, kv, kv, q_out=torch.empty_like(q), workspace=ws) == mc.ERR_INVALID_ARG
    for fn in (mc.attn_decode, mc.attn_prefill):
        assert _code(mc, fn, cache, batch, q, workspace=ws) == mc.ERR_INVALID_ARG

    class Elsewhere:  # a torch whose current device is not the tensors'
        class cuda:
            current_device = staticmethod(lambda: 0)

        def __getattr__(self, name):
            return getattr(torch, name)

    monkeypatch.setattr(mc, "_torch", lambda: Elsewhere())
    for where, refused in ((1, True), (0, False)):
        cache.index = where
        if refused:
            assert _code(mc, mc._on_current, cache) == mc.ERR_INVALID_ARG
        else:
            mc._on_current(cache)


@pytest.mark.parametrize("window,c_window", [(0, 0), (5, 5), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (2 ** 32, 2 ** 31 - 1),
                                             (2 ** 32 + 5, 2 ** 31 - 1), (-1, -1), (-2 ** 32, -1), (-2 ** 32 + 7, -1)])
def test_a_window_beyond_32_bits_is_no_shorter_one(mc, monkeypatch, window, c_window):
    """It reaches the C call (a stand-in for it here) as the longest window, and a negative one as
    one that is refused."""
    seen = []
    cache, batch = _cpu(mc)
    q, ws = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(1 << 10, dtype=torch.uint8)

    class Lib:
        def mc_attn_decode(self, *a):
            seen.append(mc._AttnOptsC.from_address(a[5]).window)
            return mc.OK

        mc_attn_prefill = mc_attn_decode

    monkeypatch.setattr(mc, "_fast_module", type("NotPlain", (), {"attention": staticmethod(lambda *a: None)}))
    monkeypatch.setattr(mc, "load", Lib)
    monkeypatch.setattr(mc, "_stream", lambda: 0)
    monkeypatch.setattr(mc, "_on_current", lambda cache: None)
    for fn in (mc.attn_decode, mc.attn_prefill):
        fn(cache, batch, q, window=window, workspace=ws)
    assert seen == [c_window] * 2


@pytest.mark.parametrize("scale,cap", [(0.0, 0.0), (-1.0, 0.0), (1e-30, 0.0), (1e30, 0.0), (1.0, 1e-30), (1.0, 1e30), (1e30, 1e-30)])
def test_scales_and_caps_out_of_range(mc, scale, cap):
    cache, batch = _cpu(mc)
    opts, fake = mc._AttnOptsC(scale, cap, 0, None, None), 0x100000
    need = mc.load().mc_attn_workspace_size(cache._ref, 4)
    for fn in (mc.load().mc_attn_decode, mc.load().mc_attn_prefill):
        assert fn(cache._ref, batch._ref, fake, 256, 4, ctypes.addressof(opts), fake, 256, None, fake, need, None) == mc.ERR_INVALID_ARG


def test_bad_options_and_pointers(mc):
    cache, batch = _cpu(mc)
    lib, need = mc.load(), mc.load().mc_attn_workspace_size(cache._ref, 4)
    assert need > 0
    fake, odd = 0x100000, 0x100008  # never dereferenced: every call below is refused

    def attn(fn=lib.mc_attn_decode, q=fake, qs=256, heads=4, out=fake, os=256, lse=None, ws=fake, nbytes=need,
             scale=0.1, cap=0.0, window=0, prefix=None, cache=cache, batch=batch):
        opts = mc._AttnOptsC(scale, cap, window, None, prefix)
        return fn(cache._ref, batch._ref, q, qs, heads, ctypes.addressof(opts), out, os, lse, ws, nbytes, None)

    nan, inf = float("nan"), float("inf")
    for bad in ({"q": None}, {"q": odd}, {"qs": 248}, {"qs": 260}, {"heads": 3}, {"heads": 0}, {"heads": 4098}, {"out": None},
                {"out": odd}, {"os": 255}, {"lse": 0x100002}, {"ws": None}, {"ws": 0x100010}, {"nbytes": need - 1},
                {"scale": nan}, {"scale": inf}, {"cap": -1.0}, {"cap": nan}, {"cap": inf}, {"window": -1}, {"prefix": fake}):
        assert attn(**bad) == mc.ERR_INVALID_ARG, bad
        assert mc.last_error()
        if "prefix" not in bad:
            assert attn(fn=lib.mc_attn_prefill, **bad) == mc.ERR_INVALID_ARG, bad
    assert attn(fn=lib.mc_attn_prefill, prefix=0x100001) == mc.ERR_INVALID_ARG
    _, ragged = _cpu(mc)
    ragged._c.cu_q = fake
    assert attn(batch=ragged) == mc.ERR_INVALID_ARG  # decode takes one token per sequence
    for field, value in (("seqs", -1), ("tokens", -1), ("tokens", 4), ("lens", None), ("table", None), ("table_width", 0)):
        _, b = _cpu(mc)
        setattr(b._c, field, value)
        assert attn(batch=b) == mc.ERR_INVALID_ARG, field
    assert lib.mc_attn_decode(None, batch._ref, fake, 256, 4, fake, fake, 256, None, fake, need, None) == mc.ERR_INVALID_ARG
    assert lib.mc_attn_decode(cache._ref, None, fake, 256, 4, fake, fake, 256, None, fake, need, None) == mc.ERR_INVALID_ARG
    assert lib.mc_attn_decode(cache._ref, batch._ref, fake, 256, 4, None, fake, 256, None, fake, need, None) == mc.ERR_INVALID_ARG
    # nothing to do: no pointer is looked at
    _, none = _cpu(mc, seqs=0)
    assert attn(batch=none, q=None, out=None, ws=None, nbytes=0) == mc.OK

    def append(q=fake, qs=256, k=fake, ks=128, v=fake, vs=128, heads=4, qn=None, kn=None, eps=1e-6, rope=None, rows=0,
               rot=0, out=fake, ws=None):
        return lib.mc_kv_append(cache._ref, batch._ref, q, qs, k, ks, v, vs, heads, qn, kn, eps, rope, rows, rot, 0, out,
                                ws, None)

    for bad in ({"q": None}, {"k": odd}, {"v": None}, {"qs": 128}, {"ks": 100}, {"vs": 129}, {"heads": 5}, {"qn": 0x100004},
                {"kn": 0x100002}, {"eps": nan}, {"eps": -1.0}, {"rot": 8, "rope": fake, "rows": 9}, {"rot": 80, "rope": fake, "rows": 9},
                {"rot": -16}, {"rot": 16}, {"rot": 16, "rope": fake}, {"rot": 16, "rope": odd, "rows": 9}, {"out": None},
                {"out": odd}, {"ws": 0x100001}):
        assert append(**bad) == mc.ERR_INVALID_ARG, bad


@pytest.mark.parametrize("seqs,tokens,width,heads", [
    (1, 1 << 20, 1 << 20, 4096),          # 2^24 row tiles over 2^17 units
    (1 << 24, 1 << 24, 1 << 22, 4),       # long tables of many sequences
    (1, (1 << 30) + 1, 1, 2),
    ((1 << 30) + 1, 1, 1, 2)])
def test_more_work_than_the_schedule_counts(mc, seqs, tokens, width, heads):
    cache, batch = _cpu(mc)
    fake, need = 0x100000, mc.load().mc_attn_workspace_size(cache._ref, heads)
    batch._c.seqs, batch._c.tokens, batch._c.table_width, batch._c.cu_q = seqs, tokens, width, fake
    opts = mc._AttnOptsC(0.1, 0.0, 0, None, None)
    assert mc.load().mc_attn_prefill(cache._ref, batch._ref, fake, heads * 64, heads, ctypes.addressof(opts), fake, heads * 64,
                                     None, fake, need, None) == mc.ERR_UNSUPPORTED
    assert mc.last_error()
