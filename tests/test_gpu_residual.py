"""The norms, gate and residual sum between two blocks against their definition in 64 bits."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def mc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2410_06270_gb300 import build
    build.build()
    import paper_2410_06270_gb300 as m
    m.load()
    return m


def _unit(x, gain, eps):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()


def _check(y, h, got_h, got_x, pre, post, gate, scale, rs, eps):
    """h_out: one rounding of a sum formed in fp32 (16 roundings of 2^-24 of the larger of its terms: the norm's sum
    of up to 65536 squares in a tree, its root, four products).  x: one rounding, of a row that is got_h."""
    d = lambda t: t.double().cpu()  # noqa: E731
    half = HALF[y.dtype]
    tiny = 2.0 ** -24 if y.dtype == torch.float16 else 1e-37
    u = d(y) if post is None else _unit(d(y), d(post), eps)
    u = u if gate is None else u * d(gate)
    want = rs * d(h) + scale * u
    size = (rs * d(h)).abs() + (scale * u).abs()
    assert ((d(got_h) - want).abs() <= half * want.abs() + 16 * 2.0 ** -24 * size + tiny).all()
    if pre is not None:
        want = _unit(d(got_h), d(pre), eps)
        assert ((d(got_x) - want).abs() <= (half + 16 * 2.0 ** -24) * want.abs() + tiny).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,H", [(1, 1), (2, 7), (3, 64), (5, 99), (1, 256), (9, 264), (4, 1000), (7, 2048), (3, 2056), (2, 4096), (1, 8192),
                                 (2, 16384), (2, 16392), (1, 65536), (3, 999), (33, 512), (310, 4099),
                                 (304, 2051), (3, 8191), (2, 8193)])
@pytest.mark.parametrize("gate,post,pre", [("none", False, True), ("channel", True, True), ("token", True, False), ("element", False, True)])
def test_matches_its_definition(mc, dtype, T, H, gate, post, pre):
    g = torch.Generator(device="cuda").manual_seed(T * H)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    y, h = 1.5 * r(T, H), 2 * r(T, H)
    shape = {"channel": (1, H), "token": (T, 1), "element": (T, H)}.get(gate)
    gt = torch.sigmoid(r(*shape)) if shape else None
    p1, p2 = ((1 + 0.1 * r(H)) if on else None for on in (post, pre))
    kept = [t.clone() for t in (y, h)]
    got_h, got_x = mc.residual_norm(y, h, pre_norm=p2, post_norm=p1, gate=gt, scale=0.3, residual_scale=0.9, eps=1e-6)
    assert torch.equal(y, kept[0]) and torch.equal(h, kept[1]) and (got_x is None) == (not pre)
    _check(y, h, got_h, got_x, p2, p1, gt, 0.3, 0.9, 1e-6)
    # in place: over the residual and over the block's output
    y2, h2 = y.clone(), h.clone()
    a, b = mc.residual_norm(y2, h2, pre_norm=p2, post_norm=p1, gate=gt, scale=0.3, residual_scale=0.9, eps=1e-6, h_out=h2, x=y2 if pre else None)
    assert a.data_ptr() == h2.data_ptr() and torch.equal(a, got_h) and (not pre or torch.equal(y2, got_x))
    y2 = y.clone()
    a, b = mc.residual_norm(y2, h, pre_norm=p2, post_norm=p1, gate=gt, scale=0.3, residual_scale=0.9, eps=1e-6, h_out=y2)
    assert torch.equal(y2, got_h) and (not pre or torch.equal(b, got_x))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("H,wide,off", [(64, 8, 8), (64, 8, 0), (64, 3, 1), (999, 1, 0), (4096, 64, 32), (4096, 1, 1), (512, 0, 4), (8192, 3, 0),
                                        (16384, 1, 3)])
def test_strides_and_alignments(mc, dtype, H, wide, off):
    """Rows of wider tensors, aligned and not, each operand alike, and what lies beside them is left alone."""
    T = 6
    g = torch.Generator(device="cuda").manual_seed(H + off)
    buf = [torch.randn(T * (H + wide) + off + 8, generator=g, device="cuda").to(dtype) for _ in range(5)]
    kept = [b.clone() for b in buf]
    rows = [b[off:off + T * (H + wide)].view(T, H + wide)[:, :H] for b in buf]
    y, h, gate, h_out, x = rows
    vec = torch.randn(2, H + 40, generator=g, device="cuda").to(dtype)
    pre, post = vec[0, off:off + H], vec[1, off:off + H]
    mc.residual_norm(y, h, pre_norm=pre, post_norm=post, gate=gate, h_out=h_out, x=x)
    _check(y, h, h_out, x, pre, post, gate, 1.0, 1.0, 1e-5)
    for i, b in enumerate(buf):
        outside = torch.ones_like(b, dtype=torch.bool)
        if i > 2:
            outside[off:off + T * (H + wide)].view(T, H + wide)[:, :H] = False
        assert torch.equal(b[outside], kept[i][outside])
    # the wide accesses and the narrow ones give the same
    a, b = mc.residual_norm(y.contiguous(), h.contiguous(), pre_norm=pre.clone(), post_norm=post.clone(), gate=gate.contiguous())
    if H % 8 == 0:
        assert torch.equal(a, h_out) and torch.equal(b, x)


@pytest.mark.parametrize("which", range(7))
def test_one_operand_off_its_alignment(mc, which):
    """The others keep their wide accesses; the result is that of aligned copies, bit for bit."""
    T, H = 5, 1000
    g = torch.Generator(device="cuda").manual_seed(3)
    full = [torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16) for _ in range(3)] + [torch.randn(H, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    y, h, gate, post, pre = full
    want = mc.residual_norm(y, h, pre_norm=pre, post_norm=post, gate=gate)
    outs = [torch.empty_like(y), torch.empty_like(y)]
    ops = full + outs
    odd = torch.empty(ops[which].numel() + 1, dtype=torch.bfloat16, device="cuda")[1:].view(ops[which].shape)
    ops[which] = odd.copy_(ops[which])
    y, h, gate, post, pre, a, b = ops
    got = mc.residual_norm(y, h, pre_norm=pre, post_norm=post, gate=gate, h_out=a, x=b)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("T,H", [(5, 64), (3, 256), (4, 1000), (2, 4096), (3, 8192), (2, 16392), (3, 77)])
def test_is_add_and_rmsnorm(mc, T, H):
    """Without gate and scales, the library's own add and rmsnorm, bit for bit."""
    g = torch.Generator(device="cuda").manual_seed(H)
    y, h = (torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    pre = torch.randn(H, generator=g, device="cuda").to(torch.bfloat16)
    a, b = mc.residual_norm(y, h, pre_norm=pre)
    want = mc.add(h, y)
    assert torch.equal(a, want) and torch.equal(b, mc.rmsnorm(want, pre))


def test_values_that_are_not_finite_and_rows_of_zero(mc):
    """NaN and infinities stay in their rows; a row of zeros is zeros, whatever eps makes of it."""
    y, h = torch.randn(6, 512, device="cuda").to(torch.bfloat16), torch.randn(6, 512, device="cuda").to(torch.bfloat16)
    one = torch.ones(512, dtype=torch.bfloat16, device="cuda")
    clean = mc.residual_norm(y, h, pre_norm=one, post_norm=one)
    y[1, 7], h[3, 500] = float("nan"), float("inf")
    a, b = mc.residual_norm(y, h, pre_norm=one, post_norm=one)
    for r in (0, 2, 4, 5):
        assert torch.equal(a[r], clean[0][r]) and torch.equal(b[r], clean[1][r])
    assert torch.isnan(a[1]).all() and torch.isnan(b[1]).all()
    assert torch.isinf(a[3, 500]) and torch.equal(a[3, :500], clean[0][3, :500]) and torch.isnan(b[3, 500]) and (b[3, :500] == 0).all()
    z = torch.zeros(2, 512, dtype=torch.bfloat16, device="cuda")
    a, b = mc.residual_norm(z, z, pre_norm=one, post_norm=one, eps=1e-5)
    assert (a == 0).all() and (b == 0).all()


def test_many_rows_a_stream_and_a_graph(mc):
    """Rows past 2^31 elements, another stream, a replayed graph with new inputs."""
    T, H = 300_000, 8192
    y = torch.randn(T, H, device="cuda", dtype=torch.bfloat16)
    one = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    h = torch.zeros(1, H, dtype=torch.bfloat16, device="cuda").expand(T, H).contiguous()
    a, b = mc.residual_norm(y, h, pre_norm=one, h_out=h)
    assert torch.equal(a[-5:], y[-5:]) and torch.equal(b[-5:], mc.rmsnorm(y[-5:].contiguous(), one))
    del y, h, a, b
    y, h = (torch.randn(16, 4096, device="cuda").to(torch.bfloat16) for _ in range(2))
    one = one[:4096]
    want = mc.residual_norm(y, h, pre_norm=one)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = mc.residual_norm(y, h, pre_norm=one)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = mc.residual_norm(y, h, pre_norm=one)
    y.mul_(2)
    graph.replay()
    want = mc.residual_norm(y, h, pre_norm=one)
    assert torch.equal(res[0], want[0]) and torch.equal(res[1], want[1])


@pytest.mark.parametrize("H", [64, 999, 4096, 20000])
def test_in_place_over_strided_rows(mc, H):
    """Over rows of a wider tensor with its stride, what comes out apart; over them with another stride, nothing."""
    g = torch.Generator(device="cuda").manual_seed(H)
    T = 40
    y, h = (torch.randn(T, H + 24, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    pre, post = (torch.randn(H, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    kept = [t.clone() for t in (y, h)]
    want = mc.residual_norm(y[:, :H], h[:, :H], pre_norm=pre, post_norm=post)
    for over in ({"h_out": h[:, :H], "x": y[:, :H]}, {"h_out": y[:, :H]}):
        y.copy_(kept[0]), h.copy_(kept[1])
        got = mc.residual_norm(y[:, :H], h[:, :H], pre_norm=pre, post_norm=post, **over)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(y[:, H:], kept[0][:, H:]) and torch.equal(h[:, H:], kept[1][:, H:])
    y.copy_(kept[0]), h.copy_(kept[1])
    flat = [t.view(-1)[:T * H].view(T, H) for t in (y, h)]  # the same first element, rows nearer together
    for over in ({"h_out": flat[1]}, {"h_out": flat[0]}, {"x": flat[0]}):
        with pytest.raises(mc.MCError) as e:
            mc.residual_norm(y[:, :H], h[:, :H], pre_norm=pre, post_norm=post, **over)
        assert e.value.code == mc.ERR_INVALID_ARG
    assert torch.equal(y, kept[0]) and torch.equal(h, kept[1])
    one = mc.residual_norm(y[:1, :H], h[:1, :H], pre_norm=pre, post_norm=post, h_out=flat[1][:1], x=flat[0][:1])
    assert all(torch.equal(a, b[:1]) for a, b in zip(one, want))
