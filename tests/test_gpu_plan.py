"""Block tables and slots from lengths against a sequential account of the pool: growth, finished sequences, shortage
of pages and of rows, unsound inputs, many sequences, steps one after the other, graphs."""
import random

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2410_06270_gb300 import build
    build.build()
    import paper_2410_06270_gb300 as m
    m.load()
    return m


class Account:
    """The pool and the tables on the host, a sequence at a time."""

    def __init__(self, seqs, width, pages, page, seed, start=0):
        rng = random.Random(seed)
        order = list(range(pages))
        rng.shuffle(order)
        self.page, self.width, self.cap = page, width, pages
        self.ring = [order[(i - start) % pages] for i in range(pages)]
        self.taken, self.returned = start, start + pages
        self.table = [[-5] * width for _ in range(seqs)]
        self.lens = [0] * seqs

    def pages(self, n):
        return -(-n // self.page)

    def step(self, add, done, tokens):
        """Returns (cu_q, positions, slots, whether all were served)."""
        fine, free = True, self.returned - self.taken
        end = self.taken + self.cap
        for b, over in enumerate(done or [0] * len(add)):
            if over:
                for p in self.table[b][:min(self.width, self.pages(max(0, self.lens[b])))]:
                    if self.returned < end:
                        self.ring[self.returned % self.cap] = p
                        self.returned += 1
                    else:
                        fine = False
                    fine &= 0 <= p < self.cap
                self.lens[b] = 0
        cu, positions, slots, asked, rows, took = [0], [], [], 0, 0, 0
        for b, n in enumerate(add):
            length = self.lens[b] = max(0, self.lens[b])
            if n < 0 or length + n > min(self.width * self.page, 1 << 30):
                fine, n = False, 0
            else:
                need = self.pages(length + n) - self.pages(length)
                asked, rows = asked + need, rows + n
                if (need and asked > free) or (n and rows > tokens):
                    fine, n = False, 0
                elif need:
                    for i in range(need):
                        self.table[b][self.pages(length) + i] = self.ring[(self.taken + asked - need + i) % self.cap]
                    took = asked
            for pos in range(length, length + n):
                p = self.table[b][pos // self.page]
                positions.append(pos)
                slots.append(p * self.page + pos % self.page if 0 <= p < self.cap else -1)
                fine &= 0 <= p < self.cap
            self.lens[b] += n
            cu.append(cu[-1] + n)
        self.taken += took
        pad = [-1] * (tokens - len(slots))
        return cu, positions + pad, slots + pad, fine


class Device:
    def __init__(self, mc, a):
        t = lambda v, d=torch.int32: torch.tensor(v, dtype=d, device="cuda")  # noqa: E731
        self.mc, self.t = mc, t
        self.table, self.lens = t(a.table), t(a.lens)
        self.pool = mc.KVPool(a.cap, a.page, ring=t(a.ring), state=t([a.taken, a.returned], torch.int64))
        self.ws = mc.kv_plan_workspace(len(a.lens))

    def step(self, add, done, tokens, **kw):
        done = None if done is None else self.t(done, torch.uint8)
        return self.mc.kv_plan(self.pool, self.table, self.lens, self.t(add), done=done, tokens=tokens, lens_out=self.lens, workspace=self.ws, **kw)

    def fine(self):
        try:
            self.mc.check_status(self.ws)
            return True
        except self.mc.MCError as e:
            assert e.code == self.mc.ERR_RANGE
            return False

    def same(self, a, plan, want):
        cu, positions, slots, fine = want
        assert plan.cu_q.tolist() == cu and plan.positions.tolist() == positions and plan.slots.tolist() == slots
        assert plan.lens.tolist() == a.lens and self.table.tolist() == a.table
        assert self.pool.state.tolist() == [a.taken, a.returned] and self.pool.ring.tolist() == a.ring
        assert self.fine() == fine


@pytest.mark.parametrize("seqs,width,pages,page,start,prompt", [
    (1, 1, 1, 16, 0, 16), (3, 4, 20, 16, 5, 40), (40, 8, 200, 16, (1 << 33) + 7, 60), (7, 3, 9, 48, 100, 90),
    (1025, 5, 3000, 16, 3, 20), (250, 40, 1500, 7, 0, 150), (2500, 3, 4000, 32, 1 << 40, 3)])
def test_steps_one_after_the_other(mc, seqs, width, pages, page, start, prompt):
    """A server's life: prompts, single tokens, finished ones replaced, pages running short now and then."""
    a = Account(seqs, width, pages, page, 1, start)
    d = Device(mc, a)
    rng = random.Random(2)
    for i in range(8):
        done = None if i == 0 else [int(rng.random() < 0.2) for _ in range(seqs)]
        add = [rng.choice([0, 1, 1, rng.randint(1, prompt)]) for _ in range(seqs)]
        tokens = sum(add) if i % 3 else max(0, sum(add) - rng.randint(0, 9)) + rng.choice([0, 5])
        plan = d.step(add, done, tokens)
        d.same(a, plan, a.step(add, done, tokens))


@pytest.mark.parametrize("seqs,tokens", [(5, 4096), (5, 4097), (1024, 3000), (1025, 3000), (3, 70000)])
def test_one_launch_and_two(mc, seqs, tokens):
    """On both sides of the sizes that one block does by itself."""
    each = tokens // seqs
    a = Account(seqs, each // 16 + 2, seqs * (each // 16 + 2), 16, 4)
    d = Device(mc, a)
    for done in (None, [b % 2 for b in range(seqs)], None):
        add = [each - (5 if b % 3 else 0) for b in range(seqs)] if done != [] else []
        d.same(a, d.step(add, done, tokens), a.step(add, done, tokens))


@pytest.mark.parametrize("short", [None, "pages", "rows"])
@pytest.mark.parametrize("seqs", [4095, 4096, 4097, 8193, 9000])
def test_more_sequences_than_a_block_takes_at_a_time(mc, seqs, short):
    """Sums that go on from one round of 4096 sequences to the next: finished ones on both sides of its border, and pages
    or rows that run short behind it (with fewer sequences: at the last ones)."""
    rng = random.Random(seqs)
    first = [rng.randint(0, 40) for _ in range(seqs)]
    add = [rng.choice([0, 1, 17, 30]) for _ in range(seqs)]
    done = [int(rng.random() < 0.2 or b in (0, 4095, 4096, 8191, 8192, seqs - 1)) for b in range(seqs)]
    pages = lambda n: -(-n // 16)  # noqa: E731
    from_ = 4096 + (seqs - 4096) // 2 if seqs > 5000 else seqs - 3  # whose claim is the last that is met
    need = sum(pages((0 if o else n) + m) - (0 if o else pages(n)) for n, m, o in list(zip(first, add, done))[:from_])
    held = sum(map(pages, first))
    a = Account(seqs, 5, held + (need if short == "pages" else 3 * seqs), 16, 47, 5)
    d = Device(mc, a)
    d.same(a, d.step(first, None, sum(first)), a.step(first, None, sum(first)))
    tokens = sum(add[:from_]) if short == "rows" else sum(add) + 9
    plan, want = d.step(add, done, tokens), a.step(add, done, tokens)
    assert want[3] == (short is None)
    d.same(a, plan, want)
    add = [b % 2 for b in range(seqs)]
    d.same(a, d.step(add, None, seqs), a.step(add, None, seqs))


def test_what_does_not_fit_is_refused_in_order(mc):
    # three pages free: the first takes two, the second wants two and gets none, the third needs none, the fourth
    # wants one more than are left after the second's claim
    a = Account(4, 4, 6, 16, 7)
    d = Device(mc, a)
    d.same(a, d.step([0, 0, 20, 10], None, 64), a.step([0, 0, 20, 10], None, 64))
    plan = d.step([32, 17, 5, 10], None, 64)
    want = a.step([32, 17, 5, 10], None, 64)
    assert want[0] == [0, 32, 32, 37, 37] and not want[3]
    d.same(a, plan, want)
    # rows of the token arrays
    plan, want = d.step([1, 1, 1, 1], None, 2), a.step([1, 1, 1, 1], None, 2)
    d.same(a, plan, want)
    # negative counts and lengths, a table row's end
    for add in ([-1, 0, 1, -2 ** 31], [100, 2 ** 31 - 1, 1, 0]):
        d.same(a, d.step(add, None, 200), a.step(add, None, 200))
    a.lens[1] = -7
    d.lens[1] = -7
    d.same(a, d.step([0, 3, 0, 0], [0, 0, 0, 1], 8), a.step([0, 3, 0, 0], [0, 0, 0, 1], 8))


def test_unsound_pages_and_a_full_ring(mc):
    """A page outside the pool is no slot; more pages than the ring holds do not come back."""
    a = Account(2, 3, 4, 16, 9)
    d = Device(mc, a)
    d.same(a, d.step([20, 5], None, 25), a.step([20, 5], None, 25))
    for bad in (4, -1, 2 ** 31 - 1):
        a.table[1][0] = bad
        d.table[1, 0] = bad
        d.same(a, d.step([1, 1], None, 2), a.step([1, 1], None, 2))
    # a length beyond what was ever taken: its row names three pages, the ring has room for what is missing from it
    a.lens[0], a.table[0] = 48, [0, 1, 2]
    d.lens[0] = 48
    d.table[0] = torch.tensor([0, 1, 2])
    a.table[1][0] = d.table[1, 0] = 3
    d.same(a, d.step([0, 0], [1, 1], 0), a.step([0, 0], [1, 1], 0))
    # a ring of nonsense stays in bounds
    d.pool.ring.fill_(-1)
    a.ring = [-1] * 4
    d.same(a, d.step([5, 0], None, 5), a.step([5, 0], None, 5))
    d.pool.state.copy_(torch.tensor([-3, 2 ** 62]))
    d.step([16, 16], [1, 1], 32)
    torch.cuda.synchronize()
    d.fine()


def test_a_preview_changes_nothing_but_may_be_repeated(mc):
    a = Account(6, 4, 30, 16, 11)
    d = Device(mc, a)
    d.same(a, d.step([10, 20, 30, 1, 0, 64], None, 130), a.step([10, 20, 30, 1, 0, 64], None, 130))
    add, done = d.t([7, 0, 40, 1, 1, 0]), d.t([0, 1, 0, 0, 0, 0], torch.uint8)
    lens, state = d.lens.clone(), d.pool.state.clone()
    plans = [mc.kv_plan(d.pool, d.table, d.lens, add, done=done, tokens=50, commit=False, workspace=d.ws) for _ in range(3)]
    assert torch.equal(d.lens, lens) and torch.equal(d.pool.state, state)
    for p in plans[1:]:
        for name in ("lens", "cu_q", "positions", "slots", "state"):
            assert torch.equal(getattr(p, name), getattr(plans[0], name))
    want = a.step([7, 0, 40, 1, 1, 0], [0, 1, 0, 0, 0, 0], 50)
    p = mc.kv_plan(d.pool, d.table, d.lens, add, done=done, tokens=50, lens_out=d.lens, workspace=d.ws)
    d.same(a, p, want)
    assert plans[0].state.tolist() == [a.taken, a.returned]
    only = mc.kv_plan(d.pool, d.table, d.lens, add, tokens=50, positions=False, slots=False, commit=False)
    assert only.positions is None and only.slots is None


REPLACED = [  # prompts of the first step, width, pages, page, new tokens of the second, done
    ([40, 20], 4, 8, 16, [20, 1], [1, 0]),
    ([40, 20, 7], 4, 16, 16, [64, 3, 0], [1, 0, 1]),          # longer and shorter than what was there
    ([2100, 3000, 40], 200, 700, 16, [3000, 1, 1500], [1, 0, 1]),  # two launches
    ([1 + b % 30 for b in range(1100)], 4, 5000, 16, [1 + b % 40 for b in range(1100)], [b % 3 == 0 for b in range(1100)])]


@pytest.mark.parametrize("previews", [1, 2])
@pytest.mark.parametrize("first,width,pages,page,add,done", REPLACED)
def test_a_preview_of_replaced_sequences_may_be_repeated_and_committed(mc, first, width, pages, page, add, done, previews):
    """A finished sequence whose place another takes in the same step: its pages are read from its row, which a call that
    does not commit leaves as it is."""
    a = Account(len(first), width, pages, page, 41)
    d = Device(mc, a)
    d.same(a, d.step(first, None, sum(first)), a.step(first, None, sum(first)))
    t_add, t_done, tokens = d.t(add), d.t([int(x) for x in done], torch.uint8), sum(add) + 3
    rows, old = d.t(done) != 0, d.table.clone()
    seen = [mc.kv_plan(d.pool, d.table, d.lens, t_add, done=t_done, tokens=tokens, commit=False, workspace=d.ws) for _ in range(previews)]
    assert torch.equal(d.table[rows], old[rows])
    with pytest.raises(mc.MCError) as e:  # (its table would name the pages that go back)
        seen[0].batch
    assert e.value.code == mc.ERR_INVALID_ARG
    want = a.step(add, done, tokens)
    plan = d.step(add, [int(x) for x in done], tokens)
    d.same(a, plan, want)
    for p in seen:
        for name in ("lens", "cu_q", "positions", "slots"):
            assert torch.equal(getattr(p, name), getattr(plan, name))
        assert p.state.tolist() == [a.taken, a.returned]
    free = [a.ring[i % pages] for i in range(a.taken, a.returned)]
    held = [p for b, n in enumerate(a.lens) for p in a.table[b][:a.pages(n)]]
    assert sorted(free + held) == list(range(pages))
    assert torch.equal(plan.batch._keep[1], d.table)


def test_counts_apart_with_lengths_in_place_are_a_step(mc):
    """A caller that keeps two sets of counts in turn and its lengths in place: rows of replaced sequences are entered."""
    a = Account(2, 4, 8, 16, 45)
    d = Device(mc, a)
    d.same(a, d.step([40, 20], None, 60), a.step([40, 20], None, 60))
    want = a.step([20, 1], [1, 0], 21)
    plan = d.step([20, 1], [1, 0], 21, commit=False)
    assert torch.equal(plan.batch._keep[1], d.table)
    d.pool.state.copy_(plan.state)
    d.same(a, plan, want)


def test_a_preview_that_is_dropped_leaves_the_sequence_whole(mc):
    """Looked at as finished and replaced, then gone on with after all."""
    a = Account(3, 8, 20, 16, 43)
    d = Device(mc, a)
    d.same(a, d.step([40, 20, 16], None, 76), a.step([40, 20, 16], None, 76))
    mc.kv_plan(d.pool, d.table, d.lens, d.t([90, 1, 1]), done=d.t([1, 0, 1], torch.uint8), tokens=92, commit=False, workspace=d.ws)
    assert d.fine()
    cu, positions, slots, fine = a.step([9, 13, 1], None, 23)
    plan = d.step([9, 13, 1], None, 23)
    assert plan.cu_q.tolist() == cu and plan.positions.tolist() == positions and plan.slots.tolist() == slots and d.fine() == fine
    assert plan.lens.tolist() == a.lens and d.pool.state.tolist() == [a.taken, a.returned]
    for b, n in enumerate(a.lens):
        assert d.table[b, :a.pages(n)].tolist() == a.table[b][:a.pages(n)]
    ring = d.pool.ring.tolist()
    assert [ring[i % 20] for i in range(a.taken, a.returned)] == [a.ring[i % 20] for i in range(a.taken, a.returned)]


def test_a_step_without_sequences(mc):
    pool = mc.KVPool(4, 16)
    none, table = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, 3, dtype=torch.int32, device="cuda")
    p = mc.kv_plan(pool, table, none, none, commit=False)
    assert p.cu_q.tolist() == [0] and p.state.tolist() == [0, 4] and p.lens.numel() == 0 == p.slots.numel()


def test_another_stream_and_other_sizes_through_one_workspace(mc):
    """Steps of one launch and of two in turn, on a stream of their own."""
    a = Account(1500, 40, 9000, 16, 19)
    d = Device(mc, a)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for add in ([1] * 1500, [3 + b % 5 for b in range(1500)], [1] * 1500):
            want = a.step(add, None, sum(add))
            plan = d.step(add, None, sum(add))
            s.synchronize()
            d.same(a, plan, want)
    b = Account(5, 40, 300, 16, 23)
    e = Device(mc, b)
    e.ws = d.ws  # (one for up to 1500 sequences)
    for add in ([600] * 5, [1] * 5):
        e.same(b, e.step(add, None, sum(add)), b.step(add, None, sum(add)))


def test_a_workspace_of_the_attentions_serves_the_plan_too(mc):
    """Its status word, and a count that they keep between calls, stay what they are."""
    g = torch.Generator().manual_seed(31)
    pools = [torch.zeros(300, 2, mc.kv4_block_size(16, 64), dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = mc.KVCache4(*pools, 16, 64)
    ws = mc.attn4_workspace(cache, 32, prompts=False)
    a = Account(1, 256, 300, 16, 29)
    d = Device(mc, a)
    d.ws = ws
    outs = []
    x = [torch.randn(4200, n, 64, generator=g).to(torch.bfloat16).cuda() for n in (32, 2, 2)]
    for _ in range(3):  # a prompt of many items, which a common count deals, after a plan of two launches
        a.lens[0], a.taken, a.returned = 0, 0, 300
        d.lens.zero_(), d.pool.state.copy_(torch.tensor([0, 300]))
        want = a.step([4000], None, 4200)
        plan = d.step([4000], None, 4200)
        d.same(a, plan, want)
        batch = mc.KVBatch(plan.lens, d.table, plan.cu_q, 4200)
        q = mc.kv4_append(cache, batch, *x, workspace=ws)
        outs.append(mc.attn4_prefill(cache, batch, q, workspace=ws)[:4000].clone())
        mc.check_status(ws)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_replayed_steps(mc):
    """A captured step, in place, replayed: each replay is the next step."""
    a = Account(20, 6, 200, 16, 13)
    d = Device(mc, a)
    add, done = [1 + b % 3 for b in range(20)], [int(b == 4) for b in range(20)]
    t_add, t_done = d.t(add), d.t(done, torch.uint8)
    call = lambda: mc.kv_plan(d.pool, d.table, d.lens, t_add, done=t_done, tokens=64, lens_out=d.lens, workspace=d.ws)  # noqa: E731
    want = a.step(add, done, 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        plan = call()
    s.synchronize()
    d.same(a, plan, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        plan = call()
    for _ in range(3):
        want = a.step(add, done, 64)
        g.replay()
        torch.cuda.synchronize()
        d.same(a, plan, want)


def test_a_plan_serves_the_cache(mc):
    """Appends and attentions over a plan's tables, prompts then single tokens, against one over a table by hand;
    the slots name the rows that the append writes."""
    heads, kv, dim, page, seqs = 4, 2, 64, 16, 5
    g = torch.Generator().manual_seed(3)
    a = Account(seqs, 8, 64, page, 17)
    d = Device(mc, a)
    pools = [torch.zeros(64, kv, mc.kv4_block_size(page, dim), dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = mc.KVCache4(*pools, page, dim)
    own = mc.KVCache4(*(torch.zeros_like(p) for p in pools), page, dim)
    table = torch.arange(seqs * 8, dtype=torch.int32, device="cuda").view(seqs, 8)
    ws = mc.attn4_workspace(cache, heads)
    lens = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    for add, done in (([40, 3, 0, 64, 17], None), ([1] * 5, None), ([1, 30, 9, 0, 1], [0, 0, 0, 1, 0]), ([1] * 5, None)):
        T = sum(add)
        plan = d.step(add, done, T)
        assert d.fine()
        x = [torch.randn(T, n, dim, generator=g).to(torch.bfloat16).cuda() for n in (heads, kv, kv)]
        if done:
            lens[3] = 0
        lens += torch.tensor(add, dtype=torch.int32).cuda()
        hand = mc.KVBatch(lens.clone(), table, plan.cu_q.clone(), T)
        outs = []
        for c, batch in ((cache, plan.batch), (own, hand)):
            q = mc.kv4_append(c, batch, *x, workspace=ws)
            outs.append(mc.attn4_prefill(c, batch, q, workspace=ws))
            k, v = mc.kv4_read(c, batch)
            outs[-1] = (outs[-1], k, v)
        mc.check_status(ws)
        for p, q in zip(*outs):
            assert torch.equal(p, q)
        t = T // 2  # the codes of a token's first head, at its slot
        slot = int(plan.slots[t])
        before = cache.k[slot // page, 0, slot % page * 32:slot % page * 32 + 32]
        b = int((plan.cu_q <= t).sum()) - 1
        pos = int(plan.positions[t])
        assert torch.equal(before, own.k[table[b, pos // page], 0, pos % page * 32:pos % page * 32 + 32]) and before.any()
