"""The example decoder over the cache in 4 bits: the append, the attentions, the pages' plan and the norms between the
blocks together, as they are used."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def decoder():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2410_06270_gb300 import build
    build.build()
    import decoder as m
    return m


def _rel(a, b):
    return float((a.float() - b.float()).norm() / b.float().norm())


def _text(n, seed, decoder):
    return torch.randint(decoder.VOCAB, (n,), generator=torch.Generator().manual_seed(seed)).cuda()


def test_steps_through_the_cache_match_one_prefill(decoder):
    """A token's keys and values are the same numbers whichever call stores them, but for elements whose hidden
    state differs in its last bits, next to the border of two codes; a routing decision near a tie may differ too, so
    the bound is on the whole."""
    lens, steps = [21, 1, 40], 5
    whole = [n + steps for n in lens]
    ids = [_text(n, 7 + n, decoder) for n in whole]
    one = decoder.Decoder(2, 3, 64, bits4=True)
    want = one.forward(torch.cat(ids), whole).split(whole)
    one.check()
    d = decoder.Decoder(2, 3, 64, bits4=True)
    got = [[x] for x in d.forward(torch.cat([t[:n] for t, n in zip(ids, lens)]), lens).split(lens)]
    for i in range(3):  # one token each
        for x, h in zip(got, d.forward(torch.stack([t[n + i] for t, n in zip(ids, lens)])).split(1)):
            x.append(h)
    # the last two at once, as a verification of drafted tokens does
    for x, h in zip(got, d.forward(torch.cat([t[n + 3:] for t, n in zip(ids, lens)]), [steps - 3] * 3).split(steps - 3)):
        x.append(h)
    d.check()
    for x, w in zip(got, want):
        assert _rel(torch.cat(x), w) <= 5e-2


def test_first_tokens_are_those_of_the_16_bit_cache_but_for_the_codes(decoder):
    """One layer: the hidden state differs by what 4 bits cost keys and values (a step of a fifteenth of a group's
    span, off by half of it at most: a tenth of an element in the mean), through an attention that averages it."""
    ids, n = _text(60, 3, decoder), [40, 20]
    a, b = (decoder.Decoder(1, 2, 64, bits4=x) for x in (False, True))
    x, y = a.forward(ids, n), b.forward(ids, n)
    a.check(), b.check()
    assert 1e-4 < _rel(y, x) <= 0.1


@pytest.mark.parametrize("bits4", [False, True])
def test_a_finished_users_pages_serve_another(decoder, bits4):
    """Texts follow each other in a user's place, over pages that others wrote before; each is as if it were alone."""
    d = decoder.Decoder(2, 2, 48, max_tokens=64, bits4=bits4)
    a = _text(30, 1, decoder)
    d.forward(torch.cat([a, a[:5]]), [30, 5])
    for i in range(4):
        text, over = _text(12 + 9 * i, 20 + i, decoder), [i % 2 == 0, i % 2 == 1]
        new = [len(text) if o else 1 for o in over]
        h = d.forward(torch.cat([text, a[:1]] if over[0] else [a[:1], text]), new, over)
        d.check()
        got = h[:len(text)] if over[0] else h[1:]
        alone = decoder.Decoder(2, 1, 48, max_tokens=64, bits4=bits4)
        assert _rel(got, alone.forward(text, [len(text)])) <= 5e-2


def test_without_pages_a_step_is_refused_and_reported(decoder):
    import paper_2410_06270_gb300 as mc
    d = decoder.Decoder(1, 2, 32, max_tokens=64, bits4=True)
    d.forward(_text(60, 4, decoder), [32, 28])
    d.check()
    d.forward(_text(2, 5, decoder))  # the first is at its table's end
    with pytest.raises(mc.MCError) as e:
        d.check()
    assert e.value.code == mc.ERR_RANGE and d.lens.tolist() == [32, 29]


def _bytes(d, rows):
    """What the caches hold of a user: its pages of every layer, keys and values."""
    return [side[rows].clone() for w in d.layers for side in (w.cache.k, w.cache.v)]


@pytest.mark.parametrize("bits4", [False, True])
@pytest.mark.parametrize("new", [None, [1, 1, 1], [3, 2, 4], [2, 5, 1]])
def test_a_refused_user_keeps_its_cache_and_goes_on(decoder, bits4, new):
    """The first is out of pages for a step: nothing of its cache changes, the others' rows are those of their own
    tokens, and when there are pages again it goes on as one that was never refused."""
    import paper_2410_06270_gb300 as mc
    n = new or [1, 1, 1]
    d, e = (decoder.Decoder(2, 3, 64, max_tokens=64, bits4=bits4) for _ in range(2))
    texts = [_text(m, 60 + m, decoder) for m in (32, 18, 5)]
    more = [_text(m, 80 + i, decoder) for i, m in enumerate(n)]
    for x in (d, e):
        x.forward(torch.cat(texts), [32, 18, 5])
        x.check()
    own = d.table[0, :2].long()
    kept, counts = _bytes(d, own), d.pool.state.clone()
    d.pool.state[1] = d.pool.state[0]  # no page is free
    got = d.forward(torch.cat(more), new).split(n)
    with pytest.raises(mc.MCError) as err:
        d.check()
    assert err.value.code == mc.ERR_RANGE and d.lens.tolist() == [32] + [18 + n[1], 5 + n[2]]
    assert all(torch.equal(x, y) for x, y in zip(_bytes(d, own), kept))
    want = e.forward(torch.cat(more[1:]), [0] + n[1:]).split(n[1:])
    for x, y in zip(got[1:], want):
        assert _rel(x, y) <= 5e-2
    assert not got[0].any()
    d.pool.state.copy_(counts)
    last = [_text(1, 90 + i, decoder) for i in range(3)]
    x = d.forward(torch.cat([more[0], last[1], last[2]]), [n[0], 1, 1])
    y = e.forward(torch.cat([more[0], last[1], last[2]]), [n[0], 1, 1])
    d.check(), e.check()
    assert _rel(x, y) <= 5e-2
