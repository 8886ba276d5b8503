"""The example decoder: tokens fed one by one through the cache give the hidden states that one
prefill of the whole text gives, and drafted tokens checked a few at a time do too."""
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


def test_steps_through_the_cache_match_one_prefill(decoder):
    """Hidden states are sums of bf16 values rounded at the same places, of attention outputs and
    expert outputs (each within 2^-8 and 5e-3 of its definition) that the two ways sum in other
    orders; a routing decision within rounding of a tie may differ for a token, so the bound is
    on the whole."""
    lens, steps = [21, 1, 40], 5
    whole = [n + steps for n in lens]
    ids = [torch.randint(decoder.VOCAB, (n,), generator=torch.Generator().manual_seed(7 + n)).cuda() for n in whole]
    one = decoder.Decoder(2, 3, 64)
    want = one.forward(torch.cat(ids), whole).split(whole)
    one.check()

    d = decoder.Decoder(2, 3, 64)
    got = [[x] for x in d.forward(torch.cat([t[:n] for t, n in zip(ids, lens)]), lens).split(lens)]
    for i in range(3):  # one token each
        for x, h in zip(got, d.forward(torch.stack([t[n + i] for t, n in zip(ids, lens)])).split(1)):
            x.append(h)
    # the last two at once, as a verification of drafted tokens does
    for x, h in zip(got, d.forward(torch.cat([t[n + 3:] for t, n in zip(ids, lens)]), [steps - 3] * 3).split(steps - 3)):
        x.append(h)
    d.check()
    for x, w in zip(got, want):
        assert _rel(torch.cat(x), w) <= 3e-2


def test_users_do_not_see_each_other(decoder):
    """A user's states do not depend on the others' tokens, nor on where its pages lie."""
    a, b = (torch.randint(decoder.VOCAB, (19,), generator=torch.Generator().manual_seed(s)).cuda() for s in (1, 2))
    both = decoder.Decoder(2, 2, 32, max_tokens=64).forward(torch.cat([a, b]), [19, 19])
    alone = decoder.Decoder(2, 1, 32, max_tokens=64).forward(a, [19])
    assert _rel(both[:19], alone) <= 3e-2
