"""The 4-bit form by its two test implementations, and what holds for every group."""
import math
import random

import pytest

torch = pytest.importorskip("torch")

import attn_ref as ref  # noqa: E402
import kv4_ref  # noqa: E402


def _groups(dtype, seed):
    rng, g = random.Random(seed), torch.Generator().manual_seed(seed)
    t = ref.DT[dtype]
    top = torch.finfo(t).max
    yield torch.zeros(64, dtype=t)
    yield torch.full((64,), top, dtype=t)
    yield torch.cat([torch.full((32,), top), torch.full((32,), -top)]).to(t)
    yield torch.cat([torch.full((32,), top * 0.992), torch.full((32,), -top * 0.12)]).to(t)
    yield torch.full((64,), 2.0 ** -24, dtype=t)
    yield torch.arange(64).to(t) - 20
    yield (torch.arange(64) % 16).to(t) * 0.5  # every element on the grid
    for _ in range(60):
        x = torch.randn(64, generator=g) * 2.0 ** rng.uniform(-30 if dtype == "bf16" else -18, 30 if dtype == "bf16" else 12)
        yield (x + rng.choice([0.0, 0.0, 3.0, -40.0]) * x.abs().mean()).clamp(-top, top).to(t)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_groups_are_near_and_exact_in_the_type(dtype):
    for x in _groups(dtype, 3):
        codes, s, z = kv4_ref.grid(x.double().tolist(), dtype)
        assert all(0 <= c <= 15 for c in codes) and 0 <= z <= 15
        assert math.frexp(s)[0] * 16 == int(math.frexp(s)[0] * 16)  # four significant bits
        y = torch.tensor([kv4_ref.value(s, z, c) for c in codes], dtype=torch.float64)
        assert torch.equal(y.to(ref.DT[dtype]).double(), y)
        # half a step, and half of one more where the zero point's rounding cut an end (or the type's largest number did)
        assert ((y - x.double()).abs() <= s * (1 + 1e-12)).all()
        c, s2, z2 = kv4_ref.grids(x.double()[None], dtype)
        assert s2.item() == s and z2.item() == z and c[0].tolist() == codes


def test_groups_that_are_not_finite():
    for bad in (math.inf, -math.inf, math.nan):
        x = [0.5] * 63 + [bad]
        assert math.isnan(kv4_ref.grid(x, "bf16")[1])
    assert kv4_ref.word(math.nan, 0) & 0x7f80 == 0x7f80
