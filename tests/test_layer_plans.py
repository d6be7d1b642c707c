"""The forms that the layers' calls take, from the plan compiled with the host
compiler (tests/layer_plans.py)."""

import random

import pytest

from layer_plans import AVAILABLE, case, compile_plans, plans

pytestmark = pytest.mark.skipif(not AVAILABLE, reason="g++ or the HIP headers not available")


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return compile_plans(tmp_path_factory.mktemp("plans"))


def draws(n, kinds=("fwd", "bwd"), dtypes=("bf16", "f32"), seed=1):
    """Random layers up to 8192 tokens and widths, half of them of whole 64s."""
    rng = random.Random(seed)

    def side(lo, hi):
        v = round(lo * (hi / lo) ** rng.random())
        return v if rng.random() < 0.5 else max(64, v // 64 * 64)

    for _ in range(n):
        yield dict(kind=rng.choice(kinds), dtype=rng.choice(dtypes), tokens=round(8192 ** rng.random()),
                   n_in=side(16, 8192), out=side(16, 8192), act=rng.randint(0, 4),
                   gated=rng.random() < 0.5, pad=rng.choice((0, 0, 1, 8)), shift=rng.choice((0, 0, 3)))


def test_every_layer_has_a_plan_whose_parts_cover_k(exe):
    all_of = list(draws(2000))
    for c, p in zip(all_of, plans(exe, [case(**c) for c in all_of])):
        assert p["status"] == 0, c
        if p["form"] == "few":
            assert c["tokens"] <= 64 and p["bytes"] == 0
            continue
        k = c["n_in"] if c["kind"] == "fwd" else c["out"] * (2 if c["gated"] else 1)
        wide = p["form"] == "planes" or c["dtype"] == "bf16"
        assert p["x_tiles_k"] == -(-k // (64 if wide else 32)) * (6 if p["form"] == "planes" else 1)
        assert 1 <= p["x_splits"] <= p["x_tiles_k"]
