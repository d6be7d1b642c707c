"""The forms that the experts' layers take, from the plan compiled with the host
compiler (tests/experts_plans.py)."""

import random

import pytest

from experts_forms import FORMS, split
from experts_plans import case, compile_plans
from layer_plans import AVAILABLE, plans

pytestmark = pytest.mark.skipif(not AVAILABLE, reason="g++ or the HIP headers not available")


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return compile_plans(tmp_path_factory.mktemp("plans"))


def draws(n, seed, odd=False):
    rng = random.Random(seed)

    def side():
        v = round(16 * 512 ** rng.random())
        return v if rng.random() < 0.5 else max(64, v // 64 * 64)

    for _ in range(n):
        c = dict(kind=rng.choice(("fwd", "bwd")), dtype=rng.choice(("bf16", "f32")),
                 gated=rng.random() < 0.5, experts=round(128 ** rng.random()),
                 rows=round(16384 ** rng.random()), n_in=side(), out=side())
        c["act"] = 4 if c["gated"] else 2
        if odd:
            c.update(pad=rng.choice((0, 1, 8)), shift=rng.choice((0, 3)), act=rng.randint(0, 4),
                     dx=rng.random() < 0.8, db=rng.random() < 0.5)
        yield c


def key(c, p):
    return c["kind"], c["dtype"], c["gated"], p["form"], p["tile"], p["copied"]


def test_the_gpu_tests_reach_the_forms_they_name(exe):
    """tests/test_gpu_experts_forms.py runs these layers."""
    cases = [case(kind, dtype, *size, act=4 if gated else 2, gated=gated, db=db)
             for kind, dtype, gated, _, _, _, db, size in FORMS]
    for (kind, dtype, gated, form, tile, copied, _, size), p in zip(FORMS, plans(exe, cases)):
        assert (p["status"], p["form"], p["tile"], p["copied"]) == (0, form, tile, copied), \
            (kind, dtype, gated, size, p)


def test_no_form_is_left_out(exe):
    """What 40000 random layers take, the listed ones take too."""
    listed = {(kind, dtype, gated, form, tile, copied)
              for kind, dtype, gated, form, tile, copied, _, _ in FORMS}
    all_of, taken = list(draws(40000, 1)), {}
    for c, p in zip(all_of, plans(exe, [case(**c) for c in all_of])):
        assert p["status"] == 0, c
        taken[key(c, p)] = taken.get(key(c, p), 0) + 1
    assert not {k: n for k, n in taken.items() if k not in listed and n > 2}


def test_offsets_within_a_wave_stay_in_31_bits(exe):
    """A wave's rows of the dZ that a gated layer makes are addressed from the
    first of them by a 32-bit offset below 2^31."""
    rng = random.Random(2)
    all_of = [dict(kind="bwd", dtype=rng.choice(("f32", "bf16")), experts=rng.choice((1, 2, 7)),
                   rows=rng.choice((1, 128, 300, 1024, 4096)), n_in=rng.choice((64, 300, 2048)),
                   act=4, gated=True, out=rng.randint(1 << 21, 16 << 20), dw=rng.random() < 0.5)
              for _ in range(600)]
    taken = 0
    for c, p in zip(all_of, plans(exe, [case(**c) for c in all_of])):
        if p["status"] or p["form"] == "direct" or not p["made"]:
            continue
        taken += 1
        size = 2 if p["form"] == "planes" or c["dtype"] == "bf16" else 4
        assert p["tile"] // 8 * p["ldd"] * size <= 1 << 31, (c, p)
    assert taken > 50


def test_launches_stay_within_the_largest_grid(exe):
    """Fewer than 2^32 threads in a launch, or the plan refuses."""
    rng, top = random.Random(3), (1 << 30) - 1
    all_of = []
    for _ in range(600):
        width = rng.choice((1, 7, 64, 300, 1024, 1 << 20))
        all_of.append(dict(kind=rng.choice(("fwd", "bwd")), dtype=rng.choice(("bf16", "f32")),
                           experts=rng.choice((1, 8, 1024)), n_in=width, act=rng.randint(1, 4),
                           rows=rng.choice((3, top, 1 << 29, rng.randint(1 << 20, top))),
                           out=rng.choice((1, 64, width, 1 << 24)), gated=rng.random() < 0.3,
                           shift=rng.choice((0, 1)), dx=rng.random() < 0.8))
    taken = 0
    for c, p in zip(all_of, plans(exe, [case(**c) for c in all_of])):
        if p["status"]:
            continue
        taken += 1
        assert p["blocks"] * 512 < 1 << 32, (c, p)
    assert taken >= 100


def test_workspaces_do_not_depend_on_the_lengths(exe):
    """The same sizes need the same bytes, whatever the offsets will hold, and
    bytes that hold what the call copies; direct forms and few rows need none."""
    all_of = list(draws(4000, 7, odd=True))
    for c, p in zip(all_of, plans(exe, [case(**c) for c in all_of])):
        if p["status"]:
            continue
        if c["kind"] == "fwd" and p["form"] in ("few", "direct"):
            assert p["bytes"] == 0
        if p["form"] == "planes":
            assert p["bytes"] > 6 * c["n_in"] * (c["rows"] if c["kind"] == "fwd" or not c["dx"] else 1)


def test_the_split_has_its_sum():
    for rows in (3, 15, 1000, 16384):
        for experts in (1, 3, 114):
            s = split(rows, experts)
            assert len(s) == experts and sum(s) == rows and min(s) >= 0
