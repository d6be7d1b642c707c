"""The forms that the layers' calls take, from the plan compiled with the host
compiler (tests/layer_plans.py)."""

import random

import pytest

from layer_plans import AVAILABLE, case, compile_plans, plans
from stage_forms import ALONE, FORMS, SINGLE

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


def test_offsets_within_a_wave_stay_in_31_bits(exe):
    """A wave's rows of an operand (an eighth of the tile's) are addressed from
    the first of them by a 32-bit offset below 2^31: also those of the dZ that a
    gated fp32 layer makes, up to 2^27 bytes wide, 32 of which would pass it."""
    all_of = list(draws(6000, kinds=("bwd",), dtypes=("f32",)))
    rng = random.Random(2)
    all_of += [dict(kind="bwd", dtype="f32", tokens=rng.choice((128, 256, 300, 513, 1024, 2048, 4096)),
                    n_in=rng.choice((64, 256, 300, 1024, 2048)), act=4, gated=True,
                    out=rng.randint(8 << 20, 16 << 20), dw=rng.random() < 0.5) for _ in range(300)]
    # weight gradients of few tokens, which used to take that form
    all_of += [dict(kind="bwd", dtype="f32", tokens=t, n_in=k, out=n, act=4, gated=True, dx=False)
               for t, k, n in ((4, 7322, 8024), (17, 139, 8640027), (2, 6910, 2434027))]
    used = set()
    for c, p in zip(all_of, plans(exe, [case(**c) for c in all_of])):
        if p["status"]:
            continue
        size = 2 if p["form"] == "planes" else 4
        if p["form"] != "direct" and p["made"]:
            assert p["tile"] // 8 * p["ldd"] * size <= 1 << 31, (c, p)
        used.add((p["form"], p["tile"]))
    assert {("tiled", 128), ("tiled", 64), ("planes", 256), ("direct", 64)} <= used


def test_launches_stay_within_the_largest_grid(exe):
    """A launch holds fewer than 2^32 threads in a dimension: layers of any
    number of tokens that the interface admits get tiles large enough for that
    (512 threads a block, the bias gradient's blocks among them), or are refused
    by the plan before anything is enqueued."""
    rng = random.Random(3)
    top = (1 << 30) - 1
    all_of = []
    for _ in range(600):
        width = rng.choice((1, 7, 16, 64, 100, 128, 300, 1024))
        c = dict(kind=rng.choice(("fwd", "bwd")), dtype=rng.choice(("bf16", "f32")),
                 tokens=rng.choice((top, 1 << 29, rng.randint(1 << 27, top))), n_in=width,
                 out=rng.choice((1, 16, 64, width)), act=rng.randint(1, 4), gated=rng.random() < 0.3,
                 shift=rng.choice((0, 1)), dx=rng.random() < 0.8)
        all_of.append(c)
    # few tokens and huge weights
    all_of += [dict(kind="bwd", dtype="bf16", tokens=3, n_in=1 << 24, out=1 << w, act=0, dx=False)
               for w in (9, 12, 13, 14, 16, 20)]
    taken = 0
    for c, p in zip(all_of, plans(exe, [case(**c) for c in all_of])):
        if p["status"]:     # the call's matrices alone pass the memory of a GPU
            size = 2 if c["dtype"] == "bf16" else 4
            rows = c["n_in"] * (1 if c["kind"] == "fwd" else 1 + c.get("dx", True)) + c["out"]
            assert size * (c["tokens"] * rows + c["out"] * c["n_in"]) > 288e9, c
            continue
        taken += 1
        bias = -(-c["out"] * (2 if c.get("gated") else 1) // 16)
        assert (p["x_blocks"] + p["w_blocks"] + bias) * 512 < 1 << 32, (c, p)
    assert taken >= 300


def test_the_gpu_tests_reach_the_forms_they_name(exe):
    """tests/test_gpu_layer_forms.py runs these layers."""
    cases = [case(kind, dtype, *size, act=4 if gated else 2, gated=gated)
             for kind, dtype, gated, _, _, _, size in FORMS]
    for (kind, dtype, gated, form, tile, parts, size), p in zip(FORMS, plans(exe, cases)):
        split = p["x_splits"] > 1 or (kind == "bwd" and p["w_splits"] > 1)
        assert (p["status"], p["form"], p["tile"]) == (0, form, tile), (kind, dtype, size, p)
        assert form == "few" or split == parts, (kind, dtype, size, p)
    for dtype, act, gated, form, tile, size, output in ALONE:
        p, = plans(exe, [case("bwd", dtype, *size, act=act, gated=gated, dx=output == "dX",
                              dw=output == "dW", db=False)])
        assert (p["status"], p["form"], p["tile"]) == (0, form, tile), (size, p)


def test_no_form_is_left_out(exe):
    """What 20000 random layers take, the listed ones take too."""
    listed = {(kind, dtype, gated, form, tile) for kind, dtype, gated, form, tile, _, _ in FORMS}
    all_of = [c for c in draws(20000, seed=4) if c["pad"] == 0 and c["shift"] == 0]
    taken = {}
    for c, p in zip(all_of, plans(exe, [case(**c) for c in all_of])):
        key = (c["kind"], c["dtype"], c["gated"], p["form"], p["tile"])
        taken[key] = taken.get(key, 0) + 1
    assert not {k: n for k, n in taken.items() if k not in listed and n > 2}


def test_layers_of_the_plane_tests_take_planes(exe):
    sizes = [(2048, 1030, 3000), (1500, 2304, 2200), (3001, 2047, 1533), (4096, 256, 4096),
             (4096, 520, 4096)]
    cases = [case("fwd", "f32", *s, act=0, gated=g) for s in sizes for g in (False, True)]
    cases += [case("bwd", "f32", *s, act=0) for s in [(520, 4096, 4096), (4096, 4096, 520)]]
    assert {p["form"] for p in plans(exe, cases)} == {"planes"}
    cases = [case("fwd", "f32", *s, act=0) for s in [(200, 520, 130), (1003, 1023, 2047)]]
    cases += [case("bwd", "f32", *s, act=0) for s in [(517, 1000, 1500), (300, 200, 100)]]
    assert "planes" not in {p["form"] for p in plans(exe, cases)}


def test_the_requested_outputs_enter_the_plan(exe):
    for dtype, act, size, single, what in SINGLE:
        both, one = plans(exe, [case("bwd", dtype, *size, act=act, db=False),
                                case("bwd", dtype, *size, act=act, db=False, dx=single == "dX",
                                     dw=single == "dW")])
        assert both[what] != one[what], (dtype, size)
