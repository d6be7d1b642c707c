"""Plans that fit no rows raise OCC_F_BAD_ROWS in the exchange, and change nothing that
they do not name."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402

pytestmark = pytest.mark.gpu

T, E, K, H = 6, 4, 2, 40


def plan():
    g = torch.Generator(device="cuda").manual_seed(3)
    r = optcc.occ_route_fwd(torch.randn(T, E, generator=g, device="cuda"), K)
    X = torch.randn(T, H, generator=g, device="cuda")
    Ys = torch.randn(T * K, H, generator=g, device="cuda")
    return r, X, Ys, torch.zeros(1, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("last,rows", [(T * K + 1, T * K), (1 << 30, T * K), (-1, 0),
                                       (-(1 << 31), 0)])
def test_dispatch_with_a_last_offset_outside_its_rows(last, rows):
    r, X, _, flags = plan()
    offsets = r.offsets.clone()
    offsets[-1] = last
    Xs = torch.full((T * K, H), 5.0, device="cuda")
    optcc.occ_dispatch(X, r._replace(offsets=offsets), Xs=Xs, flags=flags)
    assert flags.item() == optcc.OCC_F_BAD_ROWS
    assert torch.equal(Xs[:rows], X[r.order[:rows].long() // K]) and (Xs[rows:] == 5.0).all()


def test_dispatch_with_an_order_too_short_for_its_offsets():
    r, X, _, flags = plan()
    Xs = optcc.occ_dispatch(X, r._replace(order=r.order[:7].contiguous()), flags=flags)
    assert flags.item() == optcc.OCC_F_BAD_ROWS
    assert torch.equal(Xs, X[r.order[:7].long() // K])


@pytest.mark.parametrize("last", [0, 5, T * K])
def test_dispatch_of_a_part_of_its_rows(last):
    r, X, _, flags = plan()
    offsets = r.offsets.clone()
    offsets[-1] = last
    Xs = torch.full((T * K, H), 5.0, device="cuda")
    optcc.occ_dispatch(X, r._replace(offsets=offsets), Xs=Xs, flags=flags)
    assert flags.item() == 0 and (Xs[last:] == 5.0).all()


@pytest.mark.parametrize("slot,bad", [(-1, False), (-2, True), (-(1 << 31), True), (T * K, True),
                                      ((1 << 31) - 1, True)])
def test_slots_outside_the_rows(slot, bad):
    """Each counts as no row; all but -1 raise the flag."""
    r, X, Ys, flags = plan()
    slots = r.slots.clone()
    slots[2, 1] = slot
    none = torch.where(slots == slot, -1, slots).to(torch.int32)
    got = optcc.occ_combine(Ys, r._replace(slots=slots), weights=r.weights, flags=flags)
    assert flags.item() == (optcc.OCC_F_BAD_ROWS if bad else 0)
    assert torch.equal(got, optcc.occ_combine(Ys, r._replace(slots=none), weights=r.weights))
    flags.zero_()
    dYs = torch.full((T * K, H), 5.0, device="cuda")
    _, dw = optcc.occ_combine_bwd(X, Ys, r._replace(slots=slots), weights=r.weights, dYs=dYs,
                                  flags=flags)
    assert flags.item() == (optcc.OCC_F_BAD_ROWS if bad else 0)
    assert dw[2, 1] == 0 and (dYs[r.slots[2, 1].long()] == 5.0).all()
