"""The 64-bit forms of the expert layer and the token dropout, pinned to library routines, closed forms, published
vectors and differences."""
import numpy as np
import pytest
import torch

from oracle import experts as orc


# Known-answer vectors of Philox4x32-10 that its authors publish with their generator.
@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_philox_known_answers(counter, key, want):
    assert tuple(int(v) for v in orc.philox4x32(np.array(counter), key)) == want


def test_dropout_mask():
    assert orc.dropout_mask(7, 13, 0.0, 1, 2).all()
    m = orc.dropout_mask(400, 1001, 0.3, 5, 6)
    n = m.size
    assert abs(m.mean() - 0.7) < 6 * np.sqrt(0.21 / n)
    assert (orc.dropout_mask(5, 1001, 0.3, 5, 6, row0=10) == m[10:15]).all()
    for other in (orc.dropout_mask(400, 1001, 0.3, 6, 6), orc.dropout_mask(400, 1001, 0.3, 5, 7),
                  orc.dropout_mask(400, 1001, 0.3, 5, 6 + 2 ** 32)):
        assert abs((other == m).mean() - 0.58) < 6 * np.sqrt(0.25 / n)
    x = np.random.default_rng(0).standard_normal((6, 9))
    y = orc.dropout(x, 0.5, 3, 4)
    keep = orc.dropout_mask(6, 9, 0.5, 3, 4)
    assert (y == np.where(keep, 2 * x, 0)).all()
    # its own gradient: the map is linear and diagonal
    assert np.allclose(orc.dropout(x, 0.5, 3, 4, res=x) - x, y, rtol=0, atol=1e-15)


@pytest.mark.parametrize("normalise", [False, True])
def test_route_against_library(normalise):
    g = np.random.default_rng(1)
    z, bias = g.standard_normal((50, 23)).astype(np.float32), g.standard_normal(23).astype(np.float32)
    chosen, w, slots, offsets = orc.route(z, 5, normalise, bias)
    top = torch.topk(torch.from_numpy(z + bias), 5)[1].numpy()
    assert (chosen == top).all()
    t = torch.from_numpy(z).double().requires_grad_(True)
    picked = torch.gather(t, 1, torch.from_numpy(top))
    ref = torch.softmax(picked, 1) if normalise else torch.gather(torch.softmax(t, 1), 1, torch.from_numpy(top))
    assert np.allclose(w, ref.detach().numpy(), rtol=1e-13)
    dw = g.standard_normal(w.shape)
    dz, _ = orc.route_bwd(z, chosen, w, dw, normalise)
    (ref * torch.from_numpy(dw)).sum().backward()
    assert np.allclose(dz, t.grad.numpy(), rtol=1e-11, atol=1e-14)
    # the places are a permutation, in order within an expert
    assert sorted(slots.reshape(-1)) == list(range(250)) and offsets[-1] == 250
    for e in range(23):
        mine = slots[chosen == e]
        assert (np.diff(mine) > 0).all() and ((mine >= offsets[e]) & (mine < offsets[e + 1])).all()


def test_route_ties_masks_and_rows_without_a_distribution():
    inf, nan = np.inf, np.nan
    z = np.array([[1, 1, 1, 1], [0., -0., -inf, -inf], [-inf] * 4, [nan, 0, 0, 0], [inf, 0, 0, 0], [1, 2, 3, 4], [nan] * 4])
    chosen, w, slots, offsets = orc.route(z, 3, False, row_weight=np.array([1, 1, 1, 1, 1, 1, 0.]))
    assert chosen.tolist() == [[0, 1, 2], [0, 1, -1], [-1] * 3, [-1] * 3, [-1] * 3, [3, 2, 1], [-1] * 3]
    assert np.allclose(w[0], 0.25) and np.allclose(w[1], [0.5, 0.5, 0]) and (w[2] == 0).all() and np.isnan(w[3:5]).all()
    assert (w[6] == 0).all() and offsets.tolist() == [0, 2, 5, 7, 8]
    dz, _ = orc.route_bwd(z, chosen, w, np.ones(w.shape), False)
    assert np.isnan(dz[3:5]).all() and (dz[2] == 0).all() and (dz[6] == 0).all()
    assert np.allclose(dz[5].sum(), 0)


def test_products_and_exchange_are_adjoint():
    g = np.random.default_rng(2)
    offsets = np.array([0, 5, 5, 17])
    x, w, dy = g.standard_normal((20, 8)), g.standard_normal((3, 16, 8)), g.standard_normal((20, 16))
    y, live = orc.grouped_fwd(x, w, offsets)
    dx, _ = orc.grouped_dgrad(dy, w, offsets)
    dw = orc.grouped_wgrad(x, dy, offsets)
    assert live.sum() == 17 and (y[17:] == 0).all() and (dw[1] == 0).all()
    inner = (y * dy).sum()
    assert np.isclose(inner, (x * dx).sum()) and np.isclose(inner, (w * dw).sum())
    assert np.allclose(y[6], w[2] @ x[6])
    assert [tuple(v) for v in orc._groups([-3, 4, 2, 99], 20)] == [(0, 0, 4), (1, 4, 4), (2, 4, 20)]
    r, _ = orc.grouped_fwd(x, w, offsets, relu=True)
    assert (r == np.maximum(y, 0)).all()
    masked, _ = orc.grouped_dgrad(dy, w, offsets, mask=x)
    assert (masked == np.where(x > 0, dx, 0)).all()

    slots = np.array([[3, 0], [-1, 1], [2, 7]])
    t, wt = g.standard_normal((3, 4)), g.standard_normal((3, 2))
    yg, dout = g.standard_normal((4, 4)), g.standard_normal((3, 4))
    xg = orc.scatter(t, slots, np.zeros((4, 4)))
    assert (xg == t[[0, 1, 2, 0]]).all()  # slot 7 is outside
    assert np.isclose((xg * yg).sum(), (t * orc.combine(yg, slots)[0]).sum())
    out, _ = orc.combine(yg, slots, wt, res=t)
    dyg, dwt, _ = orc.combine_bwd(dout, yg, slots, wt, np.zeros((4, 4)))
    assert np.isclose(((out - t) * dout).sum(), (dyg * yg).sum()) and np.isclose((dyg * yg).sum(), (dwt * wt).sum())
