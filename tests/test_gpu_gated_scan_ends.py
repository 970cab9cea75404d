"""The gated scan where states, inputs or gradients are infinite and where gates are large, against the recurrence step by
step in 64 bits.

Every finite gate a is above 0, so an infinite state stays infinite until something else joins it; products of gates
over many steps round to 0 in fp32 (gates of 0.05 over 64 steps: 2^-276).  Finite values have the tolerance of
test_gpu_gated_scan.py; a state's infinity has to be that infinity, and NaN NaN."""
import numpy as np
import pytest
import torch

from gpu_common import check_status, load_dbl
from oracle import tokens as T
from test_gpu_gated_scan import EPS32, Case, K, carried, run
from token_cases import Rows, assert_within, precision, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def D():
    return load_dbl()


def tolerance(tol, want):
    """What is not finite has to be met exactly."""
    return np.where(np.isfinite(want), tol, 0.0)


# short sequences, one part, several parts, several blocks and clusters; aligned rows and others; lengths
CASES = [dict(n=2, t=9, c=64), dict(n=3, t=65, c=33), dict(n=2, t=300, c=64), dict(n=2, t=700, c=63, packed=True),
         dict(n=1, t=9000, c=64), dict(n=1, t=5000, c=15), dict(n=3, t=2100, c=35, lengths=[64, 2100, 128]),
         dict(n=2, t=1500, c=600)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
@pytest.mark.parametrize("where", ["h0", "x", "both signs"])
def test_an_infinite_state_stays_infinite(D, kind, case, where):
    cs = Case(kind, **case, gate_mean=-3.0)
    n, t, c = cs.n, cs.t, cs.c
    x = torch.as_strided(cs.both.buf, (n * t, c), (2 * c, 1), cs.both.offset) if cs.packed else cs.rx.view()
    first = min(t - 1, t // 3)
    if where in ("h0", "both signs"):
        cs.h0[:, 0], cs.h0[:, 3] = np.inf, -np.inf
        cs.th0.copy_(torch.from_numpy(cs.h0))
    if where in ("x", "both signs"):  # of "both signs" +infinity meets -infinity in channel 3
        for b in range(n):
            x[b * t + first, 3] = np.inf
            x[b * t + t // 2, 5] = -np.inf
    clean = (cs.both.values()[:, :c] if cs.packed else cs.rx.values()).reshape(n, t, c)
    x64, z = np.where(cs.live, clean, 0.0), cs.clean[1]
    with np.errstate(invalid="ignore"):
        wh, wl, wst, prev = T.gated_scan_fwd(x64, z, cs.h0, cs.lengths)
        a, na = T.gates(z)
        size = T.gated_scan_fwd(np.abs(x64), z, np.abs(cs.h0), cs.lengths)[0]
        E, Elast = carried(size, a, cs.live, np.zeros((n, c)))
        E = np.where(cs.live, E, 0.0)
    assert np.isinf(wh).any()
    h, last, st = run(D, cs)
    assert_within(h.values().reshape(n, t, c), wh, tolerance(E + rounding(kind, np.abs(wh) + E) * cs.live, wh), "h")
    assert_within(last.values(), wl, tolerance(Elast, wl), "h_last")
    Eprev = np.concatenate([np.zeros((n, 1, c)), carried(size, a, cs.live, np.zeros((n, c)))[0][:, :-1]], 1)
    assert_within(st.values().reshape(n, -1, c), wst, tolerance(Eprev[:, ::D.DBL_SCAN_CHUNK], wst), "states")


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_an_infinite_gradient_is_not_lost(D, kind, case):
    """Of h in one channel, of h_last in another, of both with opposite signs in a third; and gradients of finite size
    past infinite states (dgate is not finite there, dx is).  What is not finite in 64 bits is infinite or NaN, everything
    else is as if nothing were."""
    cs = Case(kind, **case, gate_mean=-3.0)
    n, t, c = cs.n, cs.t, cs.c
    cs.h0[:, 7] = np.inf
    cs.th0.copy_(torch.from_numpy(cs.h0))
    _, _, st = run(D, cs)
    lens = T._lengths(n, t, cs.lengths)
    for b in range(n):
        cs.dh.view()[b * t + 2 * lens[b] // 3, 2] = np.inf
        cs.dh.view()[b * t + lens[b] // 2, 6] = -np.inf
    cs.dlast[:, 4], cs.dlast[:, 6] = -np.inf, np.inf
    x, z = cs.clean
    with np.errstate(invalid="ignore"):
        _, _, _, prev = T.gated_scan_fwd(x, z, cs.h0, cs.lengths)
        a, na = T.gates(z)
        size = T.gated_scan_fwd(np.abs(x), z, np.abs(cs.h0), cs.lengths)[0]
        Eprev = np.concatenate([np.zeros((n, 1, c)), carried(size, a, cs.live, np.zeros((n, c)))[0][:, :-1]], 1)
        DH = np.where(cs.live, cs.dh.values().reshape(n, t, c), 0.0)
        wx, wz, w0, _ = T.gated_scan_bwd(DH, x, z, prev, cs.dlast, cs.lengths)
        G = T.gated_scan_bwd(np.abs(DH), x, z, prev, np.abs(cs.dlast), cs.lengths)[3]
        anext = np.concatenate([a[:, 1:], np.ones((n, 1, c))], 1)
        EG = carried(G[:, ::-1], anext[:, ::-1], cs.live[:, ::-1], np.zeros((n, c)))[0][:, ::-1]
        tolx = (na * EG + K * EPS32 * na * G) * cs.live
        pm = np.concatenate([np.abs(cs.h0)[:, None], size[:, :-1]], 1)
        tolz = a * na * ((EG + K * EPS32 * G) * (pm + np.abs(x)) + G * Eprev) * cs.live
        tolx, tolz = tolx + rounding(kind, np.abs(wx) + tolx) * cs.live, tolz + rounding(kind, np.abs(wz) + tolz) * cs.live
        first = np.where(cs.live[:, 0], a[:, 0] * (EG[:, 0] + K * EPS32 * G[:, 0]), 0.0)
    assert np.isinf(wx).any() and np.isnan(wx).any() and np.isinf(wz[:, :, 7]).any() and np.isfinite(wx[:, :, 7]).all()
    lib, dtype = precision(D, kind)
    ld = 2 * c if cs.packed else cs.ld
    dx, dz, dh0 = Rows(kind, n * t, c, ld), Rows(kind, n * t, c, ld), Rows("f32", n, c)
    with lib:
        D.dbl_gated_scan_bwd(cs.shape(D, dtype), cs.dh.ptr(), torch.from_numpy(cs.dlast).cuda(), cs.px, cs.pz, st.ptr(),
                             cs.len, dx.ptr(), dz.ptr(), dh0.ptr())
        check_status(D)
    for got, want, tol, what in ((dx, wx, tolx, "dx"), (dz, wz, tolz, "dgate"), (dh0, w0, first, "dh0")):
        got = got.values().reshape(want.shape)
        finite = np.isfinite(want)
        assert not np.isfinite(got[~finite]).any(), what
        assert_within(np.where(finite, got, 0.0), np.where(finite, want, 0.0), np.where(finite, tol, 0.0), what)


@pytest.mark.parametrize("t", [1, 70])
def test_gates_of_any_size_keep_their_digits(D, t):
    """One step that counts, from a zero state (h = (1 - a)*x) and from an input of zero (h = a*h0), in fp32: the exponential
    of the gate is off by (1.5*|gate| + 4)*2^-24 of itself, quotient, products and the result's rounding by at most 12 more."""
    c = 173
    z = np.linspace(-86.0, 86.0, c).astype(np.float32)
    a, na = T.gates(z)
    tol = (1.5 * np.abs(z.astype(np.float64)) + 16) * EPS32
    gate, zero = np.full((t, c), np.inf, np.float32), np.zeros((t, c), np.float32)
    gate[0] = z  # open from there on
    for value, x, h0 in ((na, zero + np.float32(1.5), None), (a, zero, np.full(c, 1.5, np.float32))):
        rx, rz, h, last = Rows("f32", t, c, values=x), Rows("f32", t, c, values=gate), Rows("f32", t, c), Rows("f32", 1, c)
        start = None if h0 is None else torch.from_numpy(h0).cuda()
        D.dbl_gated_scan_fwd(D.scan_shape(1, t, c, D.DBL_F32), rx.ptr(), rz.ptr(), start, None, h.ptr(), last.ptr(), None)
        check_status(D)
        want = np.broadcast_to(1.5 * value, (t, c))
        assert_within(h.values(), want, tol * want, "h")
        assert_within(last.values()[0], want[0], tol * want[0], "h_last")


@pytest.mark.parametrize("case", [dict(n=2, t=12, c=40), dict(n=2, t=300, c=64), dict(n=1, t=900, c=33)],
                         ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_large_gates_forward_and_backward(D, case):
    """Gates of -80 to 80 in fp32.  The bound of test_gpu_gated_scan.py with the exponential's error for |gate| = 80 in the
    place of that for 14: K = 40 + 1.5*(80 - 14) + 1."""
    big = 40 + 1.5 * 66 + 1
    g = np.random.default_rng(1)
    cs = Case("f32", **case)
    n, t, c = cs.n, cs.t, cs.c
    cs.rz.view().copy_(torch.from_numpy(g.uniform(-80, 80, (n * t, c))))
    z, x = cs.rz.values().reshape(n, t, c), cs.x
    wh, wl, _, prev = T.gated_scan_fwd(x, z, cs.h0)
    a, na = T.gates(z)
    size = T.gated_scan_fwd(np.abs(x), z, np.abs(cs.h0))[0]
    scaled = lambda s, gates, live: carried(s * (big / K), gates, live, np.zeros((n, c)))
    E, Elast = scaled(size, a, cs.live)
    h, last, st = run(D, cs)
    assert_within(h.values().reshape(n, t, c), wh, E + rounding("f32", np.abs(wh) + E), "h")
    assert_within(last.values(), wl, Elast, "h_last")
    DH = cs.dh.values().reshape(n, t, c)
    wx, wz, w0, _ = T.gated_scan_bwd(DH, x, z, prev, cs.dlast)
    G = T.gated_scan_bwd(np.abs(DH), x, z, prev, np.abs(cs.dlast))[3]
    anext = np.concatenate([a[:, 1:], np.ones((n, 1, c))], 1)
    EG = scaled(G[:, ::-1], anext[:, ::-1], cs.live[:, ::-1])[0][:, ::-1]
    Eprev = np.concatenate([np.zeros((n, 1, c)), E[:, :-1]], 1)
    pm = np.concatenate([np.abs(cs.h0)[:, None], size[:, :-1]], 1)
    # a of 2^-126 at the least where the formula's is below it
    floor = 2.0 ** -126 * (G + 1) * (pm + np.abs(x) + 1)
    tolx = na * EG + big * EPS32 * na * G + floor
    tolz = a * na * ((EG + big * EPS32 * G) * (pm + np.abs(x)) + G * Eprev) + floor
    dx, dz, dh0 = Rows("f32", n * t, c), Rows("f32", n * t, c), Rows("f32", n, c)
    D.dbl_gated_scan_bwd(cs.shape(D, D.DBL_F32), cs.dh.ptr(), torch.from_numpy(cs.dlast).cuda(), cs.px, cs.pz, st.ptr(), None,
                         dx.ptr(), dz.ptr(), dh0.ptr())
    check_status(D)
    assert_within(dx.values().reshape(n, t, c), wx, tolx + rounding("f32", np.abs(wx) + tolx), "dx")
    assert_within(dz.values().reshape(n, t, c), wz, tolz + rounding("f32", np.abs(wz) + tolz), "dgate")
    first = a[:, 0] * (EG[:, 0] + big * EPS32 * G[:, 0]) + floor[:, 0]
    assert_within(dh0.values(), w0, first + rounding("f32", np.abs(w0)), "dh0")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("t,c", [(16, 64), (200, 64), (200, 63), (3000, 16)])
def test_a_closed_gate_ends_finite_states_only(D, kind, t, c):
    """A gate of -infinity is 2^-126: it takes the input in the place of a finite state, and leaves an infinite state
    infinite and NaN NaN, each in its channel alone."""
    at = t // 2
    cs = Case(kind, 1, t, c)
    base = run(D, cs)[0].values()
    cs.rz.view()[at] = -np.inf
    cs.rx.view()[at - 1, 5] = float("nan")
    cs.h0[0, 9] = np.inf
    cs.th0.copy_(torch.from_numpy(cs.h0))
    h = run(D, cs)[0].values()
    rest = [i for i in range(c) if i not in (5, 9)]
    assert np.array_equal(h[:at, rest], base[:at, rest])
    assert np.array_equal(h[at, rest], cs.rx.values()[at, rest]) and np.isfinite(h[:, rest]).all()
    assert np.isnan(h[at - 1:, 5]).all() and np.isfinite(h[:at - 1, 5]).all()
    assert (h[:, 9] == np.inf).all()
