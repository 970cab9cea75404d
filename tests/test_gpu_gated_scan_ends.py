"""The gated scan where states, inputs or gradients are infinite, against the recurrence step by step in 64 bits.

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
