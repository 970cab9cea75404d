"""Argument checks of the token operators: refused on the host, before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2509_26092_gb300 import build_lib

P = 4096  # an aligned address that no refused call touches


@pytest.fixture(scope="module")
def D():
    build_lib.build()
    from paper_2509_26092_gb300 import dbl
    return dbl


def refused(D, code, f, *args):
    with pytest.raises(D.DblError) as e:
        f(*args, stream=0)
    assert e.value.code == code and str(e.value)


@pytest.mark.parametrize("prec", ["bf16", "f16"])
def test_layer_norm_refusals(D, prec):
    ok = D.ln_shape(4, 8)
    fwd = lambda s=ok, x=P, res=None, g=P, b=P, sm=None, y=P, m=P, i=P: (s, x, res, g, b, sm, y, m, i)
    bwd = lambda s=ok, dy=P, sk=None, x=P, g=P, m=P, i=P, dx=P, dg=P, db=P, ws=P, n=1 << 20: (s, dy, sk, x, g, m, i, dx,
                                                                                              dg, db, ws, n)
    INV = D.DBL_ERR_INVALID
    with D.precision(prec):
        for s in (D.ln_shape(-1, 8), D.ln_shape(4, 0), D.ln_shape(4, 8, 1e-5, 2), D.ln_shape(4, 8, -1.0),
                  D.ln_shape(4, 8, float("nan")), D.ln_shape(4, 8, float("inf")), D.ln_shape(4, 8, 1e-5, 1, 7),
                  D.ln_shape(4, 8, 1e-5, 1, 8, 7), D.ln_shape(4, 8, 1e-5, 1, -8)):
            refused(D, INV, D.dbl_layer_norm_fwd, *fwd(s))
            refused(D, INV, D.dbl_layer_norm_bwd, *bwd(s))
            assert D.dbl_layer_norm_workspace_bytes(s) == 0
        for kw in (dict(x=None), dict(y=None), dict(m=None), dict(i=None), dict(x=P + 1), dict(y=P + 1),
                   dict(res=P + 1), dict(sm=P + 1), dict(g=P + 2), dict(b=P + 2), dict(m=P + 2)):
            refused(D, INV, D.dbl_layer_norm_fwd, *fwd(**kw))
        for kw in (dict(dy=None), dict(x=None), dict(m=None), dict(i=None), dict(dx=None), dict(dg=None), dict(db=None),
                   dict(dy=P + 1), dict(sk=P + 1), dict(dx=P + 1), dict(dg=P + 2), dict(ws=P + 4)):
            refused(D, INV, D.dbl_layer_norm_bwd, *bwd(**kw))
        need = D.dbl_layer_norm_workspace_bytes(ok)
        assert need > 0
        refused(D, D.DBL_ERR_WORKSPACE, D.dbl_layer_norm_bwd, *bwd(n=need - 1))
        refused(D, D.DBL_ERR_WORKSPACE, D.dbl_layer_norm_bwd, *bwd(ws=None))
    L = D.lib()
    assert L.dbl_layer_norm_fwd(None, P, None, P, P, None, P, P, P, None) == INV
    assert L.dbl_layer_norm_workspace_bytes(None) == 0


@pytest.mark.parametrize("prec", ["bf16", "f16"])
def test_gated_scan_refusals(D, prec):
    ok = D.scan_shape(2, 100, 8)
    fwd = lambda s=ok, x=P, g=P, h0=P, ln=P, h=P, la=P, st=P: (s, x, g, h0, ln, h, la, st)
    bwd = lambda s=ok, dh=P, dl=P, x=P, g=P, st=P, ln=P, dx=P, dg=P, d0=P: (s, dh, dl, x, g, st, ln, dx, dg, d0)
    INV = D.DBL_ERR_INVALID
    with D.precision(prec):
        for s in (D.scan_shape(-1, 4, 8), D.scan_shape(2, -1, 8), D.scan_shape(2, 4, 0), D.scan_shape(2, 4, 8, 3),
                  D.scan_shape(2, 4, 8, 1, 7), D.scan_shape(2, 4, 8, 1, 8, 7)):
            refused(D, INV, D.dbl_gated_scan_fwd, *fwd(s))
            refused(D, INV, D.dbl_gated_scan_bwd, *bwd(s))
            assert D.dbl_gated_scan_states_bytes(s) == 0 and D.dbl_gated_scan_workspace_bytes(s, D.DBL_PASS_FWD) == 0
        for kw in (dict(x=None), dict(g=None), dict(h=None), dict(x=P + 1), dict(g=P + 1), dict(h=P + 1), dict(h0=P + 2),
                   dict(ln=P + 2), dict(la=P + 2), dict(st=P + 2)):
            refused(D, INV, D.dbl_gated_scan_fwd, *fwd(**kw))
        for kw in (dict(dh=None), dict(x=None), dict(g=None), dict(st=None), dict(dx=None), dict(dg=None),
                   dict(dh=P + 1), dict(dx=P + 1), dict(dg=P + 1), dict(dl=P + 2), dict(d0=P + 2), dict(st=P + 2)):
            refused(D, INV, D.dbl_gated_scan_bwd, *bwd(**kw))
        assert D.dbl_gated_scan_states_bytes(ok) == 4 * 2 * 2 * 8
        assert D.dbl_gated_scan_states_bytes(D.scan_shape(2, 0, 8)) == 0
        assert D.dbl_gated_scan_states_bytes(D.scan_shape(3, 1 << 30, 4096)) == 4 * 3 * (1 << 24) * 4096
    assert D.lib().dbl_gated_scan_states_bytes(None) == 0


@pytest.mark.parametrize("prec", ["bf16", "f16"])
def test_distill_refusals(D, prec):
    ok = D.distill_shape(4, 10, 3)
    a = lambda s=ok, z=P, t=P, c=P, la=P, w=P, sc=P, rl=P, lo=P, dz=P + 1024: (s, z, t, c, la, w, sc, rl, lo, dz)
    INV = D.DBL_ERR_INVALID
    nan, inf = float("nan"), float("inf")
    with D.precision(prec):
        for s in (D.distill_shape(-1, 10, 3), D.distill_shape(4, 0, 3), D.distill_shape(4, 10, -1),
                  D.distill_shape(4, 10, 3, 0.0), D.distill_shape(4, 10, 3, -1.0), D.distill_shape(4, 10, 3, nan),
                  D.distill_shape(4, 10, 3, inf), D.distill_shape(4, 10, 3, 1.0, -0.1), D.distill_shape(4, 10, 3, 1.0, 1.1),
                  D.distill_shape(4, 10, 3, 1.0, nan), D.distill_shape(4, 10, 3, 1.0, 0.5, 7),
                  D.distill_shape(4, 10, 3, 1.0, 0.5, 1, 9), D.distill_shape(4, 10, 3, 1.0, 0.5, 1, 10, 9)):
            refused(D, INV, D.dbl_distill_fwd_bwd, *a(s))
        refused(D, D.DBL_ERR_UNSUPPORTED, D.dbl_distill_fwd_bwd, *a(D.distill_shape(4, 10, D.DBL_DISTILL_MAX_K + 1)))
        for kw in (dict(z=None), dict(t=None), dict(c=None), dict(rl=None), dict(z=P + 1), dict(dz=P + 1), dict(t=P + 2),
                   dict(c=P + 2), dict(la=P + 2), dict(w=P + 2), dict(sc=P + 2), dict(rl=P + 2), dict(lo=P + 2)):
            refused(D, INV, D.dbl_distill_fwd_bwd, *a(**kw))
        refused(D, INV, D.dbl_distill_fwd_bwd, *a(D.distill_shape(4, 10, 3, 1.0, 0.5, 1, 16, 24), dz=P))  # in place
    assert D.lib().dbl_distill_fwd_bwd(None, P, P, P, P, P, P, P, P, P, None) == INV
    assert ctypes.sizeof(D.DistillShape) == 48 and ctypes.sizeof(D.LnShape) == 40 and ctypes.sizeof(D.ScanShape) == 32
