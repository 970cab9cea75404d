"""Argument checks of the expert layer and the token dropout: refused on the host, before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2509_26092_gb300 import build_lib

P = 4096  # an aligned address that no refused call touches
TOP = 2 ** 31 - 1


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
def test_route_refusals(D, prec):
    ok, INV, UNS = D.route_shape(100, 16, 2), D.DBL_ERR_INVALID, D.DBL_ERR_UNSUPPORTED
    fwd = lambda s=ok, z=P, b=P, rw=P, c=P, w=P, sl=P, o=P, ws=P, n=1 << 24: (s, z, b, rw, c, w, sl, o, ws, n)
    bwd = lambda s=ok, z=P, c=P, w=P, dw=P, dz=P: (s, z, c, w, dw, dz)
    with D.precision(prec):
        for s in (D.route_shape(-1, 16, 2), D.route_shape(4, 0, 1), D.route_shape(4, 16, 0), D.route_shape(4, 16, 17),
                  D.route_shape(4, 16, 2, dtype=2), D.route_shape(4, 16, 2, ld=15), D.route_shape(4, 16, 2, ld_grad=15),
                  D.route_shape(4, 16, 2, ld=-16)):
            refused(D, INV, D.dbl_route_fwd, *fwd(s))
            refused(D, INV, D.dbl_route_bwd, *bwd(s))
            assert D.dbl_route_workspace_bytes(s) == 0
        for s in (D.route_shape(4, 1025, 2), D.route_shape(4, 64, 33), D.route_shape(1 << 30, 16, 2),
                  D.route_shape((1 << 63) - 1, 16, 2)):
            refused(D, UNS, D.dbl_route_fwd, *fwd(s))
            refused(D, UNS, D.dbl_route_bwd, *bwd(s))
        for kw in (dict(z=None), dict(c=None), dict(w=None), dict(sl=None), dict(o=None), dict(z=P + 1), dict(b=P + 2),
                   dict(rw=P + 2), dict(c=P + 2), dict(w=P + 2), dict(sl=P + 2), dict(o=P + 2), dict(ws=P + 8)):
            refused(D, INV, D.dbl_route_fwd, *fwd(**kw))
        many = D.route_shape(65536, 16, 2)
        need = D.dbl_route_workspace_bytes(many)
        assert need > 0
        refused(D, D.DBL_ERR_WORKSPACE, D.dbl_route_fwd, *fwd(many, n=need - 1))
        refused(D, D.DBL_ERR_WORKSPACE, D.dbl_route_fwd, *fwd(many, ws=None))
        for kw in (dict(c=None), dict(w=None), dict(dw=None), dict(dz=None), dict(z=P + 1), dict(c=P + 2), dict(w=P + 2),
                   dict(dw=P + 2), dict(dz=P + 1)):
            refused(D, INV, D.dbl_route_bwd, *bwd(**kw))
        refused(D, INV, D.dbl_route_bwd, *bwd(D.route_shape(4, 16, 2, normalise=False), z=None))
    assert D.lib().dbl_route_fwd(None, P, P, P, P, P, P, P, P, 0, None) == INV
    assert D.lib().dbl_route_workspace_bytes(None) == 0


@pytest.mark.parametrize("prec", ["bf16", "f16"])
def test_exchange_refusals(D, prec):
    ok, INV, UNS = D.exchange_shape(4, 2, 8), D.DBL_ERR_INVALID, D.DBL_ERR_UNSUPPORTED
    calls = {D.dbl_expert_scatter: lambda s=ok, x=P, sl=P, g=P: (s, x, sl, g),
             D.dbl_expert_combine: lambda s=ok, g=P, sl=P, w=P, r=P, x=P: (s, g, sl, w, r, x),
             D.dbl_expert_combine_bwd: lambda s=ok, x=P, y=P, sl=P, w=P, g=P, dw=P: (s, x, y, sl, w, g, dw)}
    with D.precision(prec):
        for f, a in calls.items():
            for s in (D.exchange_shape(-1, 2, 8), D.exchange_shape(4, 0, 8), D.exchange_shape(4, 2, 0),
                      D.exchange_shape(4, 2, 8, dtype=2), D.exchange_shape(4, 2, 8, grouped_rows=-1),
                      D.exchange_shape(4, 2, 8, ld_rows=7), D.exchange_shape(4, 2, 8, ld_grouped=7)):
                refused(D, INV, f, *a(s))
            for s in (D.exchange_shape(4, 2, 1 << 30), D.exchange_shape(4, 33, 8), D.exchange_shape(1 << 30, 2, 8)):
                refused(D, UNS, f, *a(s))
            for kw in (dict(x=None), dict(sl=None), dict(g=None), dict(x=P + 1), dict(g=P + 1), dict(sl=P + 2)):
                refused(D, INV, f, *a(**kw))
        for kw in (dict(w=P + 2), dict(r=P + 1)):
            refused(D, INV, D.dbl_expert_combine, *calls[D.dbl_expert_combine](**kw))
        for kw in (dict(w=P + 2), dict(y=P + 1), dict(dw=P + 2), dict(y=None)):
            refused(D, INV, D.dbl_expert_combine_bwd, *calls[D.dbl_expert_combine_bwd](**kw))
    assert D.lib().dbl_expert_scatter(None, P, P, P, None) == INV


@pytest.mark.parametrize("prec", ["bf16", "f16"])
def test_grouped_refusals(D, prec):
    ok, INV, UNS = D.grouped_shape(100, 4, 16, 24), D.DBL_ERR_INVALID, D.DBL_ERR_UNSUPPORTED
    calls = {D.dbl_grouped_fwd: (D.DBL_PASS_FWD, lambda s=ok, a=P, b=P, o=P, y=P, ws=P, n=1 << 30: (s, a, b, o, y, ws, n)),
             D.dbl_grouped_dgrad: (D.DBL_PASS_DGRAD, lambda s=ok, a=P, b=P, o=P, m=P, y=P, ws=P, n=1 << 30: (s, a, b, o, m, y,
                                                                                                    ws, n)),
             D.dbl_grouped_wgrad: (D.DBL_PASS_WGRAD, lambda s=ok, a=P, b=P, o=P, y=P, ws=P, n=1 << 30: (s, a, b, o, y, False,
                                                                                               ws, n))}
    with D.precision(prec):
        for f, (which, a) in calls.items():
            for s in (D.grouped_shape(-1, 4, 16, 24), D.grouped_shape(100, 0, 16, 24), D.grouped_shape(100, 4, 0, 24),
                      D.grouped_shape(100, 4, 16, 0), D.grouped_shape(100, 4, 12, 24), D.grouped_shape(100, 4, 16, 20),
                      D.grouped_shape(100, 4, 16, 24, ld_in=8), D.grouped_shape(100, 4, 16, 24, ld_out=16),
                      D.grouped_shape(100, 4, 16, 24, ld_in=20), D.grouped_shape(100, 4, 16, 24, ld_out=28)):
                refused(D, INV, f, *a(s))
                assert D.dbl_grouped_workspace_bytes(s, which) == 0
            for s in (D.grouped_shape(100, 1025, 16, 24), D.grouped_shape((1 << 30) + 1, 4, 16, 24),
                      D.grouped_shape(100, 4, 1 << 24, 24), D.grouped_shape(100, 4, 16, 1 << 24)):
                refused(D, UNS, f, *a(s))
            for kw in (dict(a=None), dict(b=None), dict(o=None), dict(y=None), dict(a=P + 8), dict(b=P + 8), dict(y=P + 8),
                       dict(o=P + 2)):
                refused(D, INV, f, *a(**kw))
        refused(D, INV, D.dbl_grouped_dgrad, *calls[D.dbl_grouped_dgrad][1](m=P + 8))
        for f, s in ((D.dbl_grouped_fwd, D.grouped_shape(8, 1, 4096, 256)), (D.dbl_grouped_dgrad, D.grouped_shape(8, 1, 256, 4096)),
                     (D.dbl_grouped_wgrad, D.grouped_shape(9000, 1, 256, 256))):
            which, a = calls[f]
            need = D.dbl_grouped_workspace_bytes(s, which)
            assert need > 0 and D.dbl_grouped_workspace_bytes(s, 3) == D.dbl_grouped_workspace_bytes(s, -1) == 0
            refused(D, D.DBL_ERR_WORKSPACE, f, *a(s, n=need - 1))
            refused(D, D.DBL_ERR_WORKSPACE, f, *a(s, ws=None))
            refused(D, INV, f, *a(s, ws=P + 8))
    assert D.lib().dbl_grouped_fwd(None, P, P, P, P, None, 0, None) == INV
    assert D.lib().dbl_grouped_workspace_bytes(None, 0) == 0


@pytest.mark.parametrize("prec", ["bf16", "f16"])
def test_dropout_refusals(D, prec):
    ok, INV = D.dropout_shape(4, 8, 0.1, 1), D.DBL_ERR_INVALID
    a = lambda s=ok, x=P, r=P + 1024, st=P, y=P + 2048: (s, x, r, st, y)
    with D.precision(prec):
        for s in (D.dropout_shape(-1, 8, 0.1, 1), D.dropout_shape(4, 0, 0.1, 1), D.dropout_shape(4, 8, 1.0, 1),
                  D.dropout_shape(4, 8, -0.1, 1), D.dropout_shape(4, 8, float("nan"), 1), D.dropout_shape(4, 8, 0.1, 1, 2),
                  D.dropout_shape(4, 8, 0.1, 1, ld_in=7), D.dropout_shape(4, 8, 0.1, 1, ld_out=7)):
            refused(D, INV, D.dbl_dropout_residual, *a(s))
        refused(D, D.DBL_ERR_UNSUPPORTED, D.dbl_dropout_residual, *a(D.dropout_shape(1, 1 << 30, 0.1, 1)))
        for kw in (dict(x=None), dict(st=None), dict(y=None), dict(x=P + 1), dict(r=P + 1), dict(y=P + 1), dict(st=P + 4)):
            refused(D, INV, D.dbl_dropout_residual, *a(**kw))
        in_place = D.dropout_shape(4, 8, 0.1, 1, ld_in=16, ld_out=8)
        refused(D, INV, D.dbl_dropout_residual, *a(in_place, y=P))
        refused(D, INV, D.dbl_dropout_residual, *a(in_place, r=P + 2048))
        refused(D, INV, D.dbl_dropout_advance, None)
        refused(D, INV, D.dbl_dropout_advance, P + 4)
    assert D.lib().dbl_dropout_residual(None, P, None, P, P, None) == INV


def test_the_shapes_are_laid_out_as_in_the_header(D):
    assert ctypes.sizeof(D.RouteShape) == 40 and ctypes.sizeof(D.ExchangeShape) == 48
    assert ctypes.sizeof(D.GroupedShape) == 40 and ctypes.sizeof(D.DropoutShape) == 48
    assert D.DropoutShape.seed.offset == 32 and D.ExchangeShape.grouped_rows.offset == 24
