"""Calls whose output takes an input's place, in every form that the rows' length and alignment choose (neighbouring rows share
units of 16 bytes in most): the same bits as beside it.  And a slot that two entries name."""
import numpy as np
import pytest
import torch

from gpu_common import check_status, load_dbl, rng
from oracle import experts as orc
from test_gpu_dropout import SEED, STEP, step_of
from test_gpu_exchange import setup, shape_of
from token_cases import EPS32, Rows, assert_within, precision, rounding

pytestmark = pytest.mark.gpu

EXCHANGE = [  # rows, k, c, stride of tokens, of grouped rows, offset, grouped rows (0: as many as entries)
    (9, 4, 777, 779, 781, 3, 50), (6, 3, 4001, 4003, 4005, 1, 0), (70, 2, 270, 0, 271, 0, 0), (12, 2, 515, 0, 0, 7, 30),
    (5, 2, 2050, 2051, 2053, 5, 0), (4, 3, 1031, 1034, 1036, 2, 0), (1000, 2, 257, 0, 0, 1, 0), (400, 3, 1001, 0, 0, 0, 0),
    (300, 2, 70, 0, 0, 1, 0), (90, 2, 1002, 0, 0, 0, 0), (90, 2, 1004, 0, 0, 0, 0), (50, 3, 1000, 0, 0, 0, 0),
    # rows read again for every entry, by 4, 8 and 16 bytes
    (5, 2, 1026, 1027, 1029, 1, 0), (7, 2, 2054, 0, 0, 0, 0), (7, 3, 4100, 0, 0, 0, 0), (3, 2, 9000, 0, 0, 0, 0)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("case", EXCHANGE, ids=str)
def test_combine_bwd_in_place(kind, case, weighted):
    D = load_dbl()
    g, s, slots, tokens, grouped, total = setup(kind, case)
    rows, k, c = case[:3]
    dout, yg, dyg = tokens(g.standard_normal((rows, c))), grouped(g.standard_normal((total, c))), grouped()
    w = g.standard_normal((rows, k)).astype(np.float32) if weighted else None
    wt = None if w is None else torch.from_numpy(w).cuda()
    dw, beside = (torch.full((rows, k), float("nan"), device="cuda") for _ in range(2))
    before = yg.values()
    fmt, dtype = precision(D, kind)
    shape = shape_of(D, case, dtype)
    with fmt:
        D.dbl_expert_combine_bwd(shape, dout.ptr(), yg.ptr(), slots, wt, dyg.ptr(), beside)
        D.dbl_expert_combine_bwd(shape, dout.ptr(), yg.ptr(), slots, wt, yg.ptr(), dw)
    torch.cuda.synchronize()
    named = np.zeros(total, bool)
    named[[v for v in s.reshape(-1) if 0 <= v < total]] = True
    assert torch.equal(dw, beside)
    assert (yg.values()[named] == dyg.values()[named]).all() and (yg.values()[~named] == before[~named]).all()
    want, want_dw, size = orc.combine_bwd(dout.values(), before, s, w, before)
    tol = EPS32 * np.abs(want)
    assert_within(yg.values(), want, np.where(named[:, None], tol + rounding(kind, np.abs(want) + tol), 0), "dyg")
    assert_within(dw.double().cpu().numpy(), want_dw, 1.01 * (c + 1) * EPS32 * size, "dweights")
    for t in (dout, yg, dyg):
        t.check_guards()
    check_status(D)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("place", ["x", "res", "x without res"])
@pytest.mark.parametrize("case", [(40, 513, 520, 1), (300, 1001, 0, 0), (200, 130, 0, 2), (200, 1004, 0, 0), (500, 7, 0, 1),
                                  (777, 3, 0, 0), (900, 12, 0, 2), (64, 2050, 2051, 3), (64, 512, 0, 0)], ids=str)
def test_dropout_in_place(kind, place, case):
    D = load_dbl()
    rows, c, ld, offset = case
    g = rng(rows + c)
    x, res = (Rows(kind, rows, c, ld, offset, g.standard_normal((rows, c))) for _ in range(2))
    want = Rows(kind, rows, c, ld, offset)
    fmt, dtype = precision(D, kind)
    shape = D.dropout_shape(rows, c, 0.3, SEED, dtype, ld, ld)
    added, out = (None if place.endswith("without res") else res.ptr()), (res if place == "res" else x)
    with fmt:
        D.dbl_dropout_residual(shape, x.ptr(), added, step_of(STEP), want.ptr())
        D.dbl_dropout_residual(shape, x.ptr(), added, step_of(STEP), out.ptr())
    assert torch.equal(out.view(), want.view())
    for t in (x, res, want):
        t.check_guards()
    check_status(D)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("c", [8, 129, 1001, 2048])
def test_a_slot_that_two_tokens_name(kind, c):
    """Every element of its row is one of the two's; the other rows are as without it."""
    D = load_dbl()
    g = rng(c)
    rows, k = 64, 2
    s = g.permutation(rows * k).reshape(rows, k).astype(np.int32)
    first, second = (3, 1), (50, 0)
    s[second] = s[first]
    slots = torch.from_numpy(s).cuda()
    x, xg, dyg = Rows(kind, rows, c, values=g.standard_normal((rows, c))), Rows(kind, rows * k, c), Rows(kind, rows * k, c)
    fmt, dtype = precision(D, kind)
    shape = D.exchange_shape(rows, k, c, dtype)
    with fmt:
        D.dbl_expert_scatter(shape, x.ptr(), slots, xg.ptr())
        D.dbl_expert_combine_bwd(shape, x.ptr(), None, slots, None, dyg.ptr(), None)
    v, shared = x.values(), int(s[first])
    for out in (xg, dyg):
        got = out.values()
        assert ((got[shared] == v[first[0]]) | (got[shared] == v[second[0]])).all()
        for r in range(rows):
            for j in range(k):
                assert s[r, j] == shared or (got[s[r, j]] == v[r]).all()
        out.check_guards()
    check_status(D)
