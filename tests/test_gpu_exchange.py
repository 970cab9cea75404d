"""Tokens to their experts' groups and back against the 64-bit form."""
import numpy as np
import pytest
import torch

from gpu_common import check_status, load_dbl, rng
from oracle import experts as orc
from token_cases import EPS32, GUARD, Rows, assert_within, precision, rounding

pytestmark = pytest.mark.gpu

CASES = [  # rows, k, c, stride of tokens, of grouped rows, offset, grouped rows (0: as many as entries)
    (1, 1, 1, 0, 0, 0, 0), (1, 8, 2048, 0, 0, 0, 0), (7, 2, 8, 0, 0, 0, 0), (40, 2, 64, 0, 0, 0, 0),
    (33, 3, 130, 136, 144, 0, 0), (33, 4, 136, 144, 152, 0, 100), (20, 2, 1000, 0, 0, 0, 0), (17, 5, 1001, 0, 0, 0, 0),
    (16, 2, 513, 520, 520, 1, 40), (9, 32, 256, 264, 0, 3, 0), (3, 2, 9000, 0, 0, 0, 0), (400, 2, 12, 0, 0, 0, 0),
    (50, 6, 36, 0, 40, 2, 200), (257, 1, 72, 0, 0, 0, 0), (11, 7, 4100, 0, 0, 0, 0),
    (42, 2, 1170, 0, 0, 4, 0), (9, 2, 1602, 1604, 0, 2, 0), (6, 3, 4001, 4003, 4005, 1, 0), (9, 4, 777, 779, 781, 3, 50),
    (5, 2, 2050, 2051, 2053, 5, 0), (70, 2, 270, 0, 271, 0, 0), (4, 3, 1031, 1034, 1036, 2, 0), (12, 2, 515, 0, 0, 7, 30), (8, 3, 519, 522, 521, 0, 0)]


def slots_of(g, rows, k, total):
    """Distinct places for most entries; some absent, some out of range, one row without any."""
    s = np.full(rows * k, -1, np.int64)
    n = min(rows * k, total)
    s[:n] = g.permutation(total)[:n]
    s = g.permutation(s).reshape(rows, k).astype(np.int32)
    if rows > 3:
        s[1] = -1
        s[2, 0] = -5 if rows % 2 else total
        s[rows - 1, k - 1] = 2 ** 31 - 1
    return s


def setup(kind, case):
    rows, k, c, ld_r, ld_g, offset, total = case
    total = total or rows * k
    g = rng(rows * 10000 + k * 100 + c)
    s = slots_of(g, rows, k, total)
    return g, s, torch.from_numpy(s).cuda(), lambda v=None: Rows(kind, rows, c, ld_r, offset, v), \
        lambda v=None: Rows(kind, total, c, ld_g, offset, v), total


def shape_of(D, case, dtype):
    rows, k, c, ld_r, ld_g, _, total = case
    return D.exchange_shape(rows, k, c, dtype, total, ld_r, ld_g)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_scatter(kind, case):
    D = load_dbl()
    g, s, slots, tokens, grouped, total = setup(kind, case)
    x, xg = tokens(g.standard_normal((case[0], case[2]))), grouped()
    fmt, dtype = precision(D, kind)
    with fmt:
        D.dbl_expert_scatter(shape_of(D, case, dtype), x.ptr(), slots, xg.ptr())
    torch.cuda.synchronize()
    want = orc.scatter(x.values(), s, np.full((total, case[2]), GUARD))  # rows without an entry stay as they were
    assert (xg.values() == want).all()
    x.check_guards()
    xg.check_guards()
    check_status(D)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("weighted,with_res", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_combine(kind, case, weighted, with_res):
    D = load_dbl()
    g, s, slots, tokens, grouped, total = setup(kind, case)
    rows, k, c = case[:3]
    yg, out = grouped(g.standard_normal((total, c))), tokens()
    res = tokens(g.standard_normal((rows, c))) if with_res else None
    w = g.random((rows, k)).astype(np.float32) if weighted else None
    fmt, dtype = precision(D, kind)
    with fmt:
        D.dbl_expert_combine(shape_of(D, case, dtype), yg.ptr(), slots, None if w is None else torch.from_numpy(w).cuda(),
                             res and res.ptr(), out.ptr())
    torch.cuda.synchronize()
    want, size = orc.combine(yg.values(), s, w, res and res.values())
    # a product and an addition for every entry, one more for the residual, each rounded to fp32
    tol = 1.01 * (2 * k + 1) * EPS32 * size
    assert_within(out.values(), want, tol + rounding(kind, np.abs(want) + tol), "out")
    for t in (yg, out) + ((res,) if with_res else ()):
        t.check_guards()
    check_status(D)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("weighted,dots", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_combine_bwd(kind, case, weighted, dots):
    D = load_dbl()
    g, s, slots, tokens, grouped, total = setup(kind, case)
    rows, k, c = case[:3]
    dout, yg, dyg = tokens(g.standard_normal((rows, c))), grouped(g.standard_normal((total, c))), grouped()
    w = g.standard_normal((rows, k)).astype(np.float32) if weighted else None
    dw = torch.full((rows, k), float("nan"), device="cuda")
    fmt, dtype = precision(D, kind)
    with fmt:
        D.dbl_expert_combine_bwd(shape_of(D, case, dtype), dout.ptr(), yg.ptr() if dots else None, slots,
                                 None if w is None else torch.from_numpy(w).cuda(), dyg.ptr(), dw if dots else None)
    torch.cuda.synchronize()
    want, want_dw, size = orc.combine_bwd(dout.values(), yg.values(), s, w, np.full((total, c), GUARD))
    untouched = np.ones(total, bool)
    untouched[[v for v in s.reshape(-1) if 0 <= v < total]] = False
    assert (dyg.values()[untouched] == GUARD).all()
    tol = EPS32 * np.abs(want)
    assert_within(dyg.values(), want, np.where(untouched[:, None], 0, tol + rounding(kind, np.abs(want) + tol)), "dyg")
    if dots:
        assert_within(dw.double().cpu().numpy(), want_dw, 1.01 * (c + 1) * EPS32 * size, "dweights")
    for t in (dout, yg, dyg):
        t.check_guards()
    check_status(D)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_absent_entries_and_weights_that_are_not_numbers(kind):
    D = load_dbl()
    rows, k, c = 4, 2, 24
    s = torch.tensor([[0, 1], [-1, -1], [2, -1], [-1, -1]], dtype=torch.int32, device="cuda")
    nan = float("nan")
    w = torch.tensor([[1., 2.], [0., 0.], [3., nan], [nan, nan]], device="cuda")
    yg, res, out = Rows(kind, 8, c, values=np.ones((8, c))), Rows(kind, rows, c, values=np.ones((rows, c))), Rows(kind, rows, c)
    fmt, dtype = precision(D, kind)
    shape = D.exchange_shape(rows, k, c, dtype)
    dw = torch.empty((rows, k), device="cuda")
    with fmt:
        D.dbl_expert_combine(shape, yg.ptr(), s, w, res.ptr(), out.ptr())
        v = out.values()
        assert (v[0] == 4).all() and (v[1] == 1).all() and np.isnan(v[2:]).all()
        # a token's own rows alone: NaN in a row of the grouped tensor that no entry names does no harm
        yg.view()[5] = nan
        D.dbl_expert_combine(shape, yg.ptr(), s, None, None, out.ptr())
        assert out.values()[:, 0].tolist() == [2, 0, 1, 0]
        D.dbl_expert_combine_bwd(shape, res.ptr(), yg.ptr(), s, w, yg.ptr(), dw)  # in yg's own place
    assert dw.cpu().tolist() == [[c, c], [0, 0], [c, 0], [0, 0]]
    assert (yg.values()[:3] == np.array([1, 2, 3])[:, None]).all()


def test_weights_gradient_by_differences():
    """Slopes of the kernels' own forward pass, which is linear in each weight and in each grouped row."""
    D = load_dbl()
    g = rng(3)
    rows, k, c = 5, 3, 40
    shape = D.exchange_shape(rows, k, c, D.DBL_F32)
    new = lambda *n: torch.from_numpy(g.standard_normal(n).astype(np.float32)).cuda()
    slots = torch.from_numpy(g.permutation(15).reshape(5, 3).astype(np.int32)).cuda()
    yg, w, dout, out, dyg, dw = new(15, c), new(rows, k), new(rows, c), new(rows, c), new(15, c), new(rows, k)
    D.dbl_expert_combine_bwd(shape, dout, yg, slots, w, dyg, dw)

    def loss(w_, yg_):
        D.dbl_expert_combine(shape, yg_, slots, w_, None, out)
        return float((out.double() * dout.double()).sum())
    # every output is off by (2k + 1) 2^-24 of its terms, below 10; 40 columns of |dout| below 4 move
    tol = 2 * 7 * 2.0 ** -24 * 10 * 40 * 4
    for i, j in [(0, 0), (2, 1), (4, 2)]:
        d = torch.zeros_like(w)
        d[i, j] = 0.5
        assert abs(loss(w + d, yg) - loss(w - d, yg) - float(dw[i, j])) < tol
    for i, j in [(0, 0), (7, 39), (14, 5)]:
        d = torch.zeros_like(yg)
        d[i, j] = 0.5
        assert abs(loss(w, yg + d) - loss(w, yg - d) - float(dyg[i, j])) < tol


def test_offsets_past_2_to_the_31():
    """Grouped rows so far apart that their byte offsets pass 32 bits, and element offsets 2^31."""
    D = load_dbl()
    rows, k, c, ld = 3, 2, 64, (1 << 29) + 8
    buf = torch.zeros(5 * ld + c, dtype=torch.bfloat16, device="cuda")
    x = torch.arange(rows, device="cuda").to(torch.bfloat16)[:, None].expand(rows, c).contiguous() + 1
    slots = torch.tensor([[5, 0], [1, 4], [3, 2]], dtype=torch.int32, device="cuda")
    shape = D.exchange_shape(rows, k, c, ld_grouped=ld)
    D.dbl_expert_scatter(shape, x, slots, buf)
    assert buf.as_strided((6, c), (ld, 1))[:, 7].tolist() == [1, 2, 3, 3, 2, 1]
    out = torch.empty_like(x)
    D.dbl_expert_combine(shape, buf, slots, None, None, out)
    assert torch.equal(out, 2 * x)
    dw = torch.empty((rows, k), device="cuda")
    D.dbl_expert_combine_bwd(shape, x, buf, slots, torch.ones((rows, k), device="cuda"), buf, dw)
    assert dw.cpu().tolist() == [[64.] * 2, [256.] * 2, [576.] * 2]
