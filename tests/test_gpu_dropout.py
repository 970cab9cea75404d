"""Dropout over tokens with the residual addition against the 64-bit form: the mask bit for bit, the values within the
roundings of fp32 arithmetic and storage."""
import numpy as np
import pytest
import torch

from gpu_common import check_status, load_dbl, rng
from oracle import experts as orc
from token_cases import DTYPE, EPS32, Rows, assert_within, precision, rounding

pytestmark = pytest.mark.gpu

SEED, STEP = 0xFEDCBA9876543210, (1 << 32) + 7


def step_of(v):
    return torch.tensor([v - 2 ** 64 if v >= 2 ** 63 else v], dtype=torch.int64, device="cuda")


def expected(x, rate, seed, step, res):
    """The value and the bound of its error before it is stored: 1/(1 - rate) is rounded to fp32, then one fused
    multiplication and addition."""
    y = orc.dropout(x, rate, seed, step, res)
    kept = orc.dropout(x, rate, seed, step)
    return y, EPS32 * (np.abs(kept) * 1.01 + np.abs(y) * 1.01)


CASES = [  # rows, c, stride of what is read, of what is written, offset, rate, residual
    (1, 1, 0, 0, 0, 0.5, True), (3, 7, 0, 0, 0, 0.3, True), (5, 8, 0, 0, 0, 0.1, False), (64, 64, 0, 0, 0, 0.2, True),
    (33, 130, 144, 136, 0, 0.3, True), (33, 136, 144, 152, 0, 0.9, True), (9, 1000, 0, 0, 0, 0.1, True),
    (17, 1001, 0, 0, 0, 0.25, True), (40, 513, 520, 520, 1, 0.1, False), (21, 256, 264, 0, 3, 0.6, True),
    (300, 512, 0, 0, 0, 0.0, True), (2, 40000, 0, 0, 0, 0.5, True), (1000, 4, 0, 0, 0, 0.5, False),
    (777, 3, 0, 0, 0, 0.5, True), (500, 12, 0, 0, 2, 0.5, True), (2000, 264, 0, 0, 0, 0.3, True)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_dropout(kind, case):
    D = load_dbl()
    rows, c, ld_in, ld_out, offset, rate, with_res = case
    g = rng(rows * 1000 + c)
    x = Rows(kind, rows, c, ld_in, offset, g.standard_normal((rows, c)))
    res = Rows(kind, rows, c, ld_in, offset, g.standard_normal((rows, c)) * 2) if with_res else None
    y = Rows(kind, rows, c, ld_out, offset)
    fmt, dtype = precision(D, kind)
    with fmt:
        D.dbl_dropout_residual(D.dropout_shape(rows, c, rate, SEED, dtype, ld_in, ld_out), x.ptr(), res and res.ptr(),
                               step_of(STEP), y.ptr())
    torch.cuda.synchronize()
    want, tol = expected(x.values(), rate, SEED, STEP, res and res.values())
    assert_within(y.values(), want, tol + rounding(kind, np.abs(want) + tol), "y")
    if not with_res:
        keep = orc.dropout_mask(rows, c, rate, SEED, STEP)
        assert ((y.values() != 0) == keep).all()
    for t in (x, y) + ((res,) if with_res else ()):
        t.check_guards()
    check_status(D)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("place", ["x", "res"])
def test_in_place(kind, place):
    D = load_dbl()
    g = rng(5)
    rows, c = 37, 200
    x, res = (torch.from_numpy(g.standard_normal((rows, c))).to(DTYPE[kind]).cuda() for _ in range(2))
    want = torch.empty_like(x)
    fmt, dtype = precision(D, kind)
    shape = D.dropout_shape(rows, c, 0.3, SEED, dtype)
    with fmt:
        D.dbl_dropout_residual(shape, x, res, step_of(STEP), want)
        out = x if place == "x" else res
        D.dbl_dropout_residual(shape, x, res, step_of(STEP), out)
    assert torch.equal(out, want)


def test_what_is_dropped_may_hold_anything():
    D = load_dbl()
    rows, c = 50, 96
    keep = torch.from_numpy(orc.dropout_mask(rows, c, 0.5, SEED, STEP)).cuda()
    x = torch.ones((rows, c), dtype=torch.bfloat16, device="cuda")
    x[~keep] = float("nan")
    y = torch.empty_like(x)
    D.dbl_dropout_residual(D.dropout_shape(rows, c, 0.5, SEED), x, None, step_of(STEP), y)
    assert torch.equal(y, torch.where(keep, 2.0, 0.0).to(torch.bfloat16))


def test_gradient_by_differences():
    """The map is linear, so its slope is its value at a unit input: the backward pass is the same call."""
    D = load_dbl()
    rows, c, rate = 6, 20, 0.4
    g = rng(8)
    shape, step = D.dropout_shape(rows, c, rate, 77, D.DBL_F32), step_of(3)
    call = lambda a, r=None: D.dbl_dropout_residual(shape, a, r, step, out) or out.double().cpu().numpy()
    out = torch.empty((rows, c), device="cuda")
    x, res, dy, dskip = (torch.from_numpy(g.standard_normal((rows, c)).astype(np.float32)).cuda() for _ in range(4))
    dx = call(dy, dskip).copy()
    d = torch.zeros_like(x)
    for i, j in [(0, 0), (1, 3), (2, 19), (5, 7), (3, 11)]:
        d.zero_()
        d[i, j] = 0.5
        up, down = call(x + d, res).copy(), call(x - d, res).copy()
        slope = ((up - down) * dy.double().cpu().numpy()).sum() + float(dskip[i, j])
        # |x| + 0.5 below 5, scaled and added: each of the two values is off by 2^-24 of 20 at most
        assert abs(dx[i, j] - slope) < 4 * 2.0 ** -24 * 20


def test_a_captured_step_draws_new_masks():
    D = load_dbl()
    rows, c, rate = 64, 128, 0.5
    shape, step = D.dropout_shape(rows, c, rate, SEED), step_of(2 ** 64 - 2)
    x = torch.ones((rows, c), dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        D.dbl_dropout_residual(shape, x, None, step, y)
        D.dbl_dropout_advance(step)
    for at in (2 ** 64 - 2, 2 ** 64 - 1, 0, 1):  # the counter wraps
        graph.replay()
        torch.cuda.synchronize()
        assert ((y.float().cpu().numpy() != 0) == orc.dropout_mask(rows, c, rate, SEED, at)).all()
    assert int(step[0]) == 2


def test_many_elements_and_rows_past_2_to_the_31():
    """Offsets and block numbers past 32 bits: the last rows of a tensor of 2^31 + elements, and a stride that leaves them."""
    D = load_dbl()
    rows, c, ld = 5, 64, (1 << 29) + 8
    buf = torch.zeros((rows - 1) * ld + c, dtype=torch.bfloat16, device="cuda")
    view = buf.as_strided((rows, c), (ld, 1))
    view.fill_(1.0)
    D.dbl_dropout_residual(D.dropout_shape(rows, c, 0.5, SEED, ld_in=ld, ld_out=ld), buf, None, step_of(STEP), buf)
    assert ((view.float().cpu().numpy() != 0) == orc.dropout_mask(rows, c, 0.5, SEED, STEP)).all()
    del buf, view
    rows, c = (1 << 20) + 3, 2052
    x = torch.ones((rows, c), dtype=torch.bfloat16, device="cuda")
    D.dbl_dropout_residual(D.dropout_shape(rows, c, 0.5, SEED), x, None, step_of(STEP), x)
    for r in (0, 1 << 19, rows - 7):
        assert ((x[r:r + 7].float().cpu().numpy() != 0) == orc.dropout_mask(7, c, 0.5, SEED, STEP, row0=r)).all()
