"""Grouped products against the 64-bit form: groups of any length, widths that end inside tiles, rows of no group."""
import numpy as np
import pytest
import torch

from gpu_common import check_status, load_dbl, rng, ws
from oracle import experts as orc
from token_cases import DTYPE, GUARD, Rows, assert_within, precision, rounding

pytestmark = pytest.mark.gpu

CASES = [  # lengths of the groups, rows past the last, n_in, n_out, strides beyond the rows
    ([1], 0, 8, 8, 0), ([3], 2, 64, 64, 0), ([0, 0], 5, 64, 128, 0), ([1, 0, 2], 0, 8, 264, 8), ([64], 0, 64, 256, 0),
    ([130, 1, 0, 7], 3, 72, 136, 0), ([256, 256], 0, 128, 256, 0), ([257, 255, 31], 1, 512, 520, 16),
    ([5, 9, 0, 1, 33, 127, 128, 129], 50, 200, 1000, 24), ([700], 0, 1000, 72, 0), ([40] * 20, 0, 256, 512, 0),
    ([0, 0, 1500, 0], 9, 264, 248, 8), ([16, 17, 15, 1, 2, 300], 0, 1032, 264, 0), ([2] * 70, 1, 64, 72, 0),
    ([600, 20, 1], 0, 2048, 96, 0), ([90, 70], 0, 96, 2056, 8),
    # few tiles and long reductions, which are split: in the groups' rows (the last with parts that get none of a group), in
    # n_in, in n_out
    ([5003], 2, 72, 64, 0), ([1500, 0, 2600], 3, 264, 136, 8), ([5000, 1, 40, 700], 0, 64, 200, 0), ([9], 1, 4104, 72, 0),
    ([33, 2], 0, 72, 3080, 0), ([i % 3 if i % 7 else 40 for i in range(1024)], 5, 64, 72, 0)]


def setup(kind, case):
    lengths, tail, n_in, n_out, pad = case
    rows = sum(lengths) + tail
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    g = rng(rows * 31 + n_in + n_out)
    x = lambda v=None: Rows(kind, rows, n_in, n_in + pad, 0, v)
    y = lambda v=None: Rows(kind, rows, n_out, n_out + pad, 0, v)
    return g, rows, off, torch.from_numpy(off).cuda(), x, y


def shape_of(D, case, relu=False):
    lengths, tail, n_in, n_out, pad = case
    return D.grouped_shape(sum(lengths) + tail, len(lengths), n_in, n_out, relu, n_in + pad, n_out + pad)


def scratch(D, shape, which):
    need = D.dbl_grouped_workspace_bytes(shape, which)
    return ws(need), need


def sum_error(terms, size):
    """Products of 16-bit values are exact in fp32.  A tensor core adds 16 of them and the sum so far with their
    digits cut at its largest, 2^-23 of it for each of the 17; sums of such chains, and of the CUDA cores, round
    at 2^-24.  The sums so far are below the sum of the magnitudes."""
    return (17 * (terms / 16 + 1) * 2.0 ** -23 + 16 * 2.0 ** -24) * size


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{sum(c[0])}-{c[2]}x{c[3]}")
def test_fwd(kind, relu, case):
    D = load_dbl()
    lengths, _, n_in, n_out, _ = case
    g, rows, off, offsets, x_of, y_of = setup(kind, case)
    x, y = x_of(g.standard_normal((rows, n_in))), y_of()
    w = torch.from_numpy(g.standard_normal((len(lengths), n_out, n_in)) / n_in ** 0.5).to(DTYPE[kind]).cuda()
    if rows > off[-1]:
        x.view()[int(off[-1]):] = float("nan")  # rows of no group
    fmt, _ = precision(D, kind)
    shape = shape_of(D, case, relu)
    with fmt:
        D.dbl_grouped_fwd(shape, x.ptr(), w, offsets, y.ptr(), *scratch(D, shape, D.DBL_PASS_FWD))
    torch.cuda.synchronize()
    xv, wv = np.nan_to_num(x.values()), w.double().cpu().numpy()
    want, live = orc.grouped_fwd(xv, wv, off, relu)
    size, _ = orc.grouped_fwd(np.abs(xv), np.abs(wv), off)
    got = y.values()
    assert (got[~live] == GUARD).all()
    tol = sum_error(n_in, size)
    assert_within(got[live], want[live], (tol + rounding(kind, np.abs(want) + tol))[live], "y")
    y.check_guards()
    check_status(D)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{sum(c[0])}-{c[2]}x{c[3]}")
def test_dgrad(kind, masked, case):
    D = load_dbl()
    lengths, _, n_in, n_out, _ = case
    g, rows, off, offsets, x_of, y_of = setup(kind, case)
    dy, dx = y_of(g.standard_normal((rows, n_out))), x_of()
    mask = x_of(np.maximum(g.standard_normal((rows, n_in)), 0)) if masked else None
    w = torch.from_numpy(g.standard_normal((len(lengths), n_out, n_in)) / n_out ** 0.5).to(DTYPE[kind]).cuda()
    if rows > off[-1]:
        dy.view()[int(off[-1]):] = float("nan")
    fmt, _ = precision(D, kind)
    shape = shape_of(D, case)
    with fmt:
        D.dbl_grouped_dgrad(shape, dy.ptr(), w, offsets, mask and mask.ptr(), dx.ptr(), *scratch(D, shape, D.DBL_PASS_DGRAD))
    torch.cuda.synchronize()
    dv, wv = np.nan_to_num(dy.values()), w.double().cpu().numpy()
    want, live = orc.grouped_dgrad(dv, wv, off, mask and mask.values())
    size, _ = orc.grouped_dgrad(np.abs(dv), np.abs(wv), off)
    got = dx.values()
    assert (got[~live] == GUARD).all()
    tol = np.where(want == 0, 0, sum_error(n_out, size)) if masked else sum_error(n_out, size)
    assert_within(got[live], want[live], (tol + rounding(kind, np.abs(want) + tol))[live], "dx")
    dx.check_guards()
    check_status(D)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{sum(c[0])}-{c[2]}x{c[3]}")
def test_wgrad(kind, accumulate, case):
    D = load_dbl()
    lengths, _, n_in, n_out, _ = case
    g, rows, off, offsets, x_of, y_of = setup(kind, case)
    x, dy = x_of(g.standard_normal((rows, n_in))), y_of(g.standard_normal((rows, n_out)))
    if rows > off[-1]:  # rows of no group: what they hold must not reach a gradient
        x.view()[int(off[-1]):] = float("nan")
        dy.view()[int(off[-1]):] = float("inf")
    start = g.standard_normal((len(lengths), n_out, n_in)).astype(np.float32)
    n = start.size
    buf = torch.full((n + 64,), 3.0, device="cuda")
    buf[:n] = torch.from_numpy(start).reshape(-1) if accumulate else float("nan")
    fmt, _ = precision(D, kind)
    shape = shape_of(D, case)
    with fmt:
        D.dbl_grouped_wgrad(shape, x.ptr(), dy.ptr(), offsets, buf, accumulate, *scratch(D, shape, D.DBL_PASS_WGRAD))
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        xv, dv = (np.where(np.isfinite(t.values()), t.values(), 0) for t in (x, dy))
    want, size = orc.grouped_wgrad(xv, dv, off), orc.grouped_wgrad(np.abs(xv), np.abs(dv), off)
    if accumulate:
        want, size = want + start, size + np.abs(start)
    got = buf[:n].reshape(start.shape).double().cpu().numpy()
    assert bool((buf[n:] == 3.0).all())
    assert_within(got, want, sum_error(np.array(lengths, float)[:, None, None], size) * (size > 0), "dw")
    check_status(D)


@pytest.mark.parametrize("which", ["fwd", "dgrad"])
def test_rows_of_other_groups_may_hold_anything(which):
    """A group's tile reads its neighbour's rows: NaN there must not reach this group's."""
    D = load_dbl()
    off = torch.tensor([0, 100, 200], dtype=torch.int32, device="cuda")
    g = rng(1)
    w = torch.from_numpy(g.standard_normal((2, 64, 64))).to(torch.bfloat16).cuda()
    a = torch.from_numpy(g.standard_normal((200, 64))).to(torch.bfloat16).cuda()
    a[100:] = float("nan")
    out = torch.empty((200, 64), dtype=torch.bfloat16, device="cuda")
    shape = D.grouped_shape(200, 2, 64, 64)
    if which == "fwd":
        D.dbl_grouped_fwd(shape, a, w, off, out, *scratch(D, shape, D.DBL_PASS_FWD))
    else:
        D.dbl_grouped_dgrad(shape, a, w, off, None, out, *scratch(D, shape, D.DBL_PASS_DGRAD))
    assert bool(out[:100].isfinite().all()) and bool(out[100:].isnan().all())


@pytest.mark.parametrize("first", [1, 15, 16, 48, 63, 64, 65, 100, 600])
def test_a_neighbours_rows_do_not_reach_a_weight_gradient(first):
    """The last rows of a group are copied together with the next group's, here NaN and infinity."""
    D = load_dbl()
    rows, n_in, n_out = first + 70, 72, 136
    g = rng(first)
    x, dy = (torch.from_numpy(g.standard_normal((rows, c))).to(torch.bfloat16).cuda() for c in (n_in, n_out))
    x[first:], dy[first:] = float("nan"), float("inf")
    off = torch.tensor([0, first, rows], dtype=torch.int32, device="cuda")
    dw = torch.empty((2, n_out, n_in), device="cuda")
    shape = D.grouped_shape(rows, 2, n_in, n_out)
    D.dbl_grouped_wgrad(shape, x, dy, off, dw, False, *scratch(D, shape, D.DBL_PASS_WGRAD))
    xv, dv = (t[:first].double().cpu().numpy() for t in (x, dy))
    size = np.abs(dv).T @ np.abs(xv)
    assert_within(dw[0].double().cpu().numpy(), dv.T @ xv, sum_error(first, size), "dw")
    assert bool(dw[1].isnan().all())
    check_status(D)


def test_relu_keeps_nan():
    D = load_dbl()
    off = torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    x = torch.ones((8, 16), dtype=torch.bfloat16, device="cuda")
    x[3] = float("nan")
    w = -torch.ones((1, 8, 16), dtype=torch.bfloat16, device="cuda")
    y = torch.empty((8, 8), dtype=torch.bfloat16, device="cuda")
    shape = D.grouped_shape(8, 1, 16, 8, relu=True)
    D.dbl_grouped_fwd(shape, x, w, off, y, *scratch(D, shape, D.DBL_PASS_FWD))
    assert bool(y[3].isnan().all()) and bool((y[[0, 1, 2, 4, 5, 6, 7]] == 0).all())


@pytest.mark.parametrize("bad", [[-5, 10, 3, 1000], [40, 30, 20, 10], [0, 2 ** 31 - 1, -2 ** 31, 64], [64, 64, 64, 64]])
def test_offsets_that_are_none(bad):
    """Taken as in order and inside the tensors: no other row is written."""
    D = load_dbl()
    rows, n_in, n_out = 64, 32, 40
    g = rng(2)
    off = torch.tensor(bad, dtype=torch.int32, device="cuda")
    x, dy = Rows("bf16", rows, n_in, values=g.standard_normal((rows, n_in))), Rows("bf16", rows, n_out, values=g.standard_normal((rows, n_out)))
    w = torch.from_numpy(g.standard_normal((3, n_out, n_in))).to(torch.bfloat16).cuda()
    y, dx = Rows("bf16", rows, n_out), Rows("bf16", rows, n_in)
    dw = torch.empty((3, n_out, n_in), device="cuda")
    shape = D.grouped_shape(rows, 3, n_in, n_out)
    D.dbl_grouped_fwd(shape, x.ptr(), w, off, y.ptr(), *scratch(D, shape, D.DBL_PASS_FWD))
    D.dbl_grouped_dgrad(shape, dy.ptr(), w, off, None, dx.ptr(), *scratch(D, shape, D.DBL_PASS_DGRAD))
    D.dbl_grouped_wgrad(shape, x.ptr(), dy.ptr(), off, dw, False, *scratch(D, shape, D.DBL_PASS_WGRAD))
    wv = w.double().cpu().numpy()
    for got, (want, live), size in ((y, orc.grouped_fwd(x.values(), wv, bad), 40.0),
                                    (dx, orc.grouped_dgrad(dy.values(), wv, bad), 60.0)):
        assert (got.values()[~live] == GUARD).all()
        assert_within(got.values()[live], want[live], 2.0 ** -8 * np.abs(want[live]) + sum_error(40, size * 10), "rows")
        got.check_guards()
    assert_within(dw.double().cpu().numpy(), orc.grouped_wgrad(x.values(), dy.values(), bad), sum_error(64, 1000.0), "dw")
    check_status(D)


def test_no_rows_and_the_same_bits_again():
    D = load_dbl()
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    shape = D.grouped_shape(0, 3, 16, 24)
    dw = torch.full((3, 24, 16), 2.0, device="cuda")
    D.dbl_grouped_fwd(shape, None, None, None, None)
    D.dbl_grouped_dgrad(shape, None, None, None, None, None)
    D.dbl_grouped_wgrad(shape, None, None, off, dw, True)
    assert bool((dw == 2.0).all())
    D.dbl_grouped_wgrad(shape, None, None, off, dw, False)
    assert bool((dw == 0.0).all())
    g = rng(3)
    x = torch.from_numpy(g.standard_normal((3000, 264))).to(torch.bfloat16).cuda()
    dy = torch.from_numpy(g.standard_normal((3000, 520))).to(torch.bfloat16).cuda()
    off = torch.tensor([0, 100, 2900, 3000], dtype=torch.int32, device="cuda")
    shape = D.grouped_shape(3000, 3, 264, 520)
    a, b = (torch.empty((3, 520, 264), device="cuda") for _ in range(2))
    for out in (a, b):
        D.dbl_grouped_wgrad(shape, x, dy, off, out, False, *scratch(D, shape, D.DBL_PASS_WGRAD))
    assert torch.equal(a, b)


def test_gradients_by_differences():
    """Slopes of the kernels' own forward pass, which is linear in x and in w.  Steps and values are small whole
    numbers, so that every product, sum and stored value is exact."""
    D = load_dbl()
    g = rng(4)
    off = torch.tensor([0, 3, 3, 10], dtype=torch.int32, device="cuda")
    whole = lambda *s: torch.from_numpy(g.integers(-2, 3, s)).to(torch.bfloat16).cuda()
    x, w, dy = whole(10, 16), whole(3, 24, 16), whole(10, 24)
    shape = D.grouped_shape(10, 3, 16, 24)
    dx, dw, y = torch.empty_like(x), torch.empty((3, 24, 16), device="cuda"), torch.empty_like(dy)
    D.dbl_grouped_dgrad(shape, dy, w, off, None, dx, *scratch(D, shape, D.DBL_PASS_DGRAD))
    D.dbl_grouped_wgrad(shape, x, dy, off, dw, False, *scratch(D, shape, D.DBL_PASS_WGRAD))

    def loss(x_, w_):
        D.dbl_grouped_fwd(shape, x_, w_, off, y, *scratch(D, shape, D.DBL_PASS_FWD))
        return float((y.double() * dy.double()).sum())
    for r, c in [(0, 0), (2, 15), (3, 8), (9, 1)]:
        d = torch.zeros_like(x)
        d[r, c] = 1
        assert loss(x + d, w) - loss(x - d, w) == 2 * float(dx[r, c])
    for e, o, i in [(0, 0, 0), (0, 23, 15), (1, 3, 3), (2, 8, 9)]:
        d = torch.zeros_like(w)
        d[e, o, i] = 1
        assert loss(x, w + d) - loss(x, w - d) == 2 * float(dw[e, o, i])


def test_rows_past_2_to_the_31_elements():
    """The last rows of tensors of more than 2^31 elements, in the last of two groups."""
    D = load_dbl()
    n_in, n_out, rows = 64, 4096, (1 << 19) + 300
    x = torch.zeros((rows, n_in), dtype=torch.bfloat16, device="cuda")
    y = torch.zeros((rows, n_out), dtype=torch.bfloat16, device="cuda")
    g = rng(5)
    x[-400:] = torch.from_numpy(g.integers(-2, 3, (400, n_in))).to(torch.bfloat16)
    w = torch.from_numpy(g.integers(-2, 3, (2, n_out, n_in))).to(torch.bfloat16).cuda()
    off = torch.tensor([0, rows - 350, rows], dtype=torch.int32, device="cuda")
    shape = D.grouped_shape(rows, 2, n_in, n_out)
    D.dbl_grouped_fwd(shape, x, w, off, y, *scratch(D, shape, D.DBL_PASS_FWD))
    want = torch.cat([x[-400:-350].float() @ w[0].float().t(), x[-350:].float() @ w[1].float().t()])
    assert torch.equal(y[-400:], want.to(torch.bfloat16)) and not bool(y[:1000].any())
    dx = torch.empty_like(x)
    y[:-10] = 0
    D.dbl_grouped_dgrad(shape, y, w, off, None, dx, *scratch(D, shape, D.DBL_PASS_DGRAD))
    assert not bool(dx[:-10].any())
    exact = y[-10:].double() @ w[1].double()
    assert bool(((dx[-10:].double() - exact).abs() <= 2.0 ** -8 * exact.abs() + 2.0 ** -10 * 4096).all())
    dw = torch.empty((2, n_out, n_in), device="cuda")
    D.dbl_grouped_wgrad(shape, x, y, off, dw, False, *scratch(D, shape, D.DBL_PASS_WGRAD))
    assert not bool(dw[0].any()) and torch.equal(dw[1].double(), y[-10:].double().t() @ x[-10:].double())
