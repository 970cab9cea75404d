"""Layer norm, forward and backward, against 64 bits.

Tolerances.  A sum of c terms is taken by at least 32 threads, each thread's terms one after another, then by trees
of at most 15 steps: with c <= 70,000 columns over 256 threads and more, or 1024 over 32, a chain has at most 290
additions, so a mean is off by at most 2^-24 * 300 of the mean size of its terms, and in all cases but the widest
by far less.  Below, K = chain length + 32 (the trees, the products and the operations after the sum)."""
import numpy as np
import pytest
import torch

from gpu_common import check_status, load_dbl
from oracle import tokens as T
from token_cases import EPS32, GUARD, Rows, assert_within, precision, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def D():
    return load_dbl()


def chain(c):
    return max(32, -(-c // 256)) + 32


def features(g, rows, c):
    x = g.standard_normal((rows, c)) * 1.3 + g.standard_normal((rows, 1))
    if rows > 2:
        x[1] = 3.0          # no variance
        x[2] = 100.0 + 0.5 * g.standard_normal(c)  # an offset far above the deviation
    return x


# rows, columns, elements to the next row beyond c (read, written), offset of every base address in elements
SHAPES = [(1, 1, 0, 0, 0), (3, 7, 0, 0, 0), (5, 8, 0, 0, 0), (33, 100, 0, 0, 0), (4, 64, 8, 16, 0), (3, 64, 3, 0, 0),
          (300, 512, 0, 0, 0), (17, 513, 0, 0, 0), (9, 512, 0, 0, 1), (5, 1000, 24, 8, 8), (700, 1024, 0, 0, 0),
          (6, 1023, 1, 1, 0), (130, 2048, 0, 0, 0), (11, 2050, 0, 0, 2), (3, 4097, 0, 0, 0), (40, 8192, 0, 0, 0),
          (2, 16384, 0, 0, 0), (2, 20000, 0, 0, 0), (2, 32768, 0, 0, 0), (2, 70001, 0, 0, 0), (3000, 24, 0, 0, 0),
          (10007, 3, 0, 0, 0), (2500, 256, 0, 0, 0), (1, 65536, 0, 0, 0), (300, 1002, 0, 0, 0), (40, 10447, 0, 0, 0),
          (37, 9001, 3, 0, 1), (400, 8208, 0, 8, 0), (90, 16000, 0, 0, 0), (45, 33333, 0, 0, 0), (40000, 5, 0, 0, 0), (9000, 64, 0, 0, 0),
          (9001, 33, 0, 2, 3), (20011, 101, 0, 0, 1), (6007, 128, 0, 0, 0), (5003, 200, 0, 8, 0), (5001, 255, 0, 0, 0),
          (5001, 250, 6, 0, 0), (1, 3, 0, 0, 1)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,c,gap_in,gap_out,offset", SHAPES)
@pytest.mark.parametrize("with_res", [False, True])
def test_forward(D, kind, rows, c, gap_in, gap_out, offset, with_res):
    g = np.random.default_rng(rows + c)
    x = Rows(kind, rows, c, c + gap_in, offset, features(g, rows, c))
    res = Rows(kind, rows, c, c + gap_in, offset, g.standard_normal((rows, c))) if with_res else None
    gamma, beta = g.uniform(0.5, 1.5, c).astype(np.float32), g.standard_normal(c).astype(np.float32)
    y, s = Rows(kind, rows, c, c + gap_out, offset), Rows(kind, rows, c, c + gap_out, offset)
    mean, inv = Rows("f32", 1, rows), Rows("f32", 1, rows)
    lib, dtype = precision(D, kind)
    with lib:
        D.dbl_layer_norm_fwd(D.ln_shape(rows, c, 1e-5, dtype, c + gap_in, c + gap_out), x.ptr(),
                             res.ptr() if res else None, torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda(),
                             s.ptr() if res else None, y.ptr(), mean.ptr(), inv.ptr())
        check_status(D)
    for t in (x, y, s, mean, inv) + ((res,) if res else ()):
        t.check_guards()
    want, wm, wi, ws = T.layer_norm_fwd(x.values(), gamma, beta, 1e-5, res.values() if res else None)
    # the mean is off by e, a deviation by e and its own rounding, the variance by its sum's rounding and twice
    # the deviations'; 1/sqrt halves a relative error
    k = chain(c) * EPS32
    e = k * np.abs(ws).mean(1) + EPS32 * np.abs(ws).max(1)
    ei = k + 2 * e * wi
    assert_within(mean.values()[0], wm, e, "mean")
    assert_within(inv.values()[0], wi, wi * ei, "invstd")
    h = (ws - wm[:, None]) * wi[:, None]
    tol = np.abs(gamma) * (2 * e * wi)[:, None] + np.abs(h * gamma) * (ei + 4 * EPS32)[:, None] + 2 * EPS32 * np.abs(beta)
    assert_within(y.values(), want, tol + rounding(kind, np.abs(want) + tol), "y")
    if res:
        assert_within(s.values(), ws, rounding(kind, ws) + EPS32 * np.abs(ws), "sum")


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,c,gap_in,gap_out,offset", SHAPES)
@pytest.mark.parametrize("with_skip", [False, True])
def test_backward(D, kind, rows, c, gap_in, gap_out, offset, with_skip):
    g = np.random.default_rng(rows + c + 1)
    x = Rows(kind, rows, c, c + gap_in, offset, features(g, rows, c))
    dy = Rows(kind, rows, c, c + gap_in, offset, g.standard_normal((rows, c)) + 0.2)
    skip = Rows(kind, rows, c, c + gap_in, offset, g.standard_normal((rows, c))) if with_skip else None
    gamma = g.uniform(0.5, 1.5, c).astype(np.float32)
    _, mean, inv, _ = T.layer_norm_fwd(x.values())
    mean, inv = mean.astype(np.float32), inv.astype(np.float32)
    dx = Rows(kind, rows, c, c + gap_out, offset)
    dg, db = Rows("f32", 1, c), Rows("f32", 1, c)
    lib, dtype = precision(D, kind)
    shape = D.ln_shape(rows, c, 1e-5, dtype, c + gap_in, c + gap_out)
    tm, ti, tg = (torch.from_numpy(a).cuda() for a in (mean, inv, gamma))
    with lib:
        need = D.dbl_layer_norm_workspace_bytes(shape)
        ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
        D.dbl_layer_norm_bwd(shape, dy.ptr(), skip.ptr() if skip else None, x.ptr(), tg, tm, ti, dx.ptr(), dg.ptr(),
                             db.ptr(), ws, need)
        check_status(D)
        assert bool((ws[need:] == 255).all())
        first = [t.buf.clone() for t in (dx, dg, db)]
        D.dbl_layer_norm_bwd(shape, dy.ptr(), skip.ptr() if skip else None, x.ptr(), tg, tm, ti, dx.ptr(), dg.ptr(),
                             db.ptr(), ws, need)
        assert all(torch.equal(a.view(torch.uint8), t.buf.view(torch.uint8)) for a, t in zip(first, (dx, dg, db)))
    for t in (x, dy, dx, dg, db):
        t.check_guards()
    X, DY = x.values(), dy.values()
    wx, wg, wb = T.layer_norm_bwd(DY, X, gamma, mean, inv, skip.values() if skip else None)
    h = (X - mean[:, None].astype(np.float64)) * inv[:, None].astype(np.float64)
    # xhat is rounded after the subtraction and after the product
    eh = 2 * EPS32 * np.abs(h)
    gg = np.abs(DY * gamma)
    k = chain(c) * EPS32
    tol = inv[:, None] * (4 * EPS32 * gg + k * gg.mean(1, keepdims=True)
                          + (4 * EPS32 + k) * np.abs(h) * (gg * np.abs(h)).mean(1, keepdims=True)) + 2 * EPS32 * np.abs(wx)
    if skip:
        tol = tol + EPS32 * np.abs(skip.values())
    assert_within(dx.values(), wx, tol + rounding(kind, np.abs(wx) + tol), "dx")
    # a block of rows adds at most rows/16 of them one after another (64 at least), the blocks' sums are then
    # added one after another: at most 400
    chain_r = max(64, rows / 16) + 400
    assert_within(dg.values()[0], wg, (np.abs(DY) * (chain_r * EPS32 * np.abs(h) + eh)).sum(0), "dgamma")
    assert_within(db.values()[0], wb, chain_r * EPS32 * np.abs(DY).sum(0), "dbeta")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_optional_arguments(D, kind):
    rows, c = 21, 96
    g = np.random.default_rng(5)
    x, dy = Rows(kind, rows, c, values=g.standard_normal((rows, c))), Rows(kind, rows, c, values=g.standard_normal((rows, c)))
    lib, dtype = precision(D, kind)
    shape = D.ln_shape(rows, c, 1e-3, dtype)
    y = Rows(kind, rows, c)
    with lib:
        D.dbl_layer_norm_fwd(shape, x.ptr(), None, None, None, None, y.ptr(), None, None)
        want, mean, inv, _ = T.layer_norm_fwd(x.values(), None, None, 1e-3)
        assert_within(y.values(), want, rounding(kind, want) + 200 * EPS32 * (1 + np.abs(want)), "y")
        tm, ti = (torch.from_numpy(a.astype(np.float32)).cuda() for a in (mean, inv))
        dx = Rows(kind, rows, c)
        D.dbl_layer_norm_bwd(shape, dy.ptr(), None, x.ptr(), None, tm, ti, dx.ptr(), None, None, None, 0)
        wx, _, _ = T.layer_norm_bwd(dy.values(), x.values(), None, mean, inv)
        assert_within(dx.values(), wx, rounding(kind, wx) + 400 * EPS32 * inv.max() * np.abs(dy.values()).max(), "dx")
        # no rows: the parameters' gradients are empty sums
        none = D.ln_shape(0, c, 1e-3, dtype)
        dg, db = Rows("f32", 1, c), Rows("f32", 1, c)
        need = D.dbl_layer_norm_workspace_bytes(none)
        ws = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
        D.dbl_layer_norm_fwd(none, x.ptr(), None, None, None, None, y.ptr(), None, None)
        D.dbl_layer_norm_bwd(none, dy.ptr(), None, x.ptr(), None, tm, ti, dx.ptr(), dg.ptr(), db.ptr(), ws, need)
        check_status(D)
        assert (dg.values() == 0).all() and (db.values() == 0).all()


def test_a_row_with_nan_or_infinity_stays_by_itself(D):
    rows, c = 40, 640
    g = np.random.default_rng(6)
    v = g.standard_normal((rows, c))
    clean = v.copy()
    v[7, 3], v[11, 600] = np.nan, np.inf
    outs = []
    for vals in (clean, v):
        x, y = Rows("bf16", rows, c, values=vals), Rows("bf16", rows, c)
        D.dbl_layer_norm_fwd(D.ln_shape(rows, c), x.ptr(), None, None, None, None, y.ptr(), None, None)
        outs.append(y.values())
    keep = [r for r in range(rows) if r not in (7, 11)]
    assert (outs[0][keep] == outs[1][keep]).all()
    assert np.isnan(outs[1][7]).all() and np.isnan(outs[1][11]).all()


def test_on_another_stream_and_in_a_graph(D):
    rows, c = 64, 768
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(rows, c, device="cuda", generator=gen).to(torch.bfloat16)
    dy = torch.randn(rows, c, device="cuda", generator=gen).to(torch.bfloat16)
    shape = D.ln_shape(rows, c)
    need = D.dbl_layer_norm_workspace_bytes(shape)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def buffers():
        bf, f = dict(dtype=torch.bfloat16, device="cuda"), dict(device="cuda")
        return [torch.zeros(rows, c, **bf), torch.zeros(rows, **f), torch.zeros(rows, **f), torch.zeros(rows, c, **bf),
                torch.zeros(c, **f), torch.zeros(c, **f)]

    def run(o, stream=None):
        D.dbl_layer_norm_fwd(shape, x, None, None, None, None, o[0], o[1], o[2], stream)
        D.dbl_layer_norm_bwd(shape, dy, None, x, None, o[1], o[2], o[3], o[4], o[5], ws, need, stream)

    want, side, graphed = buffers(), buffers(), buffers()
    run(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    run(side, s)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(graphed)
    graph.replay()
    torch.cuda.synchronize()
    for a, b, d in zip(want, side, graphed):
        assert torch.equal(a, b) and torch.equal(a, d)


@pytest.mark.parametrize("rows,c", [(6, 65), (3, 700)])
def test_gradient_is_the_slope_of_the_forward_pass(D, rows, c):
    """Central differences of the kernel's own forward pass, along a direction in x, gamma and beta, in fp32: a step of
    2^-7 leaves an error of its square times the third derivatives, below 16 of the terms for rows whose deviation and
    direction are about 1, so 1e-3 of them at most; and y's rounding (64 roundings of values up to |y|) over the step."""
    g = np.random.default_rng(rows * c)
    x, dy, vx = g.standard_normal((rows, c)) + 0.5, g.standard_normal((rows, c)), g.standard_normal((rows, c))
    gamma, beta, vg, vb = g.uniform(0.5, 1.5, c), g.standard_normal(c), g.standard_normal(c), g.standard_normal(c)
    step = 2.0 ** -7
    shape = D.ln_shape(rows, c, 1e-5, D.DBL_F32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()

    def forward(s):
        y, mean, inv = torch.empty(rows, c, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        tx = dev(x + s * vx)
        D.dbl_layer_norm_fwd(shape, tx, None, dev(gamma + s * vg), dev(beta + s * vb), None, y, mean, inv)
        torch.cuda.synchronize()
        return y.double().cpu().numpy(), tx, mean, inv

    up, down = forward(step)[0], forward(-step)[0]
    slope = float(((up - down) / (2 * step) * dy.astype(np.float32)).sum())
    y, tx, mean, inv = forward(0.0)
    dx, dg, db = torch.empty(rows, c, device="cuda"), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    need = D.dbl_layer_norm_workspace_bytes(shape)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    D.dbl_layer_norm_bwd(shape, dev(dy), None, tx, dev(gamma), mean, inv, dx, dg, db, ws, need)
    check_status(D)
    parts = [a.double().cpu().numpy() * v for a, v in ((dx, vx), (dg, vg), (db, vb))]
    bound = 1e-3 * sum(np.abs(a).sum() for a in parts) + 64 * EPS32 * np.abs(y * dy).sum() / step
    assert abs(sum(a.sum() for a in parts) - slope) <= bound, (sum(a.sum() for a in parts), slope, bound)
