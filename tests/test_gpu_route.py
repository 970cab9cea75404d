"""The router against the 64-bit form: experts, places and bounds exactly, weights and gradients within fp32 roundings."""
import numpy as np
import pytest
import torch

from gpu_common import check_status, load_dbl, rng, ws
from oracle import experts as orc
from token_cases import EPS32, Rows, assert_within, precision, rounding

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def run(D, kind, z, k, normalise, bias=None, row_weight=None):
    """z: Rows of logits."""
    dev = lambda a: None if a is None else torch.from_numpy(np.asarray(a, np.float32)).cuda()
    rows = z.rows
    chosen, slots = (torch.full((rows, k), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    weights = torch.full((rows, k), 7.0, device="cuda")
    offsets = torch.full((z.c + 2,), -7, dtype=torch.int32, device="cuda")
    fmt, dtype = precision(D, kind)
    with fmt:
        shape = D.route_shape(rows, z.c, k, normalise, dtype, ld=z.ld)
        need = D.dbl_route_workspace_bytes(shape)
        scratch = torch.full((need + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        D.dbl_route_fwd(shape, z.ptr(), dev(bias), dev(row_weight), chosen, weights, slots, offsets, scratch, need)
    torch.cuda.synchronize()
    assert int(offsets[-1]) == -7 and bool((scratch[need:] == 0x5A).all())
    return chosen.cpu().numpy(), weights.double().cpu().numpy(), slots.cpu().numpy(), offsets.cpu().numpy()[:-1]


def weight_error(z, chosen, want, normalise):
    """The exponential is off by 2 ulp and by its argument's rounding, the sum by an addition for each term, then one
    division: of the weight's own size, above the smallest numbers."""
    with np.errstate(invalid="ignore"):
        live = np.where(np.isfinite(z), z, 0.0)
        spread = np.ptp(live, axis=1, keepdims=True)
    return want * EPS32 * (12 + 3 * spread + z.shape[1]) + 2.0 ** -146


CASES = [  # rows, experts, k, stride, offset
    (1, 1, 1, 0, 0), (1, 8, 2, 0, 0), (5, 3, 3, 0, 0), (64, 8, 2, 0, 0), (130, 60, 4, 0, 0), (33, 64, 8, 72, 1),
    (1000, 128, 8, 0, 0), (257, 33, 32, 0, 0), (70, 1024, 6, 0, 0), (4099, 16, 1, 0, 0), (12, 257, 32, 264, 3),
    (9000, 7, 2, 0, 0), (3, 500, 1, 0, 0), (600, 256, 8, 0, 0), (301, 160, 12, 0, 0), (20000, 32, 4, 0, 0),
    (2500, 512, 3, 0, 0), (777, 100, 9, 0, 0),
    # many rows, a thread to each: all of k, widths that end inside 16 and 64, rows of several tiles, a stride
    (21000, 100, 8, 0, 0), (30001, 17, 16, 0, 0), (20004, 512, 12, 0, 0), (24001, 65, 1, 72, 3), (19500, 130, 5, 136, 0)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("normalise", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_route(kind, normalise, case):
    D = load_dbl()
    rows, experts, k, ld, offset = case
    g = rng(rows * 7 + experts)
    v = g.standard_normal((rows, experts)) * 2
    v[g.random(v.shape) < 0.05] = -INF
    if rows > 4:
        v[2] = -INF
        v[4, 0] = NAN
    if rows > 40:
        v[33] = np.round(v[33])  # equals
        v[34] = 1.0
        v[35, experts // 2] = INF
    bias = g.standard_normal(experts) * 0.3 if rows % 2 == 0 else None
    weight = np.where(g.random(rows) < 0.15, 0.0, 0.25) if rows % 3 == 0 else None
    z = Rows(kind, rows, experts, ld, offset, v)
    got = run(D, kind, z, k, normalise, bias, weight)
    want = orc.route(z.values(), k, normalise, bias, weight)
    for a, b, what in zip(got, want, ("chosen", "weights", "slots", "offsets")):
        if what != "weights":
            assert (a == b).all(), what
    assert_within(got[1], want[1], weight_error(z.values(), want[0], np.nan_to_num(want[1]), normalise), "weights")
    z.check_guards()
    check_status(D)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 900, 20000])
def test_all_experts_equal_and_signed_zeros(kind, rows):
    D = load_dbl()
    v = np.zeros((rows, 70))
    v[:, ::3] = -0.0
    chosen, weights, slots, offsets = run(D, kind, Rows(kind, rows, 70, values=v), 5, True)
    assert (chosen == np.arange(5)).all() and np.allclose(weights, 0.2, rtol=4 * EPS32, atol=0)
    assert offsets.tolist() == [min(e, 5) * rows for e in range(71)]
    assert (slots == np.arange(5) * rows + np.arange(rows)[:, None]).all()


@pytest.mark.parametrize("rows,experts", [(100, 12), (20000, 40)])
def test_bias_of_infinity_closes_an_expert_and_padding_may_hold_anything(rows, experts):
    D = load_dbl()
    g = rng(4)
    k = 4
    v = g.standard_normal((rows, experts)).astype(np.float32)
    v[::5] = NAN
    bias, weight = np.zeros(experts), np.ones(rows)
    bias[[3, 7]] = -INF
    bias[5], bias[6] = 100, NAN
    weight[::5] = 0
    z = Rows("f32", rows, experts, values=v)
    got, want = run(D, "f32", z, k, False, bias, weight), orc.route(z.values(), k, False, bias, weight)
    for i in (0, 2, 3):
        assert (got[i] == want[i]).all()
    assert not np.isin(got[0], [3, 6, 7]).any() and (got[0][1::5, 0] == 5).all() and (got[1][::5] == 0).all()
    # fewer left than are asked for
    bias[:] = -INF
    bias[2] = 0
    got = run(D, "f32", z, k, True, bias, weight)
    assert (got[0][1] == [2, -1, -1, -1]).all() and got[1][1].tolist() == [1, 0, 0, 0] and got[3][-1] == rows * 4 // 5


def test_the_same_bits_again_and_no_rows():
    D = load_dbl()
    z = Rows("bf16", 5000, 96, values=rng(1).standard_normal((5000, 96)))
    a, b = run(D, "bf16", z, 6, False), run(D, "bf16", z, 6, False)
    assert all((x == y).all() for x, y in zip(a, b))
    offsets = torch.full((9,), 5, dtype=torch.int32, device="cuda")
    D.dbl_route_fwd(D.route_shape(0, 8, 2), None, None, None, None, None, None, offsets, None, 0)
    assert offsets.cpu().tolist() == [0] * 9


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("normalise", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_route_bwd(kind, normalise, case):
    D = load_dbl()
    rows, experts, k, ld, offset = case
    g = rng(rows * 5 + experts)
    v = g.standard_normal((rows, experts)) * 2
    v[g.random(v.shape) < 0.05] = -INF
    if rows > 4:
        v[2], v[4, 0] = -INF, NAN
    z, dz = Rows(kind, rows, experts, ld, offset, v), Rows(kind, rows, experts, ld, offset)
    weight = np.where(g.random(rows) < 0.15, 0.0, 0.25) if rows % 3 == 0 else None
    chosen, weights, _, _ = run(D, kind, z, k, normalise, None, weight)
    dw = g.standard_normal((rows, k)).astype(np.float32)
    dw[chosen < 0] = NAN  # of absent entries: not used
    fmt, dtype = precision(D, kind)
    with fmt:
        D.dbl_route_bwd(D.route_shape(rows, experts, k, normalise, dtype, ld, ld), None if normalise else z.ptr(),
                        *(torch.from_numpy(a).cuda() for a in (chosen, weights.astype(np.float32), dw)), dz.ptr())
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        want, size = orc.route_bwd(z.values(), chosen, weights, np.nan_to_num(dw), normalise)
    # each term: the softmax's error as above, products and a sum over the entries
    tol = size * EPS32 * (16 + 2 * k + (0 if normalise else 3 * 20 + experts)) + 2.0 ** -146
    assert_within(dz.values(), want, tol + rounding(kind, np.nan_to_num(np.abs(want)) + tol), "dlogits")
    dz.check_guards()
    check_status(D)


def test_an_expert_named_twice():
    D = load_dbl()
    z = Rows("f32", 1, 6, values=rng(0).standard_normal((1, 6)))
    chosen, w, dw = np.array([[4, 4, 1]]), np.array([[.25, .5, .125]], np.float32), np.array([[1., 2., 3.]], np.float32)
    for normalise in (False, True):
        dz = Rows("f32", 1, 6)
        D.dbl_route_bwd(D.route_shape(1, 6, 3, normalise, D.DBL_F32), z.ptr(), torch.from_numpy(chosen.astype(np.int32)).cuda(),
                        torch.from_numpy(w).cuda(), torch.from_numpy(dw).cuda(), dz.ptr())
        want, size = orc.route_bwd(z.values(), chosen, w, dw, normalise)
        assert_within(dz.values(), want, size * EPS32 * 60, "dlogits")


@pytest.mark.parametrize("normalise", [False, True])
def test_gradient_by_differences(normalise):
    """Slopes of the kernel's own weights, in fp32 with steps of 2^-6 that change no choice."""
    D = load_dbl()
    g = rng(6)
    rows, experts, k = 4, 10, 3
    v = np.round(g.permutation(40).reshape(rows, experts) / 8.0, 3).astype(np.float32)  # apart by 1/8 within a row
    z = Rows("f32", rows, experts, values=v)
    chosen, w, _, _ = run(D, "f32", z, k, normalise)
    dw = g.standard_normal((rows, k)).astype(np.float32)
    dz = Rows("f32", rows, experts)
    D.dbl_route_bwd(D.route_shape(rows, experts, k, normalise, D.DBL_F32), z.ptr(), torch.from_numpy(chosen).cuda(),
                    torch.from_numpy(w.astype(np.float32)).cuda(), torch.from_numpy(dw).cuda(), dz.ptr())
    got, h = dz.values(), 2.0 ** -6
    for r in range(rows):
        for e in range(experts):
            ends = []
            for sign in (1, -1):
                u = v.copy()
                u[r, e] += sign * h
                c, wt, _, _ = run(D, "f32", Rows("f32", rows, experts, values=u), k, normalise)
                assert (c == chosen).all()
                ends.append((wt * dw).sum())
            # h^2/6 of a third derivative below 6 times the largest |dw|, and the weights' errors over 2h
            tol = h * h * np.abs(dw).max() + k * np.abs(dw).max() * 40 * EPS32 / h
            assert abs((ends[0] - ends[1]) / (2 * h) - got[r, e]) < tol


def test_strides_that_pass_2_to_the_31():
    D = load_dbl()
    rows, experts, k, ld = 5, 16, 2, (1 << 29) + 8
    buf = torch.zeros((rows - 1) * ld + experts, dtype=torch.bfloat16, device="cuda")
    v = torch.from_numpy(rng(2).standard_normal((rows, experts))).to(torch.bfloat16)
    buf.as_strided((rows, experts), (ld, 1)).copy_(v)
    out = [torch.empty((rows, k), dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.int32)]
    offsets = torch.empty(experts + 1, dtype=torch.int32, device="cuda")
    shape = D.route_shape(rows, experts, k, False, ld=ld, ld_grad=ld)
    need = D.dbl_route_workspace_bytes(shape)
    D.dbl_route_fwd(shape, buf, None, None, *out, offsets, ws(need), need)
    want = orc.route(v.double().numpy(), k, False)
    assert (out[0].cpu().numpy() == want[0]).all() and (out[2].cpu().numpy() == want[2]).all()
    grad = torch.zeros_like(buf)
    D.dbl_route_bwd(shape, buf, out[0], out[1], torch.ones((rows, k), device="cuda"), grad)
    dz, _ = orc.route_bwd(v.double().numpy(), want[0], want[1], np.ones((rows, k)), False)
    got = grad.as_strided((rows, experts), (ld, 1)).double().cpu().numpy()
    assert_within(got, dz, 2.0 ** -8 * np.abs(dz) + 60 * EPS32, "dlogits")
