"""The distillation loss and its gradient against 64 bits.

Tolerances.  A sum of exponentials over v classes is taken by at least 128 threads, one term after another in each,
then by trees: relative error (v/128 + 64)*2^-24 at the most, positive terms throughout.  An exponential carries the
rounding of its argument, 3*2^-24 times its size."""
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


def problem(kind, rows, v, k, seed=0):
    g = np.random.default_rng(seed + rows + v + k)
    z = 2 * g.standard_normal((rows, v))
    top = (1.5 * g.standard_normal((rows, k)) + 4).astype(np.float32)
    cls = np.stack([g.choice(v, k, replace=k > v) for _ in range(rows)]).astype(np.int32).reshape(rows, k)
    labels = g.integers(0, v, rows).astype(np.int32)
    return z, top, cls, labels


def call(D, kind, z, top, cls, labels, weight, tau, alpha, scale=None, gap=0, gap_grad=0, offset=0, grad="apart",
         want_loss=True):
    rows, v = z.shape
    k = cls.shape[1]
    zr = Rows(kind, rows, v, v + gap, offset, z)
    seen = zr.values()
    dz = zr if grad == "in place" else Rows(kind, rows, v, v + gap_grad, offset)
    row_loss, loss = Rows("f32", 1, rows), Rows("f32", 1, 1)
    dev = lambda a, t: None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=t)).cuda()
    ttop, tcls = (dev(top, np.float32), dev(cls, np.int32)) if k else (None, None)
    tlab, tw = dev(labels, np.int32), dev(weight, np.float32)
    ts = None if scale is None else torch.tensor([scale], device="cuda")
    lib, dtype = precision(D, kind)
    with lib:
        shape = D.distill_shape(rows, v, k, tau, alpha, dtype, v + gap, v + (gap if grad == "in place" else gap_grad))
        D.dbl_distill_fwd_bwd(shape, zr.ptr(), ttop, tcls, tlab, tw, ts, row_loss.ptr(),
                              loss.ptr() if want_loss else None, None if grad is None else dz.ptr())
        check_status(D)
    for r in (zr, dz, row_loss, loss):
        r.check_guards()
    if grad != "in place":
        assert np.array_equal(zr.values(), seen, equal_nan=True)
    return seen, row_loss.values()[0], loss.values()[0, 0], dz.values()


def check(kind, seen, got, top, cls, labels, weight, tau, alpha, scale=1.0, grad=True):
    tau, alpha = float(np.float32(tau)), float(np.float32(alpha))
    _, row, loss, dz = got
    rows, v = seen.shape
    wr, wl, wz, size = T.distill(seen, top, cls, labels, weight, tau, alpha, scale)
    w = np.full(rows, 1.0 / rows) if weight is None else np.asarray(weight, np.float64)
    k = (v / 128 + 64) * EPS32
    span = np.zeros(rows)  # the largest |z - max| over what counts, and the teacher's
    for r in range(rows):
        fin = seen[r][np.isfinite(seen[r])]
        span[r] = (fin.max() - fin.min() if fin.size else 0) + np.log(v)
    ft = [top[r][np.isfinite(top[r])] for r in range(rows)] if cls.shape[1] else [np.zeros(0)] * rows
    span_t = np.array([a.max() - a.min() if a.size else 0 for a in ft]) + np.log(cls.shape[1] + 1.0)
    one = 1 + span + span_t  # no logarithm here is larger
    tol = (alpha * tau * (tau + one) + (1 - alpha) * one) * (k + 8 * EPS32) + 4 * EPS32 * one * alpha * tau * one
    assert_within(row, wr, tol, "row_loss")
    if loss != GUARD:
        assert_within(loss, wl, (np.abs(w) * tol).sum() + (rows / 1024 + 32) * EPS32 * np.abs(w * wr).sum(), "loss")
    if grad:
        e = size * (2 * k + 6 * EPS32 * (one[:, None] * max(1.0, 1.0 / tau) + 4))
        # exponentials below the smallest normal fp32 number may be taken as 0
        e = e + (np.abs(w) * scale * (alpha * tau + 1))[:, None] * 2.0 ** -125 * (size > 0)
        assert_within(dz, wz, e + rounding(kind, np.abs(wz) + e) * (w != 0)[:, None], "dlogits")


SIZES = [(1, 1, 1), (3, 7, 2), (5, 10, 10), (64, 100, 5), (300, 100, 16), (33, 1000, 16), (9, 1003, 7), (4, 2048, 64),
         (7, 5000, 33), (3, 8192, 128), (2, 20001, 1), (2, 32000, 32), (3, 50008, 20), (2, 65537, 16), (1, 131071, 64),
         (1, 260000, 8), (1, 700001, 4), (1, 2000003, 3),
         # many rows: a warp or few warps each, and parts of which two are held by an SM
         (650, 701, 5), (700, 3000, 16), (620, 6001, 130), (700, 8001, 20), (310, 17000, 70), (240, 45001, 9)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,v,k", SIZES)
@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.6)])
def test_loss_and_gradient(D, kind, rows, v, k, tau, alpha):
    z, top, cls, labels = problem(kind, rows, v, k)
    scale = 1024.0 if kind == "f16" else None
    got = call(D, kind, z, top, cls, labels, None, tau, alpha, scale)
    check(kind, got[0], got, top, cls, labels, None, tau, alpha, scale or 1.0)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,v,gap,gap_grad,offset,grad", [
    (6, 1000, 24, 24, 0, "apart"), (6, 1000, 24, 0, 0, "apart"), (5, 1001, 23, 23, 0, "apart"), (5, 999, 0, 2, 3, "apart"),
    (4, 1000, 0, 0, 1, "apart"), (6, 1000, 0, 0, 0, "in place"), (5, 1003, 5, 5, 1, "in place"),
    (2, 40000, 0, 0, 0, "in place"), (2, 120001, 7, 7, 5, "in place"), (1, 1500007, 0, 0, 0, "in place"),
    (3, 33, 1, 1, 0, "in place"), (3, 16384, 8, 8, 8, "apart"), (6, 1000, 0, 0, 0, None), (2, 90001, 0, 0, 0, None),
])
def test_strides_alignment_and_place(D, kind, rows, v, gap, gap_grad, offset, grad):
    z, top, cls, labels = problem(kind, rows, v, 9, 1)
    got = call(D, kind, z, top, cls, labels, None, 1.5, 0.5, 512.0, gap, gap_grad, offset, grad)
    check(kind, got[0], got, top, cls, labels, None, 1.5, 0.5, 512.0, grad is not None)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("v", [50, 1000, 40001])
def test_absent_entries_labels_and_weights(D, kind, v):
    """Rows: 0 plain; 1 no label; 2 no entries; 3 neither; 4 entries out of range; 5 a class named three times, the
    label among them; 6 weight 0 over NaN; 7 entries of weight 0 (minus infinity); 8 masked student classes; 9 every
    student logit at the type's lowest value; 10 all of one row masked but two classes; 11 a teacher's class masked
    for the student: an infinite loss, a finite gradient."""
    rows, k = 12, 6
    z, top, cls, labels = problem(kind, rows, v, k, 2)
    labels[1] = -1
    cls[2] = -1
    cls[3], labels[3] = v, v
    cls[4, 1::2] = [-5, v, 2 ** 31 - 1]
    cls[5, :3], labels[5] = 7, 7
    w = np.linspace(0.5, 1.5, rows).astype(np.float32)
    w[6] = 0.0
    z[6] = np.nan
    top[7, 2:] = -np.inf
    z[8, [i for i in range(v) if i % 3 == 0 and i not in cls[8] and i != labels[8]]] = -np.inf
    z[9] = {"bf16": -3.3895313892515355e38, "f32": -3.4028234663852886e38}[kind]
    z[10] = -np.inf
    z[10, [3, 11]] = [1.0, -2.0]
    cls[10] = [3, 11, -1, -1, -1, -1]
    labels[10] = 11
    z[11, cls[11, 0]] = -np.inf
    labels[11] = (cls[11, 0] + 1) % v
    got = call(D, kind, z, top, cls, labels, w, 2.0, 0.5)
    seen = got[0].copy()
    assert got[1][11] == np.inf and got[2] == np.inf and np.isfinite(got[3][11]).all()
    assert got[1][3] == 0 and (got[3][3] == 0).all() and got[1][6] == 0 and (got[3][6] == 0).all()
    with np.errstate(divide="ignore", invalid="ignore"):
        check(kind, seen, (seen, got[1], GUARD, got[3]), top, cls, labels, w, 2.0, 0.5)


def test_rows_without_a_distribution_are_nan_alone(D):
    rows, v, k = 8, 1000, 4
    for v in (1000, 70001):
        z, top, cls, labels = problem("f32", rows, v, k, 3)
        z[1] = -np.inf
        z[3, 17] = np.nan
        z[5, v - 1] = np.inf
        _, row, loss, dz = call(D, "f32", z, top, cls, None, None, 1.0, 1.0)
        assert np.isnan(row[[1, 3, 5]]).all() and np.isnan(dz[[1, 3]]).all() and np.isnan(loss)
        rest = [0, 2, 4, 6, 7]
        assert np.isfinite(row[rest]).all() and np.isfinite(dz[rest]).all()


@pytest.mark.parametrize("kind,v", [("bf16", 300), ("f32", 5000), ("f16", 131071)])
def test_labels_alone_and_large_k(D, kind, v):
    rows = 5
    z, top, cls, labels = problem(kind, rows, v, 3)
    none = np.zeros((rows, 0))
    got = call(D, kind, z, none, none, labels, None, 1.0, 0.0, 256.0)
    check(kind, got[0], got, none, none, labels, None, 1.0, 0.0, 256.0)
    got = call(D, kind, z, top, cls, labels, None, 1.0, 0.0, 256.0)  # alpha 0: the teacher does not count
    check(kind, got[0], got, none, none, labels, None, 1.0, 0.0, 256.0)
    k = D.DBL_DISTILL_MAX_K  # with v = 300 every class is named several times
    z, top, cls, labels = problem(kind, rows, v, k, 4)
    got = call(D, kind, z, top, cls, labels, None, 3.0, 0.25, 256.0, want_loss=False)
    assert got[2] == GUARD
    check(kind, got[0], got, top, cls, labels, None, 3.0, 0.25, 256.0)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("v", [40, 6000, 20001, 131071])
def test_classes_named_again_among_many(D, kind, v):
    """A hundred entries of 37 classes and absent ones; labels among them, beside them and not given."""
    rows, k = 5, 100
    z, top, cls, labels = problem(kind, rows, v, k, 6)
    g = np.random.default_rng(v)
    few = g.choice(v, 37, replace=False)
    cls = few[g.integers(0, 37, (rows, k))].astype(np.int32)
    cls[g.random((rows, k)) < 0.1] = -1
    labels[0], labels[1] = few[0], next(c for c in range(v) if c not in few)
    cls[0, 50:53] = few[0]
    cls[2, 1:] = -1
    labels[3] = -1
    got = call(D, kind, z, top, cls, labels, None, 2.0, 0.4, 64.0)
    check(kind, got[0], got, top, cls, labels, None, 2.0, 0.4, 64.0)


def test_the_same_bits_again_on_another_stream_and_in_a_graph(D):
    rows, v, k = 50, 3001, 20
    gen = torch.Generator(device="cuda").manual_seed(0)
    z = torch.randn(rows, v, device="cuda", generator=gen).to(torch.bfloat16)
    top = torch.randn(rows, k, device="cuda", generator=gen)
    cls = torch.randint(0, 40, (rows, k), device="cuda", dtype=torch.int32, generator=gen)  # many named twice
    shape = D.distill_shape(rows, v, k, 2.0, 1.0)

    def run(o, stream=None):
        D.dbl_distill_fwd_bwd(shape, z, top, cls, None, None, None, o[0], o[1], o[2], stream)

    bufs = [[torch.zeros(rows, device="cuda"), torch.zeros(1, device="cuda"),
             torch.zeros(rows, v, dtype=torch.bfloat16, device="cuda")] for _ in range(4)]
    run(bufs[0])
    run(bufs[1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    run(bufs[2], s)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(bufs[3])
    graph.replay()
    torch.cuda.synchronize()
    for o in bufs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(bufs[0], o))


def test_no_rows(D):
    loss = torch.ones(1, device="cuda")
    D.dbl_distill_fwd_bwd(D.distill_shape(0, 10, 2), 16, 16, 16, None, None, None, 16, loss, None)
    assert float(loss) == 0.0


def test_gradient_is_the_slope_of_the_loss(D):
    """Central differences of the call's own loss along a direction in the logits: a step of 2^-6 leaves an error of its
    square times the third derivatives, 1e-3 of the terms at most for directions of a few units, and the loss's
    rounding (at most 100 roundings of values up to 1 + the largest |log q|, 12 here) over the step."""
    rows, v, k, tau, alpha = 5, 130, 9, 1.5, 0.6
    z, top, cls, labels = problem("f32", rows, v, k, 2)
    direction = np.random.default_rng(8).standard_normal((rows, v))
    step = 2.0 ** -6
    z = z.astype(np.float32).astype(np.float64)
    ends = [call(D, "f32", z + s * direction, top, cls, labels, None, tau, alpha)[2] for s in (step, -step)]
    slope = (float(ends[0]) - float(ends[1])) / (2 * step)
    terms = call(D, "f32", z, top, cls, labels, None, tau, alpha)[3] * direction
    bound = 1e-3 * np.abs(terms).sum() + 100 * EPS32 * 13 * (alpha * tau * tau + 1 - alpha) / step
    assert abs(terms.sum() - slope) <= bound, (terms.sum(), slope, bound)
