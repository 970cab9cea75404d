"""The 64-bit forms of the token operators against library routines, automatic differentiation and central
differences (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import tokens as T


def central(f, x, eps=1e-6):
    """Central differences of the scalar f along every element of x."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        keep = x[i]
        x[i] = keep + eps
        up = f()
        x[i] = keep - eps
        g[i] = (up - f()) / (2 * eps)
        x[i] = keep
    return g


@pytest.mark.parametrize("rows,c", [(1, 1), (3, 2), (7, 13), (5, 64)])
def test_layer_norm_is_the_librarys(rows, c):
    g = np.random.default_rng(rows * c)
    x, res, dy, skip = (g.standard_normal((rows, c)) for _ in range(4))
    gamma, beta = g.uniform(0.5, 1.5, c), g.standard_normal(c)
    tx = torch.from_numpy(x + res).requires_grad_(True)
    tg, tb = torch.from_numpy(gamma).requires_grad_(True), torch.from_numpy(beta).requires_grad_(True)
    want = torch.nn.functional.layer_norm(tx, (c,), tg, tb, 1e-5)
    want.backward(torch.from_numpy(dy))
    y, mean, invstd, s = T.layer_norm_fwd(x, gamma, beta, 1e-5, res)
    np.testing.assert_allclose(y, want.detach().numpy(), rtol=1e-10, atol=1e-11)
    dx, dg, db = T.layer_norm_bwd(dy, s, gamma, mean, invstd, skip)
    np.testing.assert_allclose(dx, tx.grad.numpy() + skip, rtol=1e-8, atol=1e-10)
    np.testing.assert_allclose(dg, tg.grad.numpy(), rtol=1e-9, atol=1e-11)
    np.testing.assert_allclose(db, tb.grad.numpy(), rtol=1e-9, atol=1e-11)


def test_layer_norm_gradient_by_differences():
    g = np.random.default_rng(3)
    x, dy, gamma, beta = g.standard_normal((3, 5)), g.standard_normal((3, 5)), g.uniform(0.5, 1.5, 5), g.standard_normal(5)
    f = lambda: float((T.layer_norm_fwd(x, gamma, beta)[0] * dy).sum())
    _, mean, invstd, s = T.layer_norm_fwd(x, gamma, beta)
    dx, dg, db = T.layer_norm_bwd(dy, s, gamma, mean, invstd)
    for got, var in ((dx, x), (dg, gamma), (db, beta)):
        np.testing.assert_allclose(got, central(f, var), rtol=1e-6, atol=1e-8)


@pytest.mark.parametrize("t,lengths", [(1, None), (5, None), (4, [4, 0, 2]), (3, [-2, 9, 1])])
def test_gated_scan_gradient_by_differences(t, lengths):
    g = np.random.default_rng(t)
    n, c = 3, 2
    x, z, h0 = g.standard_normal((n, t, c)), g.standard_normal((n, t, c)) + 1, g.standard_normal((n, c))
    dh, dlast = g.standard_normal((n, t, c)), g.standard_normal((n, c))

    def f():
        h, last, _, _ = T.gated_scan_fwd(x, z, h0, lengths)
        return float((h * dh).sum() + (last * dlast).sum())

    prev = T.gated_scan_fwd(x, z, h0, lengths)[3]
    dx, dz, dh0, _ = T.gated_scan_bwd(dh, x, z, prev, dlast, lengths)
    for got, var in ((dx, x), (dz, z), (dh0, h0)):
        np.testing.assert_allclose(got, central(f, var), rtol=1e-6, atol=1e-8)


def test_gated_scan_closed_forms():
    n, t, c = 2, 130, 3
    g = np.random.default_rng(0)
    x, h0 = g.standard_normal((n, t, c)), g.standard_normal((n, c))
    with np.errstate(over="ignore"):
        h, last, states, _ = T.gated_scan_fwd(x, np.full((n, t, c), np.inf), h0)  # gates open: the state stays
        assert (h == h0[:, None]).all() and (last == h0).all() and (states == h0[:, None]).all()
        h, last, _, _ = T.gated_scan_fwd(x, np.full((n, t, c), -np.inf), h0)  # closed: the state is the input
        assert (h == x).all() and (last == x[:, -1]).all()
    h = T.gated_scan_fwd(x, np.zeros((n, t, c)), h0)[0]  # a = 1/2: weights 2^-(i - j + 1)
    i = 6
    want = h0 * 2.0 ** -(i + 1) + sum(x[:, j] * 2.0 ** -(i - j + 1) for j in range(i + 1))
    np.testing.assert_allclose(h[:, i], want, rtol=1e-13, atol=1e-15)
    # in two calls: the state of the first goes into the second
    z = g.standard_normal((n, t, c))
    whole, last, _, _ = T.gated_scan_fwd(x, z, h0)
    a, mid, _, _ = T.gated_scan_fwd(x[:, :50], z[:, :50], h0)
    b, end, _, _ = T.gated_scan_fwd(x[:, 50:], z[:, 50:], mid)
    assert (np.concatenate([a, b], 1) == whole).all() and (end == last).all()


def test_gates_keep_the_digits_of_the_smaller_one():
    z = np.array([-700.0, -40.0, -1.0, 0.0, 1.0, 40.0, 700.0])
    a, na = T.gates(z)
    np.testing.assert_allclose(na[5:], np.exp(-z[5:]), rtol=1e-12)
    np.testing.assert_allclose(a[:2], np.exp(z[:2]), rtol=1e-12)
    np.testing.assert_allclose(a + na, 1.0, rtol=0, atol=2e-16)


@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.5), (0.7, 0.0), (4.0, 0.9)])
def test_distillation_gradient_by_differences(tau, alpha):
    g = np.random.default_rng(int(tau * 10))
    n, v, k = 6, 7, 3
    z, top = 2 * g.standard_normal((n, v)), 2 * g.standard_normal((n, k))
    cls = np.stack([g.permutation(v)[:k] for _ in range(n)])
    cls[1, 2] = -1           # a shorter list
    cls[2] = v               # none
    cls[3] = [4, 4, 2]       # a class twice
    top[4, 0] = -np.inf      # an entry without weight
    labels = g.integers(0, v, n)
    labels[0] = -1
    w = g.uniform(0.1, 1.0, n)
    w[5] = 0.0
    f = lambda: T.distill(z, top, cls, labels, w, tau, alpha)[1]
    row, loss, dz, _ = T.distill(z, top, cls, labels, w, tau, alpha, 8.0)
    assert row[5] == 0 and (dz[5] == 0).all()
    np.testing.assert_allclose(dz / 8.0, central(f, z), rtol=1e-6, atol=1e-8)


def test_distillation_is_the_librarys_divergence_and_cross_entropy():
    g = np.random.default_rng(1)
    n, v, k, tau, alpha = 4, 9, 4, 2.0, 0.3
    z, top = g.standard_normal((n, v)), g.standard_normal((n, k))
    cls = np.stack([g.permutation(v)[:k] for _ in range(n)])
    labels = g.integers(0, v, n)
    p = np.zeros((n, v))
    for r in range(n):
        p[r, cls[r]] = torch.softmax(torch.from_numpy(top[r]) / tau, 0).numpy()
    tz = torch.from_numpy(z).requires_grad_(True)
    kl = torch.nn.functional.kl_div(torch.log_softmax(tz / tau, 1), torch.from_numpy(p), reduction="batchmean")
    ce = torch.nn.functional.cross_entropy(tz, torch.from_numpy(labels))
    want = alpha * tau ** 2 * kl + (1 - alpha) * ce
    want.backward()
    row, loss, dz, _ = T.distill(z, top, cls, labels, None, tau, alpha)
    assert abs(loss - float(want.detach())) <= 1e-12
    np.testing.assert_allclose(dz, tz.grad.numpy(), rtol=1e-10, atol=1e-13)


def test_distillation_of_the_same_distribution_has_no_loss():
    z = np.array([[0.5, 1.5, -1.0]])
    row, loss, dz, _ = T.distill(z, z[:, [2, 0, 1]], np.array([[2, 0, 1]]), temperature=3.0)
    assert abs(loss) <= 1e-15 and np.abs(dz).max() <= 1e-15
