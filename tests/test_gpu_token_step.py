"""The token model's training step: every gradient against automatic differentiation in 64 bits, the two workers and
the merge, and a training run.

Tolerance of a gradient, in its norm.  One rounding to the storage format moves a tensor by about u/2 of its norm (u the
format's largest relative error: half of it is reached in the mean over a binade), independently element by element; 23
stored tensors lie between the features and the deepest gradient and back (5 a layer and 3 forward, 4 a layer and 2
backward), which add up in squares: sqrt(23)*u/2.  Twice that for what a gate or a norm makes of an error: 2e-2 in
bfloat16, 2.4e-3 in binary16."""
import numpy as np
import pytest
import torch

from gpu_common import check_status, load_dbl
from token_cases import UNIT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def TS():
    load_dbl()
    from paper_2509_26092_gb300 import token_step
    return token_step


def setup(TS, prec, n=3, t=70, width=128, layers=2, classes=301, k=6, seed=0, scale="auto"):
    from paper_2509_26092_gb300 import dbl as D
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, device="cuda", generator=gen)
    spec = TS.TokenSpec(width, layers, classes)
    params = {}
    for e in spec.entries:
        if e.fan_in:
            params[e.name] = normal(*e.logical) / e.fan_in ** 0.5
        else:
            params[e.name] = (1.0 if e.name.endswith(".g") else 0.0) + 0.1 * normal(*e.logical)
    server = TS.ServerState(spec, params, precision=prec, loss_scale=scale)
    wk = TS.TokenWorker(spec, n, t, k, precision=prec)
    x = normal(n, t, width).to(TS.ACT_DTYPE[prec])
    cls = torch.argsort(torch.rand(n * t, classes, device="cuda", generator=gen), 1)[:, :k].to(torch.int32)
    wk.set_teacher(2 * normal(n * t, k), cls)
    wk.labels.copy_(torch.randint(0, classes, (n * t,), device="cuda", generator=gen, dtype=torch.int32))
    return D, spec, server, wk, x


def reference(spec, server, wk, x):
    """Loss and gradients of the same model in 64 bits, from the parameters that the step reads."""
    n, t, w = x.shape
    p = {}
    for e in spec.entries:
        src = server.w16 if e.fan_in else server.w
        p[e.name] = spec.view(src, e.name).double()[tuple(slice(0, d) for d in e.logical)].clone().requires_grad_(True)
    feats = x.double().clone().requires_grad_(True)
    ln = wk.lengths.long()
    s = feats.reshape(-1, w)
    norm = lambda v, name: torch.nn.functional.layer_norm(v, (w,), p[name + ".g"], p[name + ".b"], wk.eps)
    for i in range(spec.layers):
        u = (norm(s, f"layer{i}.norm") @ p[f"layer{i}.in.w"].T).reshape(n, t, 2 * w)
        a = torch.sigmoid(u[..., w:])
        h, hs = torch.zeros(n, w, dtype=torch.float64, device=x.device), []
        for j in range(t):
            new = a[:, j] * h + (1 - a[:, j]) * u[:, j, :w]
            inside = (j < ln)[:, None]
            h = torch.where(inside, new, h)
            hs.append(torch.where(inside, new, torch.zeros_like(new)))
        s = s + torch.stack(hs, 1).reshape(-1, w) @ p[f"layer{i}.out.w"].T
    z = norm(s, "norm") @ p["vocab.w"].T
    T, al = wk.loss_shape.temperature, wk.loss_shape.alpha
    pt = torch.softmax(wk.teacher_logits.double() / T, 1)
    lq = torch.log_softmax(z / T, 1).gather(1, wk.teacher_classes.long())
    kl = (pt * (pt.log() - lq)).sum(1)
    ce = -torch.log_softmax(z, 1).gather(1, wk.labels.long()[:, None])[:, 0]
    loss = (wk.weight.double() * (al * T * T * kl + (1 - al) * ce)).sum()
    names = list(p)
    grads = torch.autograd.grad(loss, [p[k] for k in names] + [feats])
    return float(loss.detach()), dict(zip(names + ["features"], grads))


@pytest.mark.parametrize("prec", ["bf16", "f16"])
@pytest.mark.parametrize("lengths", [None, [70, 1, 33]])
def test_step_matches_64_bits(TS, prec, lengths):
    D, spec, server, wk, x = setup(TS, prec)
    if lengths:
        wk.set_lengths(torch.tensor(lengths, dtype=torch.int32))
    s = torch.cuda.current_stream()
    wk.enqueue_step(server, x, wk.res, s)
    check_status(D)
    loss, want = reference(spec, server, wk, x)
    u = UNIT[prec][0]
    assert abs(float(wk.loss) - loss) <= 3 * u * loss
    scale = float(wk.scale_used) if server.scaled else 1.0
    tol = 2 * 23 ** 0.5 * u / 2
    for name, g in want.items():
        if name == "features":
            got = wk.dfeatures.double().reshape(g.shape) / scale
        else:
            whole = spec.view(wk.grad, name).double() / scale
            got = whole[tuple(slice(0, d) for d in g.shape)]
            assert float(whole.abs().sum()) == pytest.approx(float(got.abs().sum()))  # nothing in the padding
        err = float((got - g).norm() / g.norm())
        assert err <= tol, (name, err)


def test_worker_refuses_other_features(TS):
    D, spec, server, wk, x = setup(TS, "bf16")
    s = torch.cuda.current_stream()
    for bad, length in ((x[:, :-1].contiguous(), wk.res), (x.float(), wk.res), (x.transpose(0, 1), wk.res), (x, wk.res - 1)):
        with pytest.raises(ValueError):
            wk.enqueue_step(server, bad, length, s)
    with pytest.raises(ValueError):
        TS.TokenSpec(100)


@pytest.mark.parametrize("prec", ["bf16", "f16"])
def test_two_workers_merge_and_graph(TS, prec):
    """Two iterations of both workers and the merge, eagerly and as a replayed graph: the same bits."""
    def run(graph):
        D, spec, server, large, x = setup(TS, prec)
        _, _, _, small, y = setup(TS, prec, n=1, seed=1)
        it = TS.DualBatchIteration(server, large, small, large.res, lr=0.1)
        it.set_inputs(x, large.labels.clone(), y, small.labels.clone())
        if graph:
            state = [t.clone() for t in (server.w, server.u, server.w16, server.scale_state)]
            it.capture()  # runs once before it records
            for t, v in zip((server.w, server.u, server.w16, server.scale_state), state):
                t.copy_(v)
        for _ in range(2):
            it.run()
        check_status(D)
        return [t.clone() for t in (server.w, server.u, server.w16, large.loss, small.loss, large.grad, small.grad)]

    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b)


def test_training_lowers_the_loss(TS):
    losses = np.array(TS.demo(30))
    assert np.isfinite(losses).all()
    for part in np.split(losses, 3):  # one length each: the last iterations below the first of the run
        assert part[-3:].mean() < losses[0].mean()
    assert losses[-3:].mean() < 0.9 * losses[0].mean()
