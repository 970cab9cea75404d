"""A training step of the token model with a layer of experts behind each mixing layer, and with dropout: every gradient
against differentiation in 64 bits, padding, the graph, and the run of both workers.

The reference takes the experts that the step chose, the ReLU's passes and the dropout's masks as they were (the masks from the
generator's definition): a choice or a pass that a rounding turned would be another function's gradient.  Tolerance of a
gradient, in its norm, as for the model without experts: one rounding to the storage format moves a tensor by about u/2 of its
norm, independently; forward and back lie at most 23 stored tensors of the mixing layers and their ends, 16 of each layer of
experts (6 forward, 8 backward, the router's two) and 2 of each dropout, which add up in squares; twice that for what a norm, a
gate or a difference of weights' gradients makes of an error."""
import numpy as np
import pytest
import torch

from gpu_common import check_status
from oracle import experts as orc
from test_gpu_token_step import TS  # noqa: F401  (the fixture)
from token_cases import UNIT

pytestmark = pytest.mark.gpu


def setup(TS, prec, n=3, t=70, width=128, layers=2, classes=301, k=6, seed=0, experts=6, hidden=200, chosen=2, dropout=0.0):
    from paper_2509_26092_gb300 import dbl as D
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, device="cuda", generator=gen)
    spec = TS.TokenSpec(width, layers, classes, experts, hidden, chosen)
    params = {}
    for e in spec.entries:
        if e.fan_in:
            params[e.name] = normal(*e.logical) / e.fan_in ** 0.5
        else:
            params[e.name] = (1.0 if e.name.endswith(".g") else 0.0) + 0.1 * normal(*e.logical)
    server = TS.ServerState(spec, params, precision=prec)
    wk = TS.TokenWorker(spec, n, t, k, precision=prec, dropout=dropout, seed=99)
    x = normal(n, t, width).to(TS.ACT_DTYPE[prec])
    cls = torch.argsort(torch.rand(n * t, classes, device="cuda", generator=gen), 1)[:, :k].to(torch.int32)
    wk.set_teacher(2 * normal(n * t, k), cls)
    wk.labels.copy_(torch.randint(0, classes, (n * t,), device="cuda", generator=gen, dtype=torch.int32))
    return D, spec, server, wk, x


def reference(spec, server, wk, x, step):
    """Loss and gradients of the same model in 64 bits, from the parameters that the step read."""
    n, t, w = x.shape
    p = {}
    for e in spec.entries:
        src = server.w16 if e.fan_in else server.w
        p[e.name] = spec.view(src, e.name).double()[tuple(slice(0, d) for d in e.logical)].clone().requires_grad_(True)
    feats = x.double().clone().requires_grad_(True)
    ln = wk.lengths.long()
    s = feats.reshape(-1, w)
    norm = lambda v, name: torch.nn.functional.layer_norm(v, (w,), p[name + ".g"], p[name + ".b"], wk.eps)

    def drop(v, j):
        if not wk.dropout:
            return v
        shape = wk.drops[j]
        keep = torch.from_numpy(orc.dropout_mask(n * t, w, shape.rate, shape.seed, step)).to(x.device)
        return torch.where(keep, v / (1.0 - shape.rate), torch.zeros_like(v))

    for j, d in enumerate(wk.blocks[:-1]):
        a = norm(s, d["norm"])
        if d["kind"] == "mix":
            u = (a @ p[d["pre"] + ".in.w"].T).reshape(n, t, 2 * w)
            g = torch.sigmoid(u[..., w:])
            h, hs = torch.zeros(n, w, dtype=torch.float64, device=x.device), []
            for i in range(t):
                new = g[:, i] * h + (1 - g[:, i]) * u[:, i, :w]
                inside = (i < ln)[:, None]
                h = torch.where(inside, new, h)
                hs.append(torch.where(inside, new, torch.zeros_like(new)))
            v = torch.stack(hs, 1).reshape(-1, w) @ p[d["pre"] + ".out.w"].T
        else:
            chosen, slots = (d[q].reshape(-1, spec.chosen).long() for q in ("chosen", "slots"))
            live = slots >= 0
            z = a @ p[d["pre"] + ".router.w"].T
            weights = torch.softmax(z.gather(1, chosen.clamp(min=0)).masked_fill(~live, -1e300), 1)
            up, down = p[d["pre"] + ".up.w"][chosen.clamp(min=0)], p[d["pre"] + ".down.w"][chosen.clamp(min=0)]
            passes = d["hg"][slots.clamp(min=0)] > 0
            h = torch.einsum("rjhw,rw->rjh", up, a) * passes
            y = torch.einsum("rjwh,rjh->rjw", down, h) * live[..., None]
            v = (weights[..., None] * y).sum(1)
        s = s + drop(v, j)
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
@pytest.mark.parametrize("dropout", [0.0, 0.25])
@pytest.mark.parametrize("experts,lengths", [(6, None), (6, [70, 1, 33]), (0, None)])
def test_step_matches_64_bits(TS, prec, dropout, experts, lengths):  # noqa: F811
    D, spec, server, wk, x = setup(TS, prec, experts=experts, dropout=dropout)
    if lengths:
        wk.set_lengths(torch.tensor(lengths, dtype=torch.int32))
    s = torch.cuda.current_stream()
    for step in (0, 1):  # the second with other masks, over what the first left in the buffers
        wk.enqueue_step(server, x, wk.res, s)
    check_status(D)
    assert int(wk.step) == (2 if dropout else 0)
    loss, want = reference(spec, server, wk, x, step)
    u = UNIT[prec][0]
    assert abs(float(wk.loss) - loss) <= 3 * u * loss
    scale = float(wk.scale_used) if server.scaled else 1.0
    stored = 23 + (16 * spec.layers if experts else 0) + (2 * (len(wk.blocks) - 1) if dropout else 0)
    tol = 2 * stored ** 0.5 * u / 2
    for name, g in want.items():
        if name == "features":
            got = wk.dfeatures.double().reshape(g.shape) / scale
        else:
            whole = spec.view(wk.grad, name).double() / scale
            got = whole[tuple(slice(0, d) for d in g.shape)]
            assert float(whole.abs().sum()) == pytest.approx(float(got.abs().sum()))  # nothing in the padding
        err = float((got - g).norm() / g.norm())
        assert err <= tol, (name, err)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_features_past_a_length_do_not_count(TS, value):  # noqa: F811
    outs = []
    for fill in (0.0, value):
        D, spec, server, wk, x = setup(TS, "bf16", dropout=0.1)
        wk.set_lengths(torch.tensor([70, 1, 33], dtype=torch.int32))
        for b, ln in enumerate((70, 1, 33)):
            x[b, ln:] = fill
        wk.enqueue_step(server, x, wk.res, torch.cuda.current_stream())
        check_status(D)
        chosen = wk.blocks[1]["chosen"].view(3, 70, 2)
        assert bool((chosen[1, 1:] == -1).all()) and bool((chosen[0] >= 0).all())
        outs.append([t.clone() for t in (wk.loss, wk.grad, wk.dfeatures)])
        assert all(bool(torch.isfinite(t.float()).all()) for t in outs[-1])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("prec", ["bf16", "f16"])
def test_two_workers_merge_and_graph(TS, prec):  # noqa: F811
    """Two iterations of both workers and the merge, eagerly and as a replayed graph: the same bits, with new masks."""
    def run(graph):
        D, spec, server, large, x = setup(TS, prec, dropout=0.2)
        _, _, _, small, y = setup(TS, prec, n=1, seed=1, dropout=0.2)
        it = TS.DualBatchIteration(server, large, small, large.res, lr=0.1)
        it.set_inputs(x, large.labels.clone(), y, small.labels.clone())
        if graph:
            state = [t.clone() for t in (server.w, server.u, server.w16, server.scale_state)]
            it.capture()  # runs once before it records
            for t, v in zip((server.w, server.u, server.w16, server.scale_state), state):
                t.copy_(v)
            large.step.zero_()
            small.step.zero_()
        for _ in range(2):
            it.run()
        check_status(D)
        assert int(large.step) == int(small.step) == 2
        return [t.clone() for t in (server.w, server.u, server.w16, large.loss, small.loss, large.grad, small.grad)]

    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b)


def test_a_run_and_its_gradients_are_finite(TS):  # noqa: F811
    losses = np.array(TS.demo(6, experts=5, dropout=0.3))
    assert losses.shape == (6, 2) and np.isfinite(losses).all()


def test_refusals(TS):  # noqa: F811
    for kw in (dict(experts=4, hidden=100), dict(experts=4, chosen=5), dict(experts=4, chosen=0), dict(experts=2000)):
        with pytest.raises(ValueError):
            TS.TokenSpec(128, 1, 10, **kw)
