"""The expert layer's calls together, as a program makes them: forward and backward with dropout on the stream, against the
64-bit forms one after the other; one captured graph for every routing; two layers at once on two streams."""
import numpy as np
import pytest
import torch

from gpu_common import check_status, load_dbl, ws
from oracle import experts as orc
from token_cases import DTYPE, UNIT, precision

pytestmark = pytest.mark.gpu


class Layer:
    """x [rows, w] -> res + drop(sum_j weight_j down_e relu(up_e x)), and its gradients from dy."""

    def __init__(self, D, kind, rows, w, hidden, experts, k, seed):
        self.D, self.kind, self.sizes = D, kind, (rows, w, hidden, experts, k)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *s, std=1.0: (torch.randn(s, device="cuda", generator=gen) * std).to(DTYPE[kind])
        n, dt = rows * k, DTYPE[kind]
        empty = lambda *s, t=dt: torch.zeros(s, dtype=t, device="cuda")
        self.up, self.down = new(experts, hidden, w, std=w ** -0.5), new(experts, w, hidden, std=hidden ** -0.5)
        self.x, self.res, self.dy, self.logits = new(rows, w), new(rows, w), new(rows, w), new(rows, experts)
        self.weight = torch.ones(rows, device="cuda")
        self.chosen, self.slots = empty(rows, k, t=torch.int32), empty(rows, k, t=torch.int32)
        self.offsets = empty(experts + 1, t=torch.int32)
        self.weights, self.dweights = empty(rows, k, t=torch.float32), empty(rows, k, t=torch.float32)
        self.xg, self.hg, self.yg, self.v, self.y = empty(n, w), empty(n, hidden), empty(n, w), empty(rows, w), empty(rows, w)
        self.dv, self.dyg, self.dhg, self.dxg, self.dx = empty(rows, w), empty(n, w), empty(n, hidden), empty(n, w), empty(rows, w)
        self.dlogits = empty(rows, experts)
        self.dup, self.ddown = empty(experts, hidden, w, t=torch.float32), empty(experts, w, hidden, t=torch.float32)
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.route = D.route_shape(rows, experts, k, False)
        self.swap, self.drop = D.exchange_shape(rows, k, w), D.dropout_shape(rows, w, 0.25, seed)
        self.g1, self.g2 = D.grouped_shape(n, experts, w, hidden, relu=True), D.grouped_shape(n, experts, hidden, w)
        need = [D.dbl_route_workspace_bytes(self.route)]
        need += [D.dbl_grouped_workspace_bytes(s, p) for s in (self.g1, self.g2) for p in range(3)]
        self.wsb = max(need)
        self.ws = ws(self.wsb)

    def run(self, s=None):
        D, sc = self.D, (self.ws, self.wsb)
        with precision(D, self.kind)[0]:
            D.dbl_route_fwd(self.route, self.logits, None, self.weight, self.chosen, self.weights, self.slots, self.offsets, *sc, s)
            D.dbl_expert_scatter(self.swap, self.x, self.slots, self.xg, s)
            D.dbl_grouped_fwd(self.g1, self.xg, self.up, self.offsets, self.hg, *sc, s)
            D.dbl_grouped_fwd(self.g2, self.hg, self.down, self.offsets, self.yg, *sc, s)
            D.dbl_expert_combine(self.swap, self.yg, self.slots, self.weights, None, self.v, s)
            D.dbl_dropout_residual(self.drop, self.v, self.res, self.step, self.y, s)
            D.dbl_dropout_residual(self.drop, self.dy, None, self.step, self.dv, s)
            D.dbl_expert_combine_bwd(self.swap, self.dv, self.yg, self.slots, self.weights, self.dyg, self.dweights, s)
            D.dbl_grouped_wgrad(self.g2, self.hg, self.dyg, self.offsets, self.ddown, False, *sc, s)
            D.dbl_grouped_dgrad(self.g2, self.dyg, self.down, self.offsets, self.hg, self.dhg, *sc, s)
            D.dbl_grouped_wgrad(self.g1, self.xg, self.dhg, self.offsets, self.dup, False, *sc, s)
            D.dbl_grouped_dgrad(self.g1, self.dhg, self.up, self.offsets, None, self.dxg, *sc, s)
            D.dbl_expert_combine(self.swap, self.dxg, self.slots, None, self.dy, self.dx, s)  # the skip path's gradient too
            D.dbl_route_bwd(self.route, self.logits, self.chosen, self.weights, self.dweights, self.dlogits, s)
            D.dbl_dropout_advance(self.step, s)

    def outputs(self):
        return [t.clone() for t in (self.y, self.dx, self.dlogits, self.dup, self.ddown, self.chosen, self.slots, self.offsets)]


def rel(got, want):
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("sizes", [(1, 64, 128, 4, 2), (300, 136, 264, 7, 3), (700, 256, 512, 40, 2)], ids=str)
def test_against_64_bits(kind, sizes):
    """Each stored tensor is off by about half of the format's largest rounding in its norm, one call after the other: the
    outputs lie behind 5 of them (x's rows are copied), the gradients behind 9 at most; twice that."""
    D = load_dbl()
    layer = Layer(D, kind, *sizes, seed=1)
    rows, w, _, experts, k = sizes
    if rows > 10:
        layer.weight[3::5] = 0
        layer.x[3::5] = float("nan")  # rows that go nowhere
    layer.run()
    check_status(D)
    f = lambda t: t.double().cpu().numpy()
    chosen, weights, slots, off = orc.route(f(layer.logits), k, False, None, f(layer.weight))
    assert (chosen == layer.chosen.cpu().numpy()).all() and (slots == layer.slots.cpu().numpy()).all()
    n = rows * k
    xg = orc.scatter(np.nan_to_num(f(layer.x)), slots, np.zeros((n, w)))
    passes = f(layer.hg) > 0
    h = orc.grouped_fwd(xg, f(layer.up), off)[0] * passes
    yg = orc.grouped_fwd(h, f(layer.down), off)[0]
    v = orc.combine(yg, slots, weights)[0]
    y = orc.dropout(v, 0.25, 1, 0, f(layer.res))
    dv = orc.dropout(f(layer.dy), 0.25, 1, 0)
    dyg, dwt, _ = orc.combine_bwd(dv, yg, slots, weights, np.zeros((n, w)))
    dh = orc.grouped_dgrad(dyg, f(layer.down), off)[0] * passes
    dxg = orc.grouped_dgrad(dh, f(layer.up), off)[0]
    dx = orc.combine(dxg, slots, None, f(layer.dy))[0]
    dz = orc.route_bwd(f(layer.logits), chosen, weights, dwt, False)[0]
    u = UNIT[kind][0]
    # The weights' gradients are sums over the columns that may come out small beside their terms dv*y, whose errors are
    # independent: such a sum is off by 2*sqrt(9)*u/2 of the terms' norm t_j, not of itself.  A row's dlogits are the differences
    # w_j*dw_j - p*sum(w*dw), and so off by 2*sum_j(w_j*t_j) of that at most in each of the k places where p and w are large.
    t = np.linalg.norm(dv[:, None] * np.where(slots[..., None] >= 0, yg[slots], 0), axis=2)
    size = np.sqrt(k) * 2 * (weights * t).sum(1)
    assert np.linalg.norm(f(layer.dlogits) - dz) <= 2 * 9 ** 0.5 * u / 2 * np.linalg.norm(size)
    for got, want, stored in ((layer.y, y, 5), (layer.dx, dx, 9),
                              (layer.dup, orc.grouped_wgrad(xg, dh, off), 9), (layer.ddown, orc.grouped_wgrad(h, dyg, off), 9)):
        assert rel(f(got), want) <= 2 * stored ** 0.5 * u / 2


def test_one_graph_for_every_routing():
    """The groups' lengths are the device's: a graph captured with one routing serves others, empty groups among them."""
    D = load_dbl()
    layer, other = (Layer(D, "bf16", 500, 128, 256, 12, 2, seed=2) for _ in range(2))
    layer.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        layer.run()
    for case in range(4):
        gen = torch.Generator(device="cuda").manual_seed(10 + case)
        z = torch.randn((500, 12), device="cuda", generator=gen)
        if case == 1:
            z[:, 3:] = -float("inf")  # three experts take all
        if case == 2:
            z[:] = -float("inf")  # no entry at all
        for t in (layer, other):
            t.logits.copy_(z)
            t.step.fill_(case)
            for b in (t.xg, t.hg, t.yg, t.dyg, t.dhg, t.dxg):
                b.zero_()
        graph.replay()
        other.run()
        check_status(D)
        for a, b in zip(layer.outputs(), other.outputs()):
            assert torch.equal(a, b)
        if case == 2:
            assert torch.equal(layer.y, layer.res) and not bool(layer.dup.any()) and int(layer.offsets[-1]) == 0


def test_two_layers_at_once():
    """Two streams, each layer with its own tensors and workspace: the bits of one after the other."""
    D = load_dbl()
    layers = [Layer(D, "bf16", 3000, 256, 512, 16, 2, seed=s) for s in (3, 4)]
    want = []
    for t in layers:
        t.run()
        torch.cuda.synchronize()
        want.append(t.outputs())
        t.step.zero_()
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    for _ in range(5):
        for t, s in zip(layers, streams):
            with torch.cuda.stream(s):
                t.step.zero_()
            t.run(s)
    check_status(D)
    for t, w in zip(layers, want):
        for a, b in zip(t.outputs(), w):
            assert torch.equal(a, b)
