"""Graphs in which the expert layer's overlapping launches stand at every kind of edge: first of all, behind a fill, a copy or the
join of two streams, before a copy and before a fork.  A replay gives the eager call's bits, on inputs that changed in between."""
import pytest
import torch

from gpu_common import check_status, load_dbl, ws

pytestmark = pytest.mark.gpu


class Calls:
    """A split and a whole product, a weight gradient and a router of many rows."""

    def __init__(self, D):
        gen = torch.Generator(device="cuda").manual_seed(1)
        new = lambda *s: torch.randn(s, device="cuda", generator=gen).to(torch.bfloat16)
        self.D, self.rows, self.new = D, 6000, new
        self.x, self.w, self.deep = new(self.rows, 128), new(3, 192, 128), new(1, 64, 4096)
        self.few, self.logits = new(8, 4096), new(self.rows, 32)
        empty = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")
        self.y, self.small, self.dw = empty(self.rows, 192), empty(8, 64), empty(3, 192, 128, t=torch.float32)
        self.ints = [empty(self.rows, 2, t=torch.int32) for _ in range(2)] + [empty(33, t=torch.int32)]
        self.weights, self.copy = empty(self.rows, 2, t=torch.float32), empty(8, 64)
        self.off = torch.tensor([0, 1000, 1000, 5990], dtype=torch.int32, device="cuda")
        self.one = torch.tensor([0, 8], dtype=torch.int32, device="cuda")
        self.route = D.route_shape(self.rows, 32, 2)
        self.whole, self.split = D.grouped_shape(self.rows, 3, 128, 192), D.grouped_shape(8, 1, 4096, 64)
        self.need = [D.dbl_grouped_workspace_bytes(self.split, D.DBL_PASS_FWD),
                     D.dbl_grouped_workspace_bytes(self.whole, D.DBL_PASS_WGRAD), D.dbl_route_workspace_bytes(self.route)]
        assert self.need[0] and self.need[2]
        self.ws = [ws(n) for n in self.need]

    def products(self):
        self.D.dbl_grouped_fwd(self.split, self.few, self.deep, self.one, self.small, self.ws[0], self.need[0])
        self.D.dbl_grouped_fwd(self.whole, self.x, self.w, self.off, self.y)
        self.D.dbl_grouped_wgrad(self.whole, self.x, self.y, self.off, self.dw, False, self.ws[1], self.need[1])

    def router(self):
        chosen, slots, offsets = self.ints
        self.D.dbl_route_fwd(self.route, self.logits, None, None, chosen, self.weights, slots, offsets, self.ws[2], self.need[2])

    def outputs(self):
        return [self.y, self.small, self.dw, self.weights, self.copy] + self.ints

    def change(self):
        for t in (self.x, self.few, self.logits):
            t.copy_(self.new(*t.shape))


def alone(c, side):
    c.products()
    c.router()
    c.copy.copy_(c.small)


def behind_a_fill_and_a_copy(c, side):
    for t in c.outputs():
        t.zero_()
    c.copy.copy_(c.small)
    c.products()
    c.copy.copy_(c.small)  # behind the product
    c.router()


def behind_a_join(c, side):
    now = torch.cuda.current_stream()
    side.wait_stream(now)
    with torch.cuda.stream(side):
        c.router()
    c.y.zero_()
    now.wait_stream(side)
    c.products()
    side.wait_stream(now)
    with torch.cuda.stream(side):  # behind a fork
        c.copy.copy_(c.small)
        c.router()
    c.products()
    now.wait_stream(side)


def on_two_streams(c, side):
    now = torch.cuda.current_stream()
    side.wait_stream(now)
    with torch.cuda.stream(side):
        c.router()
        c.copy.zero_()
    c.products()
    now.wait_stream(side)
    c.D.dbl_grouped_fwd(c.split, c.few, c.deep, c.one, c.copy, c.ws[0], c.need[0])


@pytest.mark.parametrize("run", [alone, behind_a_fill_and_a_copy, behind_a_join, on_two_streams], ids=lambda f: f.__name__)
def test_every_edge(run):
    D = load_dbl()
    c, side = Calls(D), torch.cuda.Stream()
    run(c, side)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        run(c, side)
    for _ in range(3):
        c.change()
        for t in c.outputs():
            t.zero_()
        run(c, side)
        torch.cuda.synchronize()
        want = [t.clone() for t in c.outputs()]
        for t in c.outputs():
            t.fill_(3)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        # rows of no group stay as they were
        assert torch.equal(c.y[:5990], want[0][:5990])
        assert all(torch.equal(a, b) for a, b in zip(c.outputs()[1:], want[1:]))
    check_status(D)
