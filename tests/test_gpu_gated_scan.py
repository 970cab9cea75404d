"""The gated scan, forward and backward, against 64 bits.

Tolerances.  An error made at one step is carried on by the gates as the state is, so the bound follows the same
recurrence: with H the state's magnitude (the recurrence run on |x| and |h0|), each step adds at most K*2^-24*H_i to
what a_i passes on.  K = 40: the gates' exponential carries its argument's rounding (1.5*|gate| of 2^-24 relative, up
to |gate| = 14 here) and a few units of its own, their quotient two, and a state put together from the products of the
gates and the states of parts of the sequence rounds three times a step instead of two."""
import numpy as np
import pytest
import torch

from gpu_common import check_status, load_dbl
from oracle import tokens as T
from token_cases import DTYPE, EPS32, Rows, assert_within, precision, rounding

pytestmark = pytest.mark.gpu
K = 40


@pytest.fixture(scope="module")
def D():
    return load_dbl()


def carried(size, a, live, start):
    """e_i = a_i e_{i-1} + K 2^-24 size_i along dim 1."""
    e, out = start, np.zeros_like(size)
    for i in range(size.shape[1]):
        e = np.where(live[:, i], a[:, i] * e + K * EPS32 * size[:, i], e)
        out[:, i] = e
    return out, e


class Case:
    def __init__(self, kind, n, t, c, lengths=None, packed=False, gap=0, offset=0, h0=True, seed=0, gate_mean=2.5):
        g = np.random.default_rng(seed + 7 * n + 13 * t + c)
        self.kind, self.n, self.t, self.c, self.lengths = kind, n, t, c, lengths
        ld = 2 * c if packed else c + gap
        x, z = g.standard_normal((n * t, c)), np.clip(g.standard_normal((n * t, c)) * 1.5 + gate_mean, -14, 14)
        if lengths is not None:  # what lies past a length is not looked at
            for b, ln in enumerate(lengths):
                ln = min(max(ln, 0), t)
                x[b * t + ln:(b + 1) * t] = np.nan
                z[b * t + ln:(b + 1) * t] = np.inf
        self.ld, self.ldh = ld, c + gap
        if packed:
            self.both = Rows(kind, n * t, 2 * c, 0, offset, np.concatenate([x, z], 1))
            size = self.both.buf.element_size()
            self.px, self.pz = self.both.ptr(), self.both.ptr() + c * size
            v = self.both.values()
            self.x, self.z = v[:, :c].reshape(n, t, c), v[:, c:].reshape(n, t, c)
        else:
            self.rx, self.rz = Rows(kind, n * t, c, ld, offset, x), Rows(kind, n * t, c, ld, offset, z)
            self.px, self.pz = self.rx.ptr(), self.rz.ptr()
            self.x, self.z = self.rx.values().reshape(n, t, c), self.rz.values().reshape(n, t, c)
        self.packed, self.gap, self.offset = packed, gap, offset
        self.h0 = g.standard_normal((n, c)).astype(np.float32) if h0 else None
        self.th0 = torch.from_numpy(self.h0).cuda() if h0 else None
        self.len = torch.tensor(lengths, dtype=torch.int32, device="cuda") if lengths is not None else None
        ln = T._lengths(n, t, lengths)
        self.live = np.arange(t)[None, :, None] < ln[:, None, None]
        self.dh = Rows(kind, n * t, c, self.ldh, offset, g.standard_normal((n * t, c)))
        self.dlast = g.standard_normal((n, c)).astype(np.float32)
        self.clean = [np.where(self.live, v, 0.0) for v in (self.x, self.z)]

    def shape(self, D, dtype):
        return D.scan_shape(self.n, self.t, self.c, dtype, self.ld, self.ldh)


def run(D, case, states=True, last=True):
    lib, dtype = precision(D, case.kind)
    n, t, c = case.n, case.t, case.c
    chunks = -(-t // D.DBL_SCAN_CHUNK)
    h = Rows(case.kind, n * t, c, case.ldh, case.offset)
    out_last = Rows("f32", n, c)
    st = Rows("f32", n * chunks, c)
    with lib:
        shape = case.shape(D, dtype)
        assert D.dbl_gated_scan_states_bytes(shape) == 4 * n * chunks * c
        need = D.dbl_gated_scan_workspace_bytes(shape, D.DBL_PASS_FWD)
        ws = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
        D.dbl_gated_scan_fwd(shape, case.px, case.pz, case.th0, case.len, h.ptr(), out_last.ptr() if last else None,
                             st.ptr() if states else None, ws, need)
        check_status(D)
    for r in (h, out_last, st):
        r.check_guards()
    return h, out_last, st


CASES = [
    dict(n=1, t=1, c=1), dict(n=64, t=1, c=512), dict(n=3, t=2, c=5), dict(n=2, t=16, c=64), dict(n=2, t=17, c=66),
    dict(n=2, t=63, c=32), dict(n=1, t=64, c=64), dict(n=3, t=65, c=33), dict(n=2, t=127, c=8), dict(n=1, t=128, c=130),
    dict(n=5, t=129, c=64), dict(n=2, t=300, c=256, packed=True), dict(n=2, t=200, c=63, packed=True),
    dict(n=1, t=700, c=48, gap=5), dict(n=1, t=400, c=64, offset=1), dict(n=2, t=260, c=40, gap=8, offset=8),
    dict(n=1, t=5000, c=16), dict(n=1, t=4097, c=130), dict(n=1, t=9000, c=64), dict(n=40, t=196, c=256),
    dict(n=300, t=70, c=64), dict(n=700, t=3, c=96), dict(n=2, t=1500, c=600),
    dict(n=4, t=150, c=64, lengths=[150, 0, 1, 77]), dict(n=3, t=2100, c=35, lengths=[64, 2100, 128]),
    dict(n=6, t=64, c=64, lengths=[-3, 0, 99, 63, 64, 1]), dict(n=3, t=1, c=24, lengths=[0, 1, 1]),
    dict(n=2, t=600, c=64, lengths=[0, 0]), dict(n=2, t=333, c=48, h0=False), dict(n=2, t=900, c=64, gate_mean=9.0),
    dict(n=2, t=300, c=64, gate_mean=-3.0),
    # lengths that end whole parts of a block or a cluster before the tensor does
    dict(n=3, t=9000, c=64, lengths=[100, 9000, 4500]), dict(n=2, t=9000, c=15, lengths=[0, 8193]),
    dict(n=4, t=3001, c=101, lengths=[1024, 3000, 1, 2048], packed=True), dict(n=40, t=300, c=200, lengths=[7 * i for i in range(40)]),
]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_forward_and_backward(D, kind, case):
    cs = Case(kind, **case)
    n, t, c = cs.n, cs.t, cs.c
    h, last, st = run(D, cs)
    x, z = cs.clean
    wh, wl, wst, prev = T.gated_scan_fwd(x, z, cs.h0, cs.lengths)
    a, na = T.gates(z)
    size = T.gated_scan_fwd(np.abs(x), z, None if cs.h0 is None else np.abs(cs.h0), cs.lengths)
    E, Elast = carried(size[0], a, cs.live, np.zeros((n, c)))
    E = np.where(cs.live, E, 0.0)
    assert_within(h.values().reshape(n, t, c), wh, E + rounding(kind, np.abs(wh) + E) * cs.live, "h")
    assert_within(last.values(), wl, Elast, "h_last")
    Eprev = np.concatenate([np.zeros((n, 1, c)), carried(size[0], a, cs.live, np.zeros((n, c)))[0][:, :-1]], 1)
    chunk = D.DBL_SCAN_CHUNK
    assert_within(st.values().reshape(n, -1, c), wst, Eprev[:, ::chunk], "states")

    # the backward pass, from the forward pass's own states
    lib, dtype = precision(D, kind)
    width, ld = (2 * c, 2 * c) if cs.packed else (c, cs.ld)
    both = Rows(kind, n * t, width, ld, cs.offset)
    dz = None if cs.packed else Rows(kind, n * t, c, ld, cs.offset)
    dh0 = Rows("f32", n, c)
    dlast = torch.from_numpy(cs.dlast).cuda()
    pz = both.ptr() + c * both.buf.element_size() if cs.packed else dz.ptr()
    with lib:
        shape = cs.shape(D, dtype)
        need = D.dbl_gated_scan_workspace_bytes(shape, D.DBL_PASS_DGRAD)
        ws = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
        runs = []
        for _ in range(2):
            D.dbl_gated_scan_bwd(shape, cs.dh.ptr(), dlast, cs.px, cs.pz, st.ptr(), cs.len, both.ptr(), pz, dh0.ptr(),
                                 ws, need)
            runs.append([b.buf.clone() for b in (both, dh0) + (() if cs.packed else (dz,))])
        check_status(D)
    assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(*runs))
    for r in (both, dh0) + (() if cs.packed else (dz,)):
        r.check_guards()
    got = both.values()
    gx, gz = (got[:, :c], got[:, c:]) if cs.packed else (got, dz.values())
    DH = cs.dh.values().reshape(n, t, c)
    wx, wz, w0, whole = T.gated_scan_bwd(DH, x, z, prev, cs.dlast, cs.lengths)
    G = T.gated_scan_bwd(np.abs(DH), x, z, prev, np.abs(cs.dlast), cs.lengths)[3]
    # errors run from the last step to the first; a_{i+1} takes them from step i+1 to step i
    anext = np.concatenate([a[:, 1:], np.ones((n, 1, c))], 1)
    EG = carried(G[:, ::-1], anext[:, ::-1], cs.live[:, ::-1], np.zeros((n, c)))[0][:, ::-1]
    tolx = (na * EG + K * EPS32 * na * G) * cs.live
    assert_within(gx.reshape(n, t, c), wx, tolx + rounding(kind, np.abs(wx) + tolx) * cs.live, "dx")
    pm = np.concatenate([np.abs(cs.h0)[:, None] if cs.h0 is not None else np.zeros((n, 1, c)), size[0][:, :-1]], 1)
    tolz = a * na * ((EG + K * EPS32 * G) * (pm + np.abs(x)) + G * Eprev) * cs.live
    assert_within(gz.reshape(n, t, c), wz, tolz + rounding(kind, np.abs(wz) + tolz) * cs.live, "dgate")
    first = a[:, 0] * (EG[:, 0] + K * EPS32 * G[:, 0])
    assert_within(dh0.values(), w0, np.where(cs.live[:, 0], first, 0.0), "dh0")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_continued_call_by_call(D, kind):
    """A sequence in calls of 1, 70 and the remaining steps, the state updated in its own buffer, is the sequence
    in one call up to the order of its sums."""
    n, t, c = 3, 150, 80
    cs = Case(kind, n, t, c)
    lib, dtype = precision(D, kind)
    whole, last, _ = run(D, cs)
    state = cs.th0.clone()
    out = torch.zeros(n, t, c, dtype=DTYPE[kind], device="cuda")
    x, z = (r.view().reshape(n, t, c) for r in (cs.rx, cs.rz))
    at = 0
    with lib:
        for steps in (1, 70, t - 71):
            px, pz = x[:, at:at + steps].contiguous(), z[:, at:at + steps].contiguous()
            h = torch.empty(n, steps, c, dtype=DTYPE[kind], device="cuda")
            D.dbl_gated_scan_fwd(D.scan_shape(n, steps, c, dtype), px, pz, state, None, h, state, None)
            out[:, at:at + steps] = h
            at += steps
    wh, wl, _, _ = T.gated_scan_fwd(cs.x, cs.z, cs.h0)
    a, _ = T.gates(cs.z)
    size = T.gated_scan_fwd(np.abs(cs.x), cs.z, np.abs(cs.h0))[0]
    E, Elast = carried(size, a, cs.live, np.zeros((n, c)))
    assert_within(out.double().cpu().numpy(), wh, E + rounding(kind, np.abs(wh) + E), "h")
    assert_within(state.double().cpu().numpy(), wl, Elast, "state")


def test_gates_at_their_ends(D):
    """Infinite gates: open ones keep the state, closed ones take the input; a closed gate also ends what was not a
    number before it in no channel but its own."""
    n, t, c = 2, 200, 64
    for value in (np.inf, -np.inf):
        cs = Case("f32", n, t, c)
        cs.rz.view().fill_(value)
        h, last, st = run(D, cs)
        want = np.repeat(cs.h0[:, None], t, 1) if value > 0 else cs.x
        assert (h.values().reshape(n, t, c) == want).all() and (last.values() == want[:, -1]).all()
    cs = Case("f32", n, t, c)
    cs.rx.view()[70, 5] = float("nan")
    h, _, _ = run(D, cs)
    bad = np.isnan(h.values().reshape(n, t, c))
    assert bad[0, 70:, 5].all() and bad.sum() == t - 70
    h2, _, _ = run(D, Case("f32", n, t, c))
    assert (np.where(bad, 0, h.values().reshape(n, t, c)) == np.where(bad, 0, h2.values().reshape(n, t, c))).all()


def test_no_steps_and_no_sequences(D):
    c, n = 40, 3
    state = torch.randn(n, c, device="cuda")
    out = torch.zeros(n, c, device="cuda")
    none = D.scan_shape(n, 0, c)
    D.dbl_gated_scan_fwd(none, None, None, state, None, None, out, None)
    assert torch.equal(out, state)
    D.dbl_gated_scan_fwd(none, None, None, None, None, None, out, None)
    assert not out.any()
    D.dbl_gated_scan_bwd(none, None, state, None, None, None, None, None, None, out)
    assert torch.equal(out, state)
    D.dbl_gated_scan_fwd(D.scan_shape(0, 5, c), None, None, None, None, None, None, None)
    check_status(D)


def test_on_another_stream_and_in_a_graph(D):
    n, t, c = 2, 1000, 128
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, z, dh = (torch.randn(n, t, c, device="cuda", generator=gen).to(torch.bfloat16) for _ in range(3))
    shape = D.scan_shape(n, t, c)
    need = max(D.dbl_gated_scan_workspace_bytes(shape, p) for p in (D.DBL_PASS_FWD, D.DBL_PASS_DGRAD))
    ws = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
    chunks = -(-t // D.DBL_SCAN_CHUNK)

    def buffers():
        return ([torch.zeros(n, t, c, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
                + [torch.zeros(n, c, device="cuda"), torch.zeros(n, chunks, c, device="cuda"), torch.zeros(n, c, device="cuda")])

    def run_on(o, stream=None):
        D.dbl_gated_scan_fwd(shape, x, z, None, None, o[0], o[3], o[4], ws, need, stream)
        D.dbl_gated_scan_bwd(shape, dh, None, x, z, o[4], None, o[1], o[2], o[5], ws, need, stream)

    want, side, graphed = buffers(), buffers(), buffers()
    run_on(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    run_on(side, s)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_on(graphed)
    graph.replay()
    torch.cuda.synchronize()
    for a, b, d in zip(want, side, graphed):
        assert torch.equal(a, b) and torch.equal(a, d)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_gradient_is_the_slope_of_the_forward_pass(D, kind):
    """Central differences of the kernel's own forward pass, along a direction in x, gate and h0: in fp32 states
    (h_last) a step of 2^-4 leaves an error of its square times the third derivatives, 1e-3 of the slope at most here,
    and the states' rounding over the step."""
    n, t, c = 2, 90, 32
    cs = Case("f32", n, t, c, seed=4)
    g = np.random.default_rng(9)
    vx, vz, v0 = g.standard_normal((n * t, c)), g.standard_normal((n * t, c)), g.standard_normal((n, c))
    x0, z0, h00 = cs.rx.view().clone(), cs.rz.view().clone(), cs.th0.clone()
    step = 2.0 ** -4
    ends = []
    for s in (step, -step):
        cs.rx.view().copy_(x0 + s * torch.from_numpy(vx).cuda())
        cs.rz.view().copy_(z0 + s * torch.from_numpy(vz).cuda())
        cs.th0.copy_(h00 + s * torch.from_numpy(v0).cuda())
        ends.append(run(D, cs)[1].values())
    slope = float(((ends[0] - ends[1]) / (2 * step) * cs.dlast).sum())
    cs.rx.view().copy_(x0)
    cs.rz.view().copy_(z0)
    cs.th0.copy_(h00)
    _, _, st = run(D, cs)
    dt = DTYPE[kind]
    dx, dz = (torch.zeros(n, t, c, dtype=dt, device="cuda") for _ in range(2))
    dh0 = torch.zeros(n, c, device="cuda")
    lib, dtype = precision(D, kind)
    dh = torch.zeros(n, t, c, dtype=dt, device="cuda")
    with lib:
        D.dbl_gated_scan_bwd(D.scan_shape(n, t, c, dtype), dh, torch.from_numpy(cs.dlast).cuda(), cs.rx.view().to(dt),
                             cs.rz.view().to(dt), st.view(), None, dx, dz, dh0)
        torch.cuda.synchronize()
    got = sum(float((a.double().cpu().numpy().reshape(v.shape) * v).sum()) for a, v in ((dx, vx), (dz, vz), (dh0, v0)))
    terms = sum(float(np.abs(a.double().cpu().numpy().reshape(v.shape) * v).sum()) for a, v in ((dx, vx), (dz, vz), (dh0, v0)))
    assert abs(got - slope) <= (2e-3 if kind == "f32" else 2e-3 + 2.0 ** -8) * terms
