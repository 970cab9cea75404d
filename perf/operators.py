"""Performance cases of the token operators: layer norm, the gated scan and the distillation loss.

They are the layers of a model over tokens that is trained as the ResNet-18 is (two workers, pushes merged by
the server, sizes that change from stage to stage): layer norm before each mixing layer and before the
vocabulary's product, the gated linear recurrence that mixes along the sequence, and the loss against a
teacher's stored top logits.  With ``own`` the passes are the package's entry points; without, the same
formulas in elementary torch operations.
"""
import math
import random

import torch

own = False

EPS = 1e-5
CHUNK = 64  # steps between the states that the scan's forward pass leaves for its backward pass
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # pooled features of a ResNet-18 worker (batch 256, 512 channels) before a classifier: bound by latency
        dict(name="ln_fwd_256x512", kind="ln_fwd", rows=256, c=512, res=False, dtype="bf16"),
        # a block's residual addition and norm in one pass over a worker's tokens, binary16 storage
        dict(name="ln_fwd_res_32768x1024_f16", kind="ln_fwd", rows=32768, c=1024, res=True, dtype="f16"),
        # odd rows and columns in fp32
        dict(name="ln_bwd_10007x1537_f32", kind="ln_bwd", rows=10007, c=1537, res=False, dtype="f32"),
        # backward of the residual form for a large worker: the gradient of the skip path joins dx
        dict(name="ln_bwd_res_65536x2048", kind="ln_bwd", rows=65536, c=2048, res=True, dtype="bf16"),
        # serving: one token for each of 64 sequences, the state carried from call to call
        dict(name="scan_fwd_64x1x512", kind="scan_fwd", n=64, t=1, c=512, ragged=False, packed=False, train=False,
             dtype="bf16"),
        # the positions of 14 x 14 maps (224 px) as tokens, an odd batch; x and gate are halves of one projection
        dict(name="scan_fwd_185x196x256_f16", kind="scan_fwd", n=185, t=196, c=256, ragged=False, packed=True,
             train=True, dtype="f16"),
        # one long sequence of few channels: little to do beside each other but along the sequence
        dict(name="scan_fwd_1x65536x512", kind="scan_fwd", n=1, t=65536, c=512, ragged=False, packed=False,
             train=True, dtype="bf16"),
        # sequences of different lengths in one batch, odd sizes
        dict(name="scan_bwd_ragged_12x3001x393", kind="scan_bwd", n=12, t=3001, c=393, ragged=True, packed=False,
             dtype="bf16"),
        # a large worker's backward pass, into the two halves of the projection's gradient
        dict(name="scan_bwd_8x8192x1024", kind="scan_bwd", n=8, t=8192, c=1024, ragged=False, packed=True,
             dtype="bf16"),
        # a classifier's 1000 classes, the paper's large batch at 288 px, with labels
        dict(name="distill_740x1000_f32", kind="distill", rows=740, classes=1000, k=16, labels=True, masked=False,
             temperature=2.0, alpha=0.5, dtype="f32"),
        # few rows of a large odd vocabulary, some rows without a target, logits in rows padded to 64
        dict(name="distill_9x131071_f16", kind="distill", rows=9, classes=131071, k=64, labels=False, masked=True,
             temperature=1.0, alpha=1.0, dtype="f16"),
        # a worker's tokens over a vocabulary, teacher and labels together
        dict(name="distill_4096x32000", kind="distill", rows=4096, classes=32000, k=32, labels=True, masked=True,
             temperature=2.0, alpha=0.7, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: any operator, sizes over the whole ranges, odd ones included."""
    kind = rng.choice(["ln_fwd", "ln_bwd", "scan_fwd", "scan_bwd", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("ln_fwd", "ln_bwd"):
        c = _log_int(rng, 8, 16384)
        if rng.random() < 0.5:
            c = -(-c // 64) * 64  # widths that a program picks
        rows = _log_int(rng, 1, min(65536, 2 ** 26 // c))
        return dict(kind=kind, rows=rows, c=c, res=rng.random() < 0.5, dtype=dtype)
    if kind in ("scan_fwd", "scan_bwd"):
        c = _log_int(rng, 16, 4096)
        if rng.random() < 0.5:
            c = -(-c // 64) * 64
        t = _log_int(rng, 1, min(65536, 2 ** 25 // c))
        n = _log_int(rng, 1, max(1, min(512, 2 ** 25 // (c * t))))
        case = dict(kind=kind, n=n, t=t, c=c, ragged=rng.random() < 0.4, packed=rng.random() < 0.4, dtype=dtype)
        if kind == "scan_fwd":
            case["train"] = rng.random() < 0.6
        return case
    classes = _log_int(rng, 10, 200000)
    if rng.random() < 0.4:
        classes = -(-classes // 8) * 8
    rows = _log_int(rng, 1, min(8192, 2 ** 26 // classes))
    labels = rng.random() < 0.5
    return dict(kind=kind, rows=rows, classes=classes, k=min(classes, _log_int(rng, 1, 128)), labels=labels,
                masked=rng.random() < 0.5, temperature=rng.choice([1.0, 1.5, 2.0, 4.0]),
                alpha=rng.choice([0.3, 0.5, 0.9]) if labels else 1.0, dtype=dtype)


# ------------------------------------------------------------------------------------------ helpers
class Gen:
    """Inputs drawn on the GPU from a seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, shape, std=1.0, dtype=torch.float32, mean=0.0):
        return torch.empty(shape, device="cuda").normal_(mean, std, generator=self.g).to(dtype)

    def uniform(self, shape, lo, hi):
        return torch.empty(shape, device="cuda").uniform_(lo, hi, generator=self.g)

    def ints(self, shape, hi):
        return torch.randint(0, hi, shape, generator=self.g, device="cuda", dtype=torch.int32)


def _lengths(case):
    """The lengths of a ragged batch: any from 0 to t, one sequence full.  Their sum goes by the case alone."""
    rng = random.Random(1000003 * case["n"] + case["t"])
    return [case["t"]] + [rng.randint(0, case["t"]) for _ in range(case["n"] - 1)]


def _size(case):
    return 4 if case["dtype"] == "f32" else 2


def work(case):
    e, kind = _size(case), case["kind"]
    if kind in ("ln_fwd", "ln_bwd"):
        n, c = case["rows"], case["c"]
        if kind == "ln_fwd":
            return {"bytes": n * c * e * (4 if case["res"] else 2) + 8 * n + 8 * c, "flops": 8 * n * c}
        return {"bytes": n * c * e * (4 if case["res"] else 3) + 8 * n + 12 * c, "flops": 14 * n * c}
    if kind in ("scan_fwd", "scan_bwd"):
        n, t, c = case["n"], case["t"], case["c"]
        live = (sum(_lengths(case)) if case["ragged"] else n * t) * c
        states = 4 * n * c * -(-t // CHUNK)
        if kind == "scan_fwd":
            return {"bytes": (2 * live + n * t * c) * e + 8 * n * c + (states if case["train"] else 0),
                    "flops": 8 * live}
        return {"bytes": (3 * live + 2 * n * t * c) * e + 8 * n * c + states, "flops": 16 * live}
    n, v, k = case["rows"], case["classes"], case["k"]
    return {"bytes": 2 * n * v * e + 8 * n * k + 8 * n + (4 * n if case["labels"] else 0),
            "flops": n * v * (16 if case["labels"] else 9)}


def _storage(case):
    """The library that stores in the case's format, and the element type that its calls are given."""
    from paper_2509_26092_gb300 import dbl as D
    return D, D.precision("f16" if case["dtype"] == "f16" else "bf16"), D.DBL_F32 if case["dtype"] == "f32" else D.DBL_BF16


def _workspace(st, need):
    """Scratch of the pass, kept with the state as a training program keeps it."""
    if need and ("ws" not in st or st["ws"].numel() < need):
        st["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return st.get("ws")


# ------------------------------------------------------------------------------------------ layer norm
def _prepare_ln(case, seed):
    """Rows of features with an offset of their own, as a network's are, and what the pass is given."""
    g, dt = Gen(seed), DTYPE[case["dtype"]]
    n, c = case["rows"], case["c"]
    st = {"case": case, "x": (g.normal((n, c), 1.3) + g.normal((n, 1), 0.5)).to(dt), "gamma": g.uniform((c,), 0.5, 1.5),
          "beta": g.normal((c,), 0.1)}
    out = {}
    if case["kind"] == "ln_fwd":
        st["res"] = g.normal((n, c), 1.0, dt) if case["res"] else None
        out["sum"] = torch.empty_like(st["x"]) if case["res"] else None
        out["y"] = torch.empty_like(st["x"])
        out["mean"], out["istd"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    else:
        x = st["x"].float()
        var, mean = torch.var_mean(x, 1, correction=0)
        st["mean"], st["istd"] = mean, torch.rsqrt(var + EPS)
        del x
        st["dy"] = g.normal((n, c), 1.0, dt)
        st["skip"] = g.normal((n, c), 1.0, dt) if case["res"] else None
        out["dx"] = torch.empty_like(st["x"])
        out["dgamma"], out["dbeta"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    st["out"] = out
    return st


def _own_ln(st):
    case, out = st["case"], st["out"]
    D, fmt, dtype = _storage(case)
    shape = D.ln_shape(case["rows"], case["c"], EPS, dtype)
    with fmt:
        if case["kind"] == "ln_fwd":
            D.dbl_layer_norm_fwd(shape, st["x"], st["res"], st["gamma"], st["beta"], out["sum"], out["y"], out["mean"],
                                 out["istd"])
            return [out["y"], out["mean"], out["istd"]] + ([out["sum"]] if case["res"] else [])
        need = D.dbl_layer_norm_workspace_bytes(shape)
        D.dbl_layer_norm_bwd(shape, st["dy"], st["skip"], st["x"], st["gamma"], st["mean"], st["istd"], out["dx"],
                             out["dgamma"], out["dbeta"], _workspace(st, need), need)
        return [out["dx"], out["dgamma"], out["dbeta"]]


def _plain_ln(st):
    case, dt = st["case"], DTYPE[st["case"]["dtype"]]
    x = st["x"].float()
    if case["kind"] == "ln_fwd":
        if case["res"]:
            x = x + st["res"].float()
        mean = x.mean(1, keepdim=True)
        d = x - mean
        istd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
        y = d * istd * st["gamma"] + st["beta"]
        return [y.to(dt), mean[:, 0], istd[:, 0]] + ([x.to(dt)] if case["res"] else [])
    dy = st["dy"].float()
    xhat = (x - st["mean"][:, None]) * st["istd"][:, None]
    g = dy * st["gamma"]
    dx = st["istd"][:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    if case["res"]:
        dx = dx + st["skip"].float()
    return [dx.to(dt), (dy * xhat).sum(0), dy.sum(0)]


def _exact_ln(st):
    case, c = st["case"], st["case"]["c"]
    outs = []
    sums = [torch.zeros(c, dtype=torch.float64, device="cuda") for _ in range(2)]
    step = max(1, 2 ** 26 // c)
    for i in range(0, case["rows"], step):
        at = slice(i, i + step)
        x = st["x"][at].double()
        if case["kind"] == "ln_fwd":
            if case["res"]:
                x += st["res"][at].double()
            m = x.sum(1) / c
            v = torch.einsum("rc,rc->r", x - m[:, None], x - m[:, None]) / c
            s = (v + EPS) ** -0.5
            y = torch.addcmul(st["beta"].double(), (x - m[:, None]) * s[:, None], st["gamma"].double())
            outs.append([y, m, s] + ([x] if case["res"] else []))
            continue
        dy, s = st["dy"][at].double(), st["istd"][at].double()
        h = (x - st["mean"][at].double()[:, None]) * s[:, None]
        sums[0] += torch.einsum("rc,rc->c", dy, h)
        sums[1] += dy.sum(0)
        g = dy * st["gamma"].double()
        dx = g - g.sum(1, keepdim=True) / c - h * (torch.einsum("rc,rc->r", g, h) / c)[:, None]
        dx *= s[:, None]
        if case["res"]:
            dx += st["skip"][at].double()
        outs.append([dx])
    whole = [torch.cat(o) for o in zip(*outs)]
    return whole if case["kind"] == "ln_fwd" else whole + sums


# ------------------------------------------------------------------------------------------ gated scan
def _pair(g, case, first, second):
    """Two [n, t, c] tensors, or the two halves of one [n, t, 2c] as a single projection writes them."""
    n, t, c, dt = case["n"], case["t"], case["c"], DTYPE[case["dtype"]]
    both = torch.empty((n, t, 2 * c) if case["packed"] else (2, n, t, c), dtype=dt, device="cuda")
    a, b = (both[..., :c], both[..., c:]) if case["packed"] else (both[0], both[1])
    if first is not None:
        for i in range(n):
            a[i] = g.normal((t, c), first[1], dt, first[0])
            b[i] = g.normal((t, c), second[1], dt, second[0])
    return both, a, b


def _prepare_scan(case, seed):
    """Inputs N(0, 1) and gates with memories from a few steps to some hundred: sigma of N(2.5, 1.5)."""
    g, dt = Gen(seed), DTYPE[case["dtype"]]
    n, t, c = case["n"], case["t"], case["c"]
    st = {"case": case, "h0": g.normal((n, c), 0.5)}
    st["both"], st["x"], st["gate"] = _pair(g, case, (0.0, 1.0), (2.5, 1.5))
    st["len"] = None
    if case["ragged"]:
        order = list(range(n))
        random.Random(seed).shuffle(order)
        ln = _lengths(case)
        st["len"] = torch.tensor([ln[i] for i in order], dtype=torch.int32, device="cuda")
    chunks = -(-t // CHUNK)
    out = {}
    if case["kind"] == "scan_fwd":
        out["h"] = torch.empty((n, t, c), dtype=dt, device="cuda")
        out["last"] = torch.empty((n, c), device="cuda")
        out["states"] = torch.empty((n, chunks, c), device="cuda") if case["train"] else None
    else:
        st["dh"] = g.normal((n, t, c), 1.0, dt)
        st["dlast"] = g.normal((n, c), 1.0)
        hs, _ = _scan_states(st)
        st["states"] = torch.cat([st["h0"][:, None], hs[:, CHUNK - 1:t - 1:CHUNK]], 1).contiguous()
        del hs
        out["both"], out["dx"], out["dgate"] = _pair(g, case, None, None)
        out["dh0"] = torch.empty((n, c), device="cuda")
    st["out"] = out
    return st


def _own_scan(st):
    case, out = st["case"], st["out"]
    D, fmt, dtype = _storage(case)
    shape = D.scan_shape(case["n"], case["t"], case["c"], dtype, 2 * case["c"] if case["packed"] else 0)
    with fmt:
        if case["kind"] == "scan_fwd":
            need = D.dbl_gated_scan_workspace_bytes(shape, D.DBL_PASS_FWD)
            D.dbl_gated_scan_fwd(shape, st["x"], st["gate"], st["h0"], st["len"], out["h"], out["last"], out["states"],
                                 _workspace(st, need), need)
            return [out["h"], out["last"]] + ([out["states"]] if case["train"] else [])
        need = D.dbl_gated_scan_workspace_bytes(shape, D.DBL_PASS_DGRAD)
        D.dbl_gated_scan_bwd(shape, st["dh"], st["dlast"], st["x"], st["gate"], st["states"], st["len"], out["dx"],
                             out["dgate"], out["dh0"], _workspace(st, need), need)
        return [out["dx"], out["dgate"], out["dh0"]]


def _live(st):
    """[n, t, 1]: the steps inside each sequence's length, or None where all are."""
    if st["len"] is None:
        return None
    return (torch.arange(st["case"]["t"], device="cuda")[None, :] < st["len"][:, None])[..., None]


def _scan(a, b):
    """Inclusive scan of h = a*h + b along dim 1 by doubling: (products of a, h from a zero state)."""
    t, s = a.shape[1], 1
    a, b = a.clone(), b.clone()
    while s < t:
        b[:, s:] = b[:, s:] + a[:, s:] * b[:, :-s]
        a[:, s:] = a[:, s:] * a[:, :-s]
        s *= 2
    return a, b


def _gates(st):
    """a = sigma(gate), 1 - a, from the exponential of -|gate|, which keeps the digits of the smaller one."""
    z = st["gate"].float()
    e = torch.exp(-z.abs())
    big, small = 1.0 / (1.0 + e), e / (1.0 + e)
    return torch.where(z >= 0, big, small), torch.where(z >= 0, small, big)


def _scan_states(st):
    """The states after every step (a step past a sequence's length leaves its state as it was), and the last."""
    a, na = _gates(st)
    b = na * st["x"].float()
    live = _live(st)
    if live is not None:
        a, b = torch.where(live, a, 1.0), torch.where(live, b, 0.0)
    p, h = _scan(a, b)
    h = h + p * st["h0"][:, None]
    return h, h[:, -1]


def _plain_scan(st):
    case, dt, live = st["case"], DTYPE[st["case"]["dtype"]], _live(st)
    t = case["t"]
    if case["kind"] == "scan_fwd":
        h, last = _scan_states(st)
        out = [(h if live is None else torch.where(live, h, 0.0)).to(dt), last.clone()]
        if case["train"]:
            out.append(torch.cat([st["h0"][:, None], h[:, CHUNK - 1:t - 1:CHUNK]], 1))
        return out
    h, _ = _scan_states(st)  # from the state before the sequence: the kept states are not needed here
    prev = torch.cat([st["h0"][:, None], h[:, :-1]], 1)
    del h
    a, na = _gates(st)
    dh = st["dh"].float()
    if live is not None:
        a, dh = torch.where(live, a, 1.0), torch.where(live, dh, 0.0)
    dh[:, -1] += st["dlast"]  # it reaches a shorter sequence's last step through gates of 1
    # total gradient of each state: G_t = dh_t + a_{t+1} G_{t+1}
    nxt = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    gt = _scan(nxt.flip(1), dh.flip(1))[1].flip(1)
    del nxt, dh
    dx, dz = na * gt, gt * (prev - st["x"].float()) * a * na
    if live is not None:
        dx, dz = torch.where(live, dx, 0.0), torch.where(live, dz, 0.0)
    return [dx.to(dt), dz.to(dt), a[:, 0] * gt[:, 0]]


def _exact_scan(st):
    """Step by step in 64 bits."""
    case = st["case"]
    n, t, c = case["n"], case["t"], case["c"]
    x, z = st["x"], st["gate"]
    ln = st["len"].long()[:, None] if st["len"] is not None else torch.full((n, 1), t, device="cuda")
    h = st["h0"].double()
    if case["kind"] == "scan_fwd":
        out = torch.empty((n, t, c), dtype=torch.float64, device="cuda")
        states = []
        for i in range(t):
            if i % CHUNK == 0:
                states.append(h)
            s = torch.sigmoid(z[:, i].double())
            new = torch.lerp(x[:, i].double(), h, s)
            inside = i < ln
            h = torch.where(inside, new, h)
            out[:, i] = new * inside
        return [out, h] + ([torch.stack(states, 1)] if case["train"] else [])
    prev = torch.empty((n, t, c), dtype=torch.float64, device="cuda")
    for i in range(t):
        prev[:, i] = h
        h = torch.where(i < ln, torch.lerp(x[:, i].double(), h, torch.sigmoid(z[:, i].double())), h)
    dx, dz = torch.zeros_like(prev), torch.zeros_like(prev)
    g = st["dlast"].double()
    for i in reversed(range(t)):
        inside = i < ln
        total = g + st["dh"][:, i].double()
        zi = z[:, i].double()
        s, r = torch.sigmoid(zi), torch.sigmoid(-zi)
        dx[:, i] = total * r * inside
        dz[:, i] = total * (prev[:, i] - x[:, i].double()) * (s * r) * inside
        g = torch.where(inside, total * s, g)
    return [dx, dz, g]


# ------------------------------------------------------------------------------------------ distillation
def _prepare_distill(case, seed):
    """A student's logits, the teacher's largest logits with their classes (largest first), labels near them.
    ``masked``: rows padded to 64 classes, some rows without weight, some of the teacher's lists shorter, some
    student logits of minus infinity."""
    g, dt = Gen(seed), DTYPE[case["dtype"]]
    n, v, k = case["rows"], case["classes"], case["k"]
    ld = -(-v // 64) * 64 if case["masked"] else v
    buf = torch.zeros((n, ld), dtype=dt, device="cuda")
    st = {"case": case, "buf": buf, "z": buf[:, :v], "labels": None, "weight": None, "scale": None}
    for i in range(0, n, 512):
        st["z"][i:i + 512] = g.normal((min(512, n - i), v), 2.0, dt)
    top, idx = [], []
    for i in range(0, n, 64):
        m = min(64, n - i)
        order = torch.argsort(g.uniform((m, v), 0.0, 1.0), 1)[:, :k]  # distinct classes
        idx.append(order.to(torch.int32))
        top.append(torch.sort(g.normal((m, k), 1.5), 1, descending=True)[0] + 6.0)
    st["top"], st["idx"] = torch.cat(top).contiguous(), torch.cat(idx).contiguous()
    # the student has begun to follow its teacher
    at = st["idx"].long()
    st["z"].scatter_(1, at, (st["z"].gather(1, at).float() * 0.5 + 0.8 * st["top"]).to(dt))
    if case["labels"]:
        st["labels"] = st["idx"][:, 0].clone()
        st["labels"][::5] = g.ints((n,), v)[::5]
    if case["masked"]:
        w = torch.ones(n, device="cuda")
        w[3::7] = 0.0
        st["weight"] = w / w.sum()
        st["idx"][4::6, k // 2:] = -1
        if case["labels"]:
            st["labels"][2::9] = -1
        free = torch.ones((n, v), dtype=torch.bool, device="cuda").scatter_(1, at, False)
        if case["labels"]:
            free.scatter_(1, st["labels"].long().clamp(min=0)[:, None], False)
        for i in range(0, n, 512):
            some = g.uniform((min(512, n - i), v), 0.0, 1.0) < 0.01
            st["z"][i:i + 512].masked_fill_(some & free[i:i + 512], -math.inf)
    if case["dtype"] == "f16":
        st["scale"] = torch.full((1,), 2.0 ** 10, device="cuda")  # the loss scaling of binary16 training
    st["out"] = {"buf": torch.zeros_like(buf), "row_loss": torch.empty(n, device="cuda"),
                 "loss": torch.empty(1, device="cuda")}
    st["out"]["dz"] = st["out"]["buf"][:, :v]
    return st


def _own_distill(st):
    case, out = st["case"], st["out"]
    D, fmt, dtype = _storage(case)
    shape = D.distill_shape(case["rows"], case["classes"], case["k"], case["temperature"], case["alpha"], dtype,
                            st["buf"].stride(0), out["buf"].stride(0))
    with fmt:
        D.dbl_distill_fwd_bwd(shape, st["z"], st["top"], st["idx"], st["labels"], st["weight"], st["scale"],
                              out["row_loss"], out["loss"], out["dz"])
    return [out["row_loss"], out["loss"], out["dz"]]


def _plain_distill(st):
    case = st["case"]
    n, v, tau, alpha = case["rows"], case["classes"], case["temperature"], case["alpha"]
    z = st["z"].float()
    there = (st["idx"] >= 0) & (st["idx"] < v) & (st["top"] != -math.inf)
    at = torch.where(there, st["idx"], 0).long()
    t = torch.where(there, st["top"], -math.inf) / tau
    t = t - t.max(1, keepdim=True)[0]
    p = torch.exp(t)
    total = p.sum(1, keepdim=True)
    p = p / total
    logp = t - torch.log(total)
    z = z - z.max(1, keepdim=True)[0]
    s = z / tau
    e = torch.exp(s)
    sum_e = e.sum(1, keepdim=True)
    logq = s.gather(1, at) - torch.log(sum_e)
    term = torch.where(there & (p > 0), p * (logp - logq), 0.0)
    some = there.any(1)
    loss = alpha * tau * tau * term.sum(1)
    dz = (alpha * tau) * (e / sum_e).scatter_add_(1, at, torch.where(there, -p, 0.0))
    dz = torch.where(some[:, None], dz, 0.0)
    if case["labels"]:
        lab = st["labels"].long()
        given = (lab >= 0) & (lab < v)
        lab = torch.where(given, lab, 0)[:, None]
        e = torch.exp(z)
        sum_e = e.sum(1, keepdim=True)
        ce = torch.log(sum_e) - z.gather(1, lab)
        loss = loss + (1 - alpha) * torch.where(given, ce[:, 0], 0.0)
        d = (e / sum_e).scatter_add_(1, lab, torch.full_like(ce, -1.0))
        dz = dz + (1 - alpha) * torch.where(given[:, None], d, 0.0)
    w = st["weight"] if st["weight"] is not None else torch.full((n,), 1.0 / n, device="cuda")
    loss = torch.where(w != 0, loss, 0.0)
    factor = w if st["scale"] is None else w * st["scale"]
    dz = torch.where(w[:, None] != 0, dz * factor[:, None], 0.0)
    return [loss, (w * loss).sum()[None], dz.to(DTYPE[case["dtype"]])]


def _exact_distill(st):
    """Row by row in 64 bits, the gradient by differentiating the loss."""
    case = st["case"]
    n, v, tau, alpha = case["rows"], case["classes"], case["temperature"], case["alpha"]
    w = st["weight"].double() if st["weight"] is not None else torch.full((n,), 1.0 / n, dtype=torch.float64,
                                                                          device="cuda")
    s = st["scale"].double() if st["scale"] is not None else 1.0
    losses, grads = [], []
    step = max(1, 2 ** 26 // v)
    for i in range(0, n, step):
        r = slice(i, min(n, i + step))
        z = st["z"][r].double().requires_grad_(True)
        idx = st["idx"][r].long()
        there = (idx >= 0) & (idx < v) & (st["top"][r] != -math.inf)
        p = torch.softmax(torch.where(there, st["top"][r].double() / tau, -1e30), 1) * there
        logq = torch.log_softmax(z / tau, 1)
        logq = torch.gather(logq, 1, idx.clamp(0, v - 1))
        kl = (torch.special.xlogy(p, p) - torch.where(p > 0, p * logq, 0.0)).sum(1)
        loss = alpha * tau ** 2 * kl
        if case["labels"]:
            lab = st["labels"][r].long()
            given = (lab >= 0) & (lab < v)
            nll = -torch.log_softmax(z, 1).gather(1, lab.clamp(0, v - 1)[:, None])[:, 0]
            loss = loss + (1 - alpha) * torch.where(given, nll, 0.0)
        loss = torch.where(w[r] != 0, loss, 0.0)
        grads.append(torch.autograd.grad((loss * w[r] * s).sum(), z)[0])
        losses.append(loss.detach())
    loss = torch.cat(losses)
    return [loss, (loss * w).sum()[None], torch.cat(grads)]


# ------------------------------------------------------------------------------------------ the interface
_KINDS = {"ln": (_prepare_ln, _own_ln, _plain_ln, _exact_ln), "scan": (_prepare_scan, _own_scan, _plain_scan, _exact_scan),
          "distill": (_prepare_distill, _own_distill, _plain_distill, _exact_distill)}


def _of(case):
    return _KINDS[case["kind"].split("_")[0]]


def prepare(case, seed):
    return _of(case)[0](case, seed)


def run(state):
    return _of(state["case"])[1 if own else 2](state)


def exact(case, seed):
    return _of(case)[3](prepare(case, seed))
