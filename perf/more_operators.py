"""Performance cases of the expert layer and of the dropout over tokens.

A layer of experts stands in a model over tokens where a block's second product stands: a router names the k
experts of every token and groups the tokens by expert, the tokens go to their groups, every group has products
of its own (with ReLU between the two), and the tokens take back the weighted sum of what their experts gave.
Dropout with the residual's addition follows, its rate raised from stage to stage.  With ``own`` the passes are
the package's entry points; without, the same formulas in elementary torch operations.
"""
import math
import random

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the tokens of one small request batch before a layer of few experts: bound by latency
        dict(name="route_fwd_64x8_f32", kind="route_fwd", rows=64, experts=8, k=2, normalise=True, bias=False,
             masked=False, dtype="f32"),
        # a large worker's tokens over many experts, with the balancing bias, padding rows and masked experts
        dict(name="route_fwd_65536x128", kind="route_fwd", rows=65536, experts=128, k=8, normalise=False, bias=True,
             masked=True, dtype="bf16"),
        # the router's gradient, odd sizes, weights out of the softmax over all experts
        dict(name="route_bwd_20011x60_f16", kind="route_bwd", rows=20011, experts=60, k=4, normalise=False, bias=False,
             masked=True, dtype="f16"),
        # the first product of a small worker's few tokens: every group is small, the weights are what is read
        dict(name="grouped_fwd_122x8_512x2048", kind="grouped_fwd", rows=122, groups=8, n_in=512, n_out=2048,
             relu=True, tail=0, dtype="bf16"),
        # the same product for a large worker: long groups of different lengths
        dict(name="grouped_fwd_65536x64_1024x4096", kind="grouped_fwd", rows=65536, groups=64, n_in=1024, n_out=4096,
             relu=True, tail=0, dtype="bf16"),
        # the gradient of the second product's input through the ReLU: odd widths, empty groups, rows past the last
        dict(name="grouped_dgrad_30011x24_2040x1000_f16", kind="grouped_dgrad", rows=30011, groups=24, n_in=2040,
             n_out=1000, relu=True, tail=500, dtype="f16"),
        # the weights' gradients of a large worker
        dict(name="grouped_wgrad_32768x16_1024x4096", kind="grouped_wgrad", rows=32768, groups=16, n_in=1024,
             n_out=4096, relu=False, tail=0, dtype="bf16"),
        # tokens to their two experts' groups
        dict(name="scatter_16384x2x1024", kind="scatter", rows=16384, k=2, c=1024, masked=False, dtype="bf16"),
        # the weighted sum back onto the residual stream, odd sizes, padding rows
        dict(name="combine_20011x2x1000_f16", kind="combine", rows=20011, k=2, c=1000, masked=True, dtype="f16"),
        # its gradients: the groups' rows and the weights
        dict(name="combine_bwd_32768x4x1024", kind="combine_bwd", rows=32768, k=4, c=1024, masked=False, dtype="bf16"),
        # dropout of a few rows in fp32: bound by latency
        dict(name="dropout_256x512_f32", kind="dropout", rows=256, c=512, rate=0.1, res=False, dtype="f32"),
        # dropout of a block's output onto the residual stream of a large worker
        dict(name="dropout_res_65536x2048", kind="dropout", rows=65536, c=2048, rate=0.3, res=True, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: any operator, sizes over the whole ranges, odd ones included."""
    kind = rng.choice(["route_fwd", "route_bwd", "grouped_fwd", "grouped_dgrad", "grouped_wgrad", "scatter", "combine",
                       "combine_bwd", "dropout"])
    if kind.startswith("route"):
        experts = _log_int(rng, 2, 512)
        return dict(kind=kind, rows=_log_int(rng, 1, min(65536, 2 ** 23 // experts)), experts=experts,
                    k=min(experts, _log_int(rng, 1, 12)), normalise=rng.random() < 0.5, bias=rng.random() < 0.5,
                    masked=rng.random() < 0.5, dtype=rng.choice(["bf16", "f16", "f32"]))
    if kind.startswith("grouped"):
        n_in, n_out = (8 * _log_int(rng, 8, 512) for _ in range(2))
        if rng.random() < 0.5:
            n_in, n_out = (-(-n // 64) * 64 for n in (n_in, n_out))
        groups = _log_int(rng, 1, min(128, 2 ** 28 // (n_in * n_out)))
        rows = _log_int(rng, 1, min(65536, 2 ** 38 // (n_in * n_out)))
        return dict(kind=kind, rows=rows, groups=groups, n_in=n_in, n_out=n_out, relu=rng.random() < 0.5,
                    tail=rng.choice([0, rows // 9]), dtype=rng.choice(["bf16", "bf16", "f16"]))
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    c = _log_int(rng, 8, 8192)
    if rng.random() < 0.5:
        c = -(-c // 64) * 64
    if kind == "dropout":
        return dict(kind=kind, rows=_log_int(rng, 1, min(65536, 2 ** 26 // c)), c=c, rate=rng.choice([0.05, 0.1, 0.2, 0.5]),
                    res=rng.random() < 0.5, dtype=dtype)
    k = _log_int(rng, 1, 8)
    return dict(kind=kind, rows=_log_int(rng, 1, min(65536, 2 ** 26 // (c * k))), k=k, c=c, masked=rng.random() < 0.5,
                dtype=dtype)


# ------------------------------------------------------------------------------------------ helpers
class Gen:
    """Inputs drawn on the GPU from a seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, device="cuda").normal_(0.0, std, generator=self.g).to(dtype)

    def uniform(self, shape, lo=0.0, hi=1.0):
        return torch.empty(shape, device="cuda").uniform_(lo, hi, generator=self.g)


def _size(case):
    return 4 if case["dtype"] == "f32" else 2


def _counts(case):
    """Rows of each group: some groups several times as long as others, an eighth of them empty, `tail` rows of
    the tensors in no group.  They go by the case alone."""
    groups, rows = case["groups"], case["rows"] - case["tail"]
    rng = random.Random(1000003 * groups + rows)
    share = [0.0 if groups >= 8 and i % 8 == 5 else math.exp(rng.gauss(0.0, 0.5)) for i in range(groups)]
    total, ends, run = sum(share), [], 0.0
    for s in share:
        run += s
        ends.append(min(rows, int(round(rows * run / total))))
    ends[-1] = rows
    return [b - a for a, b in zip([0] + ends, ends)]


def work(case):
    e, kind = _size(case), case["kind"]
    rows = case["rows"]
    if kind.startswith("route"):
        v, k = case["experts"], case["k"]
        if kind == "route_fwd":
            return {"bytes": rows * v * e + 12 * rows * k + 4 * (v + 1) + (4 * rows if case["masked"] else 0)
                    + (4 * v if case["bias"] else 0), "flops": rows * v * (k + 4)}
        return {"bytes": rows * v * e * (1 if case["normalise"] else 2) + 12 * rows * k, "flops": rows * v * 6}
    if kind.startswith("grouped"):
        counts, n_in, n_out = _counts(case), case["n_in"], case["n_out"]
        live, used = sum(counts), sum(1 for c in counts if c)
        weights = (4 * len(counts) if kind == "grouped_wgrad" else e * used) * n_in * n_out
        mask = e * live * n_in if kind == "grouped_dgrad" and case["relu"] else 0
        return {"bytes": e * live * (n_in + n_out) + weights + mask + 4 * (len(counts) + 1),
                "flops": 2 * live * n_in * n_out}
    c = case["c"]
    if kind == "dropout":
        return {"bytes": rows * c * e * (3 if case["res"] else 2), "flops": 20 * rows * c}
    k = case["k"]
    live = rows - rows // 8 if case["masked"] else rows
    if kind == "scatter":
        return {"bytes": live * c * e * (1 + k) + 4 * rows * k, "flops": 0}
    if kind == "combine":
        return {"bytes": c * e * (2 * rows + k * live) + 8 * rows * k, "flops": 2 * live * k * c}
    return {"bytes": live * c * e * (1 + 2 * k) + 12 * rows * k, "flops": 3 * live * k * c}


def _storage(case):
    """The library that stores in the case's format, and the element type that its calls are given."""
    from paper_2509_26092_gb300 import dbl as D
    return D, D.precision("f16" if case["dtype"] == "f16" else "bf16"), D.DBL_F32 if case["dtype"] == "f32" else D.DBL_BF16


def _workspace(st, need):
    """Scratch of the pass, kept with the state as a training program keeps it."""
    if need and ("ws" not in st or st["ws"].numel() < need):
        st["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return st.get("ws")


def _group_by_expert(chosen, experts):
    """Each entry's row among all entries ordered by expert, then by row and entry (-1: no expert), and where each
    expert's rows begin and end."""
    flat = torch.where(chosen >= 0, chosen, experts).reshape(-1).long()
    order = torch.sort(flat, stable=True)[1]
    slots = torch.empty_like(order)
    slots[order] = torch.arange(flat.numel(), device=flat.device)
    slots = torch.where(flat < experts, slots, -1).to(torch.int32).reshape(chosen.shape)
    counts = torch.zeros(experts + 1, dtype=torch.int64, device=flat.device).scatter_add_(0, flat, torch.ones_like(flat))
    offsets = torch.cat([counts.new_zeros(1), torch.cumsum(counts[:experts], 0)]).to(torch.int32)
    return slots, offsets


# ------------------------------------------------------------------------------------------ the router
def _prepare_route(case, seed):
    """Logits of experts that are not all alike.  ``masked``: padding rows of weight 0 (an eighth, at the ends of
    sequences), some experts closed to some rows (-infinity)."""
    g, dt = Gen(seed), DTYPE[case["dtype"]]
    rows, v, k = case["rows"], case["experts"], case["k"]
    z = g.normal((rows, v), 1.5) + g.normal((v,), 0.5)
    st = {"case": case, "weight": None, "bias": g.normal((v,), 0.2) if case["bias"] else None}
    if case["masked"]:
        at = torch.arange(rows, device="cuda")
        st["weight"] = torch.where(at % 64 >= 56, 0.0, 1.0 / rows)
        z = torch.where(g.uniform((rows, v)) < 0.05, -math.inf, z)
    st["z"] = z.to(dt)
    if case["kind"] == "route_fwd":
        st["out"] = {"chosen": torch.empty((rows, k), dtype=torch.int32, device="cuda"),
                     "weights": torch.empty((rows, k), device="cuda"),
                     "slots": torch.empty((rows, k), dtype=torch.int32, device="cuda"),
                     "offsets": torch.empty(v + 1, dtype=torch.int32, device="cuda")}
    else:
        st["chosen"], st["weights"] = (t.contiguous() for t in _choose(st))
        st["dw"] = g.normal((rows, k))
        st["out"] = torch.empty_like(st["z"])
    return st


def _choose(st):
    """The k largest of logit + bias in every row (the first of equals), and the softmax's weights."""
    case, z = st["case"], st["z"].float()
    key = z if st["bias"] is None else z + st["bias"]
    top, at = torch.sort(key, dim=1, descending=True, stable=True)
    top, at = top[:, :case["k"]], at[:, :case["k"]]
    there = top > -math.inf
    if st["weight"] is not None:
        there = there & (st["weight"] != 0)[:, None]
    zc = torch.where(there, z.gather(1, at), -math.inf)
    over = zc if case["normalise"] else z
    peak = over.max(1, keepdim=True)[0]
    peak = torch.where(peak > -math.inf, peak, 0.0)
    weights = torch.exp(zc - peak) / torch.exp(over - peak).sum(1, keepdim=True)
    return torch.where(there, at, -1).to(torch.int32), torch.where(there, weights, 0.0)


def _own_route(st):
    case, out = st["case"], st["out"]
    D, fmt, dtype = _storage(case)
    shape = D.route_shape(case["rows"], case["experts"], case["k"], case["normalise"], dtype)
    with fmt:
        if case["kind"] == "route_fwd":
            need = D.dbl_route_workspace_bytes(shape)
            D.dbl_route_fwd(shape, st["z"], st["bias"], st["weight"], out["chosen"], out["weights"], out["slots"],
                            out["offsets"], _workspace(st, need), need)
            return [out["chosen"], out["weights"], out["slots"], out["offsets"]]
        D.dbl_route_bwd(shape, st["z"], st["chosen"], st["weights"], st["dw"], out)
    return [out]


def _plain_route(st):
    case = st["case"]
    if case["kind"] == "route_fwd":
        chosen, weights = _choose(st)
        slots, offsets = _group_by_expert(chosen, case["experts"])
        return [chosen, weights, slots, offsets]
    there = st["chosen"] >= 0
    at = torch.where(there, st["chosen"], 0).long()
    wdw = torch.where(there, st["weights"] * st["dw"], 0.0)
    dot = wdw.sum(1, keepdim=True)
    if case["normalise"]:
        dz = torch.zeros(st["z"].shape, device="cuda")
        dz.scatter_add_(1, at, torch.where(there, wdw - st["weights"] * dot, 0.0))
    else:
        z = st["z"].float()
        peak = z.max(1, keepdim=True)[0]
        e = torch.exp(z - torch.where(peak > -math.inf, peak, 0.0))
        dz = -dot * (e / e.sum(1, keepdim=True))
        dz.scatter_add_(1, at, wdw)
        dz = torch.where(there.any(1, keepdim=True), dz, 0.0)
    return [dz.to(DTYPE[case["dtype"]])]


def _exact_route(st):
    case = st["case"]
    z = st["z"].double()
    if case["kind"] == "route_fwd":
        key = (st["z"].float() + (st["bias"] if st["bias"] is not None else 0.0)).double()
        picked, logit = [], []
        for _ in range(case["k"]):
            best = key.argmax(1, keepdim=True)  # the first of equals
            ok = key.gather(1, best) > -math.inf
            if st["weight"] is not None:
                ok &= st["weight"][:, None] != 0
            picked.append(ok)
            logit.append(z.gather(1, best))
            key = key.scatter(1, best, -math.inf)
        ok, zc = torch.cat(picked, 1), torch.cat(logit, 1).masked_fill(~torch.cat(picked, 1), -math.inf)
        norm = torch.logsumexp(zc if case["normalise"] else z, 1, keepdim=True)
        return [None, torch.exp(zc - norm).masked_fill(~ok, 0.0), None, None]
    there = st["chosen"] >= 0
    at = st["chosen"].long().clamp(min=0)
    some = there.any(1, keepdim=True)
    safe = torch.where(some, z, 0.0).requires_grad_(True)
    if case["normalise"]:
        w = torch.softmax(safe.gather(1, at).masked_fill(~there, -1e300), 1)
    else:
        w = torch.softmax(safe, 1).gather(1, at)
    dz = torch.autograd.grad(torch.where(there, w * st["dw"].double(), 0.0).sum(), safe)[0]
    return [torch.where(some, dz, 0.0)]


# ------------------------------------------------------------------------------------------ grouped products
def _prepare_grouped(case, seed):
    """Tokens, experts' weights [groups, out, in] of the usual scale, and the groups' ends on the device."""
    g, dt, kind = Gen(seed), DTYPE[case["dtype"]], case["kind"]
    rows, n_in, n_out, groups = case["rows"], case["n_in"], case["n_out"], case["groups"]
    st = {"case": case, "counts": _counts(case)}
    ends = [0]
    for c in st["counts"]:
        ends.append(ends[-1] + c)
    st["offsets"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    if kind != "grouped_wgrad":
        st["w"] = torch.cat([g.normal((1, n_out, n_in), n_in ** -0.5, dt) for _ in range(groups)])
    if kind != "grouped_dgrad":
        st["x"] = g.normal((rows, n_in), 1.0, dt)
    if kind != "grouped_fwd":
        st["dy"] = g.normal((rows, n_out), 1.0, dt)
    if kind == "grouped_dgrad":
        # what the ReLU before this product left
        st["mask"] = torch.clamp(g.normal((rows, n_in), 1.0, dt), min=0) if case["relu"] else None
    shape = {"grouped_fwd": (rows, n_out), "grouped_dgrad": (rows, n_in), "grouped_wgrad": (groups, n_out, n_in)}[kind]
    st["out"] = torch.zeros(shape, dtype=torch.float32 if kind == "grouped_wgrad" else dt, device="cuda")
    return st


def _own_grouped(st):
    case, out = st["case"], st["out"]
    D, fmt, _ = _storage(case)
    kind = case["kind"]
    shape = D.grouped_shape(case["rows"], case["groups"], case["n_in"], case["n_out"], relu=case["relu"])
    with fmt:
        which = {"grouped_fwd": D.DBL_PASS_FWD, "grouped_dgrad": D.DBL_PASS_DGRAD, "grouped_wgrad": D.DBL_PASS_WGRAD}[kind]
        need = D.dbl_grouped_workspace_bytes(shape, which)
        ws = _workspace(st, need)
        if kind == "grouped_fwd":
            D.dbl_grouped_fwd(shape, st["x"], st["w"], st["offsets"], out, ws, need)
        elif kind == "grouped_dgrad":
            D.dbl_grouped_dgrad(shape, st["dy"], st["w"], st["offsets"], st["mask"], out, ws, need)
        else:
            D.dbl_grouped_wgrad(shape, st["x"], st["dy"], st["offsets"], out, False, ws, need)
    return [out]


def _plain_grouped(st):
    """Each group's product of exactly its rows."""
    case, out, kind = st["case"], st["out"], st["case"]["kind"]
    at = 0
    for i, c in enumerate(st["counts"]):
        r = slice(at, at + c)
        at += c
        if kind == "grouped_fwd":
            y = st["x"][r].float() @ st["w"][i].float().t()
            out[r] = (torch.clamp(y, min=0) if case["relu"] else y).to(out.dtype)
        elif kind == "grouped_dgrad":
            y = st["dy"][r].float() @ st["w"][i].float()
            out[r] = (torch.where(st["mask"][r] > 0, y, 0.0) if case["relu"] else y).to(out.dtype)
        else:
            out[i] = st["dy"][r].float().t() @ st["x"][r].float()
    return [out]


def _exact_grouped(st):
    case, kind = st["case"], st["case"]["kind"]
    parts, at = [], 0
    for i, c in enumerate(st["counts"]):
        if kind == "grouped_wgrad":
            parts.append(torch.einsum("po,pi->oi", st["dy"][at:at + c].double(), st["x"][at:at + c].double())[None])
        elif kind == "grouped_fwd":
            y = torch.einsum("pi,oi->po", st["x"][at:at + c].double(), st["w"][i].double())
            parts.append(y.relu() if case["relu"] else y)
        else:
            y = torch.einsum("po,oi->pi", st["dy"][at:at + c].double(), st["w"][i].double())
            parts.append(y * (st["mask"][at:at + c] > 0) if case["relu"] else y)
        at += c
    if kind != "grouped_wgrad":
        parts.append(torch.zeros((case["tail"], parts[0].shape[1]), dtype=torch.float64, device="cuda"))
    return [torch.cat(parts)]


# ------------------------------------------------------------------------------------------ tokens to groups and back
def _prepare_exchange(case, seed):
    """A routing over 16 experts (or k, if that is more); ``masked``: every eighth row goes nowhere."""
    g, dt, kind = Gen(seed), DTYPE[case["dtype"]], case["kind"]
    rows, k, c = case["rows"], case["k"], case["c"]
    experts = max(16, k)
    chosen = torch.argsort(g.uniform((rows, experts)) ** g.uniform((experts,), 0.5, 2.0), 1)[:, :k].to(torch.int32)
    weights = g.uniform((rows, k), 0.1, 1.0)
    if case["masked"]:
        nowhere = torch.arange(rows, device="cuda") % 8 == 7
        chosen = torch.where(nowhere[:, None], -1, chosen)
        weights = torch.where(nowhere[:, None], 0.0, weights)
    st = {"case": case, "weights": (weights / weights.sum(1, keepdim=True).clamp(min=1e-6)).contiguous()}
    st["slots"] = _group_by_expert(chosen, experts)[0].contiguous()
    if kind == "scatter":
        st["x"] = g.normal((rows, c), 1.0, dt)
        st["out"] = torch.zeros((rows * k, c), dtype=dt, device="cuda")
        return st
    st["yg"] = g.normal((rows * k, c), 1.0, dt)
    if kind == "combine":
        st["res"] = g.normal((rows, c), 1.0, dt)
        st["out"] = torch.empty((rows, c), dtype=dt, device="cuda")
    else:
        st["dout"] = g.normal((rows, c), 1.0, dt)
        st["out"] = torch.zeros((rows * k, c), dtype=dt, device="cuda")
        st["dweights"] = torch.empty((rows, k), device="cuda")
    return st


def _own_exchange(st):
    case, out, kind = st["case"], st["out"], st["case"]["kind"]
    D, fmt, dtype = _storage(case)
    shape = D.exchange_shape(case["rows"], case["k"], case["c"], dtype=dtype)
    with fmt:
        if kind == "scatter":
            D.dbl_expert_scatter(shape, st["x"], st["slots"], out)
        elif kind == "combine":
            D.dbl_expert_combine(shape, st["yg"], st["slots"], st["weights"], st["res"], out)
        else:
            D.dbl_expert_combine_bwd(shape, st["dout"], st["yg"], st["slots"], st["weights"], out, st["dweights"])
            return [out, st["dweights"]]
    return [out]


def _plain_exchange(st):
    case, out, kind = st["case"], st["out"], st["case"]["kind"]
    rows, k, c = case["rows"], case["k"], case["c"]
    there = (st["slots"] >= 0)[..., None]
    at = torch.where(st["slots"] >= 0, st["slots"], rows * k).long()  # a row more than there are takes what goes nowhere
    if kind == "scatter":
        grouped = torch.zeros((rows * k + 1, c), dtype=out.dtype, device="cuda")
        grouped[at] = st["x"][:, None]
        return [grouped[:-1]]
    y = torch.where(there, st["yg"][at.clamp(max=rows * k - 1)].float(), 0.0)
    if kind == "combine":
        return [(st["res"].float() + (st["weights"][..., None] * y).sum(1)).to(out.dtype)]
    d = st["dout"].float()[:, None]
    grouped = torch.zeros((rows * k + 1, c), dtype=out.dtype, device="cuda")
    grouped[at] = (st["weights"][..., None] * d).to(out.dtype)
    return [grouped[:-1], (y * d).sum(2)]


def _exact_exchange(st):
    case, kind = st["case"], st["case"]["kind"]
    rows, k, c = case["rows"], case["k"], case["c"]
    row = torch.arange(rows, device="cuda")[:, None].expand(rows, k)
    live = st["slots"] >= 0
    slot = st["slots"][live].long()
    if kind == "combine":
        total = st["res"].double()
        return [total.index_add(0, row[live], st["yg"][slot].double() * st["weights"][live].double()[:, None])]
    grouped = torch.zeros((rows * k, c), dtype=torch.float64, device="cuda")
    if kind == "scatter":
        return [grouped.index_copy(0, slot, st["x"][row[live]].double())]
    d = st["dout"][row[live]].double()
    dots = torch.zeros((rows, k), dtype=torch.float64, device="cuda")
    dots[live] = torch.einsum("rc,rc->r", d, st["yg"][slot].double())
    return [grouped.index_copy(0, slot, d * st["weights"][live].double()[:, None]), dots]


# ------------------------------------------------------------------------------------------ dropout
SEED, STEP = 0x9D2C5680A3F1, 77


def _prepare_dropout(case, seed):
    g, dt = Gen(seed), DTYPE[case["dtype"]]
    shape = (case["rows"], case["c"])
    return {"case": case, "x": g.normal(shape, 1.0, dt), "res": g.normal(shape, 1.0, dt) if case["res"] else None,
            "step": torch.full((1,), STEP, dtype=torch.int64, device="cuda"), "seed": SEED + int(seed),
            "out": torch.empty(shape, dtype=dt, device="cuda")}


def _own_dropout(st):
    case = st["case"]
    D, fmt, dtype = _storage(case)
    shape = D.dropout_shape(case["rows"], case["c"], case["rate"], st["seed"], dtype)
    with fmt:
        D.dbl_dropout_residual(shape, st["x"], st["res"], st["step"], st["out"])
    return [st["out"]]


def _threshold(case):
    """A word below it is dropped; the rate is the fp32 value."""
    rate = float(torch.tensor(case["rate"], dtype=torch.float32))
    return int(rate * 2.0 ** 32), rate


def _plain_dropout(st):
    """Philox4x32-10 (Salmon et al., SC 2011): block r*ceil(c/4) + c/4 of the call's step, one word an element."""
    case, x = st["case"], st["x"]
    rows, c, low = case["rows"], case["c"], 0xFFFFFFFF
    per = -(-c // 4)
    block = torch.arange(rows * per, device="cuda")
    c0, c1 = block & low, block >> 32
    c2, c3 = st["step"] & low, st["step"] >> 32
    k0, k1 = st["seed"] & low, st["seed"] >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # the low 64 bits, which are all of them
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    threshold, rate = _threshold(case)
    keep = torch.stack([c0 >= threshold, c1 >= threshold, c2 >= threshold, c3 >= threshold], 1).view(rows, 4 * per)[:, :c]
    y = torch.where(keep, x.float() / (1.0 - rate), 0.0)
    return [(y if st["res"] is None else y + st["res"].float()).to(x.dtype)]


def _exact_dropout(st):
    """The same words from 16-bit halves, all four counters as one tensor."""
    case, x = st["case"], st["x"]
    rows, c = case["rows"], case["c"]
    per = -(-c // 4)
    threshold, rate = _threshold(case)
    outs, step = [], max(1, 2 ** 25 // c)

    def product(m, v):
        """(high, low) 32 bits of m*v."""
        ml, mh, vl, vh = m & 65535, m >> 16, v & 65535, v >> 16
        mid = (ml * vl >> 16) + (mh * vl & 65535) + (ml * vh & 65535)
        return mh * vh + (mh * vl >> 16) + (ml * vh >> 16) + (mid >> 16), (mid & 65535) << 16 | (ml * vl & 65535)

    for r in range(0, rows, step):
        n = min(step, rows - r)
        index = torch.arange(r * per, (r + n) * per, device="cuda")
        w = [index % 2 ** 32, index // 2 ** 32, torch.full_like(index, STEP), torch.zeros_like(index)]
        for i in range(10):
            key = [((st["seed"] >> s) + i * m) % 2 ** 32 for s, m in ((0, 0x9E3779B9), (32, 0xBB67AE85))]
            (h0, l0), (h1, l1) = product(0xD2511F53, w[0]), product(0xCD9E8D57, w[2])
            w = [h1 ^ w[1] ^ key[0], l1, h0 ^ w[3] ^ key[1], l0]
        dropped = torch.cat([v[:, None] for v in w], 1).reshape(n, -1)[:, :c] < threshold
        y = (x[r:r + n].double() / (1.0 - rate)).masked_fill(dropped, 0.0)
        outs.append(y if st["res"] is None else y + st["res"][r:r + n].double())
    return [torch.cat(outs)]


# ------------------------------------------------------------------------------------------ the interface
_ROUTE = (_prepare_route, _own_route, _plain_route, _exact_route)
_GROUPED = (_prepare_grouped, _own_grouped, _plain_grouped, _exact_grouped)
_EXCHANGE = (_prepare_exchange, _own_exchange, _plain_exchange, _exact_exchange)
_DROPOUT = (_prepare_dropout, _own_dropout, _plain_dropout, _exact_dropout)
_KINDS = {"route": _ROUTE, "grouped": _GROUPED, "scatter": _EXCHANGE, "combine": _EXCHANGE, "dropout": _DROPOUT}


def _of(case):
    return _KINDS[case["kind"].split("_")[0]]


def prepare(case, seed):
    return _of(case)[0](case, seed)


def run(state):
    return _of(state["case"])[1 if own else 2](state)


def exact(case, seed):
    return _of(case)[3](prepare(case, seed))
