"""Training step of a small model over tokens, for the scheme's server and workers.

The scheme asks of a model only that a worker turns a batch into its batch-mean gradient (Eq. 1 of
arXiv 2509.26092): the server's merge (Sec. 3.4), the two workers on their streams and the graph
capture are those of ``resnet18.py`` (``ServerState``, ``DualBatchIteration``).  Where cyclic
progressive learning (Sec. 4.1) raises the resolution of images from sub-stage to sub-stage, here it
is the length of the sequences: one ``TokenWorker`` per length, all on the same server.

The model takes features [n, t, width] (the positions of a feature map, or embeddings) and predicts
one of ``classes`` at every token:

    s = features
    for each layer:  s = s + drop( out.w * scan( in.w * norm(s) ) )   (x and gate: the halves of in.w's output)
        with experts:  s = s + drop( sum_j weight_j * down.w[e_j] * relu( up.w[e_j] * norm(s) ) )
    logits = vocab.w * norm(s)

with layer norm, the gated scan and the distillation loss against a teacher's stored top logits
(``dbl_layer_norm_*``, ``dbl_gated_scan_*``, ``dbl_distill_fwd_bwd``) and the products as 1x1
convolutions.  A layer of experts (``experts`` of them, ``chosen`` for a token, of ``hidden`` channels) takes
the largest of router.w * norm(s) with their softmax as weights (``dbl_route_*``), the tokens to their experts'
rows and back (``dbl_expert_*``) and the products of each expert's rows (``dbl_grouped_*``).  drop is dropout
(``dbl_dropout_residual``), whose rate cyclic progressive learning raises with the sub-stage; without it the
residual additions run inside the norms, forward and backward.
"""
import argparse
import itertools

import torch

from . import dbl as D
from .resnet18 import ACT_DTYPE, DualBatchIteration, FlatSpec, ServerState


# the seeds of workers that are given none, far from those that programs give
_next_seed = itertools.count(1 << 63)


class TokenSpec(FlatSpec):
    """Parameters of the model: ``width`` channels (a multiple of 64), ``layers``, ``classes`` (any number;
    stored in rows padded to a multiple of 64, the padding staying zero).  ``experts`` > 0: a layer of experts
    behind each mixing layer, of ``hidden`` channels (a multiple of 8; 0: 4 * width), ``chosen`` for each token."""

    def __init__(self, width=512, layers=2, classes=1000, experts=0, hidden=0, chosen=2):
        super().__init__()
        if width % 64:
            raise ValueError("width must be a multiple of 64")
        hidden = hidden or 4 * width
        if experts and (hidden < 8 or hidden % 8 or not 1 <= chosen <= min(experts, D.DBL_ROUTE_MAX_K)
                        or experts > D.DBL_ROUTE_MAX_EXPERTS):
            raise ValueError(f"a layer of experts has 1 to {D.DBL_ROUTE_MAX_EXPERTS} experts, 1 to "
                             f"{D.DBL_ROUTE_MAX_K} of them for a token, and a multiple of 8 hidden channels")
        self.width, self.layers, self.classes = width, layers, classes
        self.experts, self.hidden, self.chosen = experts, hidden, chosen
        self.padded = -(-classes // 64) * 64
        self.routed = -(-experts // 64) * 64  # the router's output, padded likewise
        for i in range(layers):
            self._norm(f"layer{i}.norm")
            self.add(f"layer{i}.in.w", (2 * width, width), (2 * width, width), width)
            self.add(f"layer{i}.out.w", (width, width), (width, width), width)
            if experts:
                self._norm(f"layer{i}.experts.norm")
                self.add(f"layer{i}.router.w", (self.routed, width), (experts, width), width)
                self.add(f"layer{i}.up.w", (experts, hidden, width), (experts, hidden, width), width)
                self.add(f"layer{i}.down.w", (experts, width, hidden), (experts, width, hidden), hidden)
        self._norm("norm")
        self.add("vocab.w", (self.padded, width), (classes, width), width)

    def _norm(self, name):
        self.add(name + ".g", (self.width,), (self.width,), None)
        self.add(name + ".b", (self.width,), (self.width,), None)


class TokenWorker:
    """Activations, gradients and scratch of one worker: ``n`` sequences of ``t`` tokens, a teacher of ``k``
    logits per token.  ``lengths`` ([n] int32, all t at first) ends sequences earlier; tokens past them count
    neither in the loss nor in the states nor, whatever their features hold, in a gradient, and go to no expert.
    ``dropout``: the rate of what each layer adds to the stream, its masks drawn from ``seed`` and ``step``, the
    worker's count of its iterations on the device.  Workers of the same seed have the same masks at the same step;
    one that is given none has its own, the next in the order in which the program makes them.  What a step reads
    (teacher, lengths, labels) is set on the current stream, which the next iteration follows."""

    def __init__(self, spec, n, t, k, temperature=2.0, alpha=0.5, device="cuda", eps=1e-5, precision="bf16",
                 dropout=0.0, seed=None):
        self.spec, self.batch, self.res, self.k, self.eps, self.precision = spec, n, t, k, eps, precision
        rows, w = n * t, spec.width
        self.rows = rows
        dt = ACT_DTYPE[precision]

        def act(c):
            return torch.zeros((rows, c), dtype=dt, device=device)

        def vec(m, dtype=torch.float32):
            return torch.zeros(m, dtype=dtype, device=device)

        def entries(c):
            return torch.zeros((rows * spec.chosen, c), dtype=dt, device=device)

        self.norm_shape = D.ln_shape(rows, w, eps)
        self.scan_shape = D.scan_shape(n, t, w, ld_x=2 * w)  # x and gate are the halves of one projection
        self.loss_shape = D.distill_shape(rows, spec.classes, k, temperature, alpha, ld=spec.padded, ld_grad=spec.padded)
        self.in_shape = D.conv_shape(n, t, 1, w, 2 * w, 1, 1, 0)
        self.out_shape = D.conv_shape(n, t, 1, w, w, 1, 1, 0)
        self.vocab_shape = D.conv_shape(n, t, 1, w, spec.padded, 1, 1, 0)
        chunks = D.dbl_gated_scan_states_bytes(self.scan_shape) // 4
        # what reads the stream, in order; each has the norm's output, s (but the first) and the norm's statistics,
        # and what it adds to the stream (v); the last is the norm before the vocabulary
        def block(kind, pre, norm, **more):
            return dict(kind=kind, pre=pre, norm=norm, a=act(w), v=act(w) if kind else None, mean=vec(rows), istd=vec(rows),
                        s=act(w) if self.blocks else None, **more)

        self.blocks = []
        for i in range(spec.layers):
            self.blocks.append(block("mix", f"layer{i}", f"layer{i}.norm", u=act(2 * w), h=act(w), states=vec(chunks),
                                     layer=i))
            if spec.experts:
                self.blocks.append(block("experts", f"layer{i}", f"layer{i}.experts.norm", r=act(spec.routed),
                                         chosen=vec(rows * spec.chosen, torch.int32), slots=vec(rows * spec.chosen, torch.int32),
                                         weights=vec(rows * spec.chosen), offsets=vec(spec.experts + 1, torch.int32),
                                         xg=entries(w), hg=entries(spec.hidden), yg=entries(w)))
        self.blocks.append(block(None, None, "norm"))
        self.last = self.blocks[-1]
        if spec.experts:
            self.router_shape = D.conv_shape(n, t, 1, w, spec.routed, 1, 1, 0)
            self.route_shape = D.route_shape(rows, spec.experts, spec.chosen, True, ld=spec.routed, ld_grad=spec.routed)
            self.exchange_shape = D.exchange_shape(rows, spec.chosen, w)
            self.up_shape = D.grouped_shape(rows * spec.chosen, spec.experts, w, spec.hidden, relu=True)
            self.down_shape = D.grouped_shape(rows * spec.chosen, spec.experts, spec.hidden, w)
            self.dhg, self.dr, self.dweights = entries(spec.hidden), act(spec.routed), vec(rows * spec.chosen)
        self.dropout, self.step = float(dropout), torch.zeros(1, dtype=torch.int64, device=device)
        seed = next(_next_seed) if seed is None else seed
        self.drops = [D.dropout_shape(rows, w, dropout, seed ^ (0x9E3779B97F4A7C15 * (i + 1)))
                      for i in range(len(self.blocks) - 1)]
        self.dv = act(w) if self.dropout else None
        self.h_last = torch.zeros((spec.layers, n, w), device=device)
        self.logits = act(spec.padded)  # its gradient takes its place; the padding stays zero
        self.da, self.dh, self.du, self.ds = act(w), act(w), act(2 * w), [act(w), act(w)]
        self.teacher_logits = torch.zeros((rows, k), device=device)
        self.teacher_classes = torch.full((rows, k), -1, dtype=torch.int32, device=device)
        self.labels = torch.full((rows,), -1, dtype=torch.int32, device=device)
        self.lengths = torch.full((n,), t, dtype=torch.int32, device=device)
        self.weight = torch.full((rows,), 1.0 / rows, device=device)
        # the features that count: of the others a NaN would reach the weights' gradients as NaN times 0
        self.live = torch.ones((n, t, 1), dtype=torch.bool, device=device)
        self.features, self.none = act(w).view(n, t, w), torch.zeros((), dtype=dt, device=device)
        self.row_loss, self.loss = vec(rows), vec(1)
        self.grad = vec(spec.n_flat)
        self.scale_used = torch.ones(1, device=device)
        need = [D.dbl_layer_norm_workspace_bytes(self.norm_shape),
                D.dbl_gated_scan_workspace_bytes(self.scan_shape, D.DBL_PASS_FWD),
                D.dbl_gated_scan_workspace_bytes(self.scan_shape, D.DBL_PASS_DGRAD)]
        passes, convs = (D.DBL_PASS_FWD, D.DBL_PASS_DGRAD, D.DBL_PASS_WGRAD), [self.in_shape, self.out_shape, self.vocab_shape]
        if spec.experts:
            convs.append(self.router_shape)
            need.append(D.dbl_route_workspace_bytes(self.route_shape))
            need += [D.dbl_grouped_workspace_bytes(s, p) for s in (self.up_shape, self.down_shape) for p in passes]
        need += [D.dbl_conv_workspace_bytes(s, p) for s in convs for p in passes]
        self.ws = torch.empty(int(max(need)) + 256, dtype=torch.uint8, device=device)

    def set_teacher(self, logits, classes):
        """The teacher's top logits of this batch ([n*t, k] fp32) and their classes (int32; -1: none)."""
        self.teacher_logits.copy_(logits.reshape(self.rows, self.k))
        self.teacher_classes.copy_(classes.reshape(self.rows, self.k))

    def set_lengths(self, lengths):
        """Tokens that count in each sequence ([n] int32); the loss is the mean over them all."""
        self.lengths.copy_(lengths)
        steps = torch.arange(self.res, device=self.lengths.device)
        self.live.copy_((steps[None, :] < self.lengths[:, None])[..., None])
        live = self.live.float().reshape(-1)
        self.weight.copy_(live / live.sum().clamp(min=1.0))

    def enqueue_step(self, server, features, native_len, stream):
        """Forward, loss, backward; gradients land in self.grad (means over the tokens that count, times the
        loss scale under loss scaling).  features: [n, t, width] in the storage format."""
        if server.precision != self.precision:
            raise ValueError(f"worker stores {self.precision}, the model's copy is {server.precision}")
        if native_len != self.res or tuple(features.shape) != (self.batch, self.res, self.spec.width) \
                or features.dtype != ACT_DTYPE[self.precision] or not features.is_contiguous():
            raise ValueError(f"features must be contiguous [{self.batch}, {self.res}, {self.spec.width}] "
                             f"{ACT_DTYPE[self.precision]}")
        with D.precision(self.precision):
            st = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream)
            with torch.cuda.stream(st):
                if server.scaled:
                    self.scale_used.copy_(server.scale_state[0:1].view(torch.float32))
                torch.where(self.live, features, self.none, out=self.features)
            self._enqueue_step(server, self.features, stream)

    def _enqueue_step(self, server, features, stream):
        s = stream.cuda_stream if hasattr(stream, "cuda_stream") else stream
        spec, ws, wsb, norm, w = self.spec, self.ws, self.ws.numel(), self.norm_shape, self.spec.width
        wv, pv, gv = spec.addresses(server.w16), spec.addresses(server.w), spec.addresses(self.grad)
        gate = lambda u: u.data_ptr() + w * u.element_size()  # the projection's second half
        # ---- forward
        x, v = features, None
        for j, d in enumerate(self.blocks):
            pre = d["norm"]
            if v is not None and self.dropout:
                D.dbl_dropout_residual(self.drops[j - 1], v, x, self.step, d["s"], s)
                x, v = d["s"], None
            # the stream takes up the layer before (x + v) as the norm reads it
            D.dbl_layer_norm_fwd(norm, x if v is None else v, None if v is None else x, pv(pre + ".g"), pv(pre + ".b"),
                                 None if v is None else d["s"], d["a"], d["mean"], d["istd"], s)
            if v is not None:
                x = d["s"]
            d["x"], v = x, d["v"]
            if d["kind"] == "mix":
                D.dbl_conv_fwd(self.in_shape, d["a"], wv(d["pre"] + ".in.w"), d["u"], None, None, ws, wsb, s)
                D.dbl_gated_scan_fwd(self.scan_shape, d["u"], gate(d["u"]), None, self.lengths, d["h"],
                                     self.h_last[d["layer"]], d["states"], ws, wsb, s)
                D.dbl_conv_fwd(self.out_shape, d["h"], wv(d["pre"] + ".out.w"), v, None, None, ws, wsb, s)
            elif d["kind"] == "experts":
                D.dbl_conv_fwd(self.router_shape, d["a"], wv(d["pre"] + ".router.w"), d["r"], None, None, ws, wsb, s)
                D.dbl_route_fwd(self.route_shape, d["r"], None, self.weight, d["chosen"], d["weights"], d["slots"],
                                d["offsets"], ws, wsb, s)
                D.dbl_expert_scatter(self.exchange_shape, d["a"], d["slots"], d["xg"], s)
                D.dbl_grouped_fwd(self.up_shape, d["xg"], wv(d["pre"] + ".up.w"), d["offsets"], d["hg"], ws, wsb, s)
                D.dbl_grouped_fwd(self.down_shape, d["hg"], wv(d["pre"] + ".down.w"), d["offsets"], d["yg"], ws, wsb, s)
                D.dbl_expert_combine(self.exchange_shape, d["yg"], d["slots"], d["weights"], None, v, s)
        D.dbl_conv_fwd(self.vocab_shape, self.last["a"], wv("vocab.w"), self.logits, None, None, ws, wsb, s)
        # ---- loss; the logits' gradient in their place
        D.dbl_distill_fwd_bwd(self.loss_shape, self.logits, self.teacher_logits, self.teacher_classes, self.labels,
                              self.weight, self.scale_used if server.scaled else None, self.row_loss, self.loss,
                              self.logits, s)
        # ---- backward
        d, ds = self.last, self.ds[0]
        D.dbl_conv_wgrad(self.vocab_shape, d["a"], self.logits, gv("vocab.w"), False, ws, wsb, s)
        D.dbl_conv_dgrad(self.vocab_shape, self.logits, wv("vocab.w"), self.da, ws, wsb, s)
        D.dbl_layer_norm_bwd(norm, self.da, None, d["x"], pv("norm.g"), d["mean"], d["istd"], ds, gv("norm.g"),
                             gv("norm.b"), ws, wsb, s)
        for j in reversed(range(len(self.blocks) - 1)):
            d, dv = self.blocks[j], ds
            pre, du = d["pre"], self.du
            if self.dropout:
                dv = self.dv
                D.dbl_dropout_residual(self.drops[j], ds, None, self.step, dv, s)
            if d["kind"] == "mix":
                D.dbl_conv_wgrad(self.out_shape, d["h"], dv, gv(pre + ".out.w"), False, ws, wsb, s)
                D.dbl_conv_dgrad(self.out_shape, dv, wv(pre + ".out.w"), self.dh, ws, wsb, s)
                D.dbl_gated_scan_bwd(self.scan_shape, self.dh, None, d["u"], gate(d["u"]), d["states"], self.lengths, du,
                                     gate(du), None, ws, wsb, s)
                D.dbl_conv_wgrad(self.in_shape, d["a"], du, gv(pre + ".in.w"), False, ws, wsb, s)
                D.dbl_conv_dgrad(self.in_shape, du, wv(pre + ".in.w"), self.da, ws, wsb, s)
            else:
                # the grouped rows' gradients take the rows' places, but for hg's, which the weights' gradient reads
                D.dbl_expert_combine_bwd(self.exchange_shape, dv, d["yg"], d["slots"], d["weights"], d["yg"], self.dweights, s)
                D.dbl_grouped_wgrad(self.down_shape, d["hg"], d["yg"], d["offsets"], gv(pre + ".down.w"), False, ws, wsb, s)
                D.dbl_grouped_dgrad(self.down_shape, d["yg"], wv(pre + ".down.w"), d["offsets"], d["hg"], self.dhg, ws, wsb, s)
                D.dbl_grouped_wgrad(self.up_shape, d["xg"], self.dhg, d["offsets"], gv(pre + ".up.w"), False, ws, wsb, s)
                D.dbl_grouped_dgrad(self.up_shape, self.dhg, wv(pre + ".up.w"), d["offsets"], None, d["xg"], ws, wsb, s)
                # the router's part of the norm's gradient, then the experts' added to it
                D.dbl_route_bwd(self.route_shape, d["r"], d["chosen"], d["weights"], self.dweights, self.dr, s)
                D.dbl_conv_wgrad(self.router_shape, d["a"], self.dr, gv(pre + ".router.w"), False, ws, wsb, s)
                D.dbl_conv_dgrad(self.router_shape, self.dr, wv(pre + ".router.w"), self.dh, ws, wsb, s)
                D.dbl_expert_combine(self.exchange_shape, d["xg"], d["slots"], None, self.dh, self.da, s)
            # the gradient of the stream past the norm joins the one through it
            out = self.ds[1] if ds is self.ds[0] else self.ds[0]
            D.dbl_layer_norm_bwd(norm, self.da, ds, d["x"], pv(d["norm"] + ".g"), d["mean"], d["istd"], out,
                                 gv(d["norm"] + ".g"), gv(d["norm"] + ".b"), ws, wsb, s)
            ds = out
        if self.dropout:
            D.dbl_dropout_advance(self.step, s)
        self.dfeatures = ds


def demo(iterations=30, precision="bf16", device="cuda", experts=0, dropout=0.0):
    """Dual-batch training of a student on a fixed random teacher over three lengths, shortest first: returns
    the losses (large worker, small worker) of every iteration.  dropout: the rate at the last length, raised
    to in three equal steps."""
    gen = torch.Generator(device=device).manual_seed(0)
    spec, k = TokenSpec(256, 2, 500, experts, 512), 8
    normal = lambda *shape: torch.randn(shape, device=device, generator=gen)
    params = {e.name: (normal(*e.logical) / e.fan_in ** 0.5 if e.fan_in else
                       torch.ones(e.logical, device=device) if e.name.endswith(".g") else
                       torch.zeros(e.logical, device=device)) for e in spec.entries}
    server = ServerState(spec, params, precision=precision, device=device)
    mix = normal(spec.width, spec.classes) / 4.0
    losses = []
    for stage, t in enumerate((64, 96, 128)):
        workers = [TokenWorker(spec, n, t, k, precision=precision, device=device, dropout=dropout * (stage + 1) / 3,
                               seed=2 * stage + i) for i, n in enumerate((16, 4))]
        it = DualBatchIteration(server, *workers, t, lr=0.5, f_small=19.0 / 21.0)
        for _ in range(iterations // 3):
            data = []
            for wk in workers:
                x = normal(wk.batch, t, spec.width).to(ACT_DTYPE[precision])
                top, cls = torch.topk(x.float().reshape(-1, spec.width) @ mix, k)
                wk.set_teacher(top, cls.to(torch.int32))
                data += [x, cls[:, 0].to(torch.int32)]
            it.set_inputs(*data)
            it.run()
            losses.append(tuple(float(wk.loss) for wk in workers))
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description="Trains a small model over tokens by two workers.")
    parser.add_argument("--experts", type=int, default=0, help="experts of the layer behind each mixing layer (0: none)")
    parser.add_argument("--dropout", type=float, default=0.0, help="rate at the last length")
    args = parser.parse_args()
    for i, (large, small) in enumerate(demo(experts=args.experts, dropout=args.dropout)):
        print(f"iteration {i}: loss {large:.4f} (large worker), {small:.4f} (small)")
