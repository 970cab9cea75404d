"""Training step of a small model over tokens, for the scheme's server and workers.

The scheme asks of a model only that a worker turns a batch into its batch-mean gradient (Eq. 1 of
arXiv 2509.26092): the server's merge (Sec. 3.4), the two workers on their streams and the graph
capture are those of ``resnet18.py`` (``ServerState``, ``DualBatchIteration``).  Where cyclic
progressive learning (Sec. 4.1) raises the resolution of images from sub-stage to sub-stage, here it
is the length of the sequences: one ``TokenWorker`` per length, all on the same server.

The model takes features [n, t, width] (the positions of a feature map, or embeddings) and predicts
one of ``classes`` at every token:

    s = features
    for each layer:  s = s + out.w * scan( in.w * norm(s) )      (x and gate: the halves of in.w's output)
    logits = vocab.w * norm(s)

with layer norm, the gated scan and the distillation loss against a teacher's stored top logits
(``dbl_layer_norm_*``, ``dbl_gated_scan_*``, ``dbl_distill_fwd_bwd``) and the products as 1x1
convolutions.  The residual additions run inside the norms, forward and backward.
"""
import torch

from . import dbl as D
from .resnet18 import ACT_DTYPE, DualBatchIteration, FlatSpec, ServerState


class TokenSpec(FlatSpec):
    """Parameters of the model: ``width`` channels (a multiple of 64), ``layers``, ``classes`` (any number;
    stored in rows padded to a multiple of 64, the padding staying zero)."""

    def __init__(self, width=512, layers=2, classes=1000):
        super().__init__()
        if width % 64:
            raise ValueError("width must be a multiple of 64")
        self.width, self.layers, self.classes = width, layers, classes
        self.padded = -(-classes // 64) * 64
        for i in range(layers):
            self._norm(f"layer{i}.norm")
            self.add(f"layer{i}.in.w", (2 * width, width), (2 * width, width), width)
            self.add(f"layer{i}.out.w", (width, width), (width, width), width)
        self._norm("norm")
        self.add("vocab.w", (self.padded, width), (classes, width), width)

    def _norm(self, name):
        self.add(name + ".g", (self.width,), (self.width,), None)
        self.add(name + ".b", (self.width,), (self.width,), None)


class TokenWorker:
    """Activations, gradients and scratch of one worker: ``n`` sequences of ``t`` tokens, a teacher of ``k``
    logits per token.  ``lengths`` ([n] int32, all t at first) ends sequences earlier; tokens past them count
    neither in the loss nor in the states nor, whatever their features hold, in a gradient.  What a step reads
    (teacher, lengths, labels) is set on the current stream, which the next iteration follows."""

    def __init__(self, spec, n, t, k, temperature=2.0, alpha=0.5, device="cuda", eps=1e-5, precision="bf16"):
        self.spec, self.batch, self.res, self.k, self.eps, self.precision = spec, n, t, k, eps, precision
        rows, w = n * t, spec.width
        self.rows = rows
        dt = ACT_DTYPE[precision]

        def act(c):
            return torch.zeros((rows, c), dtype=dt, device=device)

        def vec(m, dtype=torch.float32):
            return torch.zeros(m, dtype=dtype, device=device)

        self.norm_shape = D.ln_shape(rows, w, eps)
        self.scan_shape = D.scan_shape(n, t, w, ld_x=2 * w)  # x and gate are the halves of one projection
        self.loss_shape = D.distill_shape(rows, spec.classes, k, temperature, alpha, ld=spec.padded, ld_grad=spec.padded)
        self.in_shape = D.conv_shape(n, t, 1, w, 2 * w, 1, 1, 0)
        self.out_shape = D.conv_shape(n, t, 1, w, w, 1, 1, 0)
        self.vocab_shape = D.conv_shape(n, t, 1, w, spec.padded, 1, 1, 0)
        chunks = D.dbl_gated_scan_states_bytes(self.scan_shape) // 4
        # per layer: the norm's output, the projection, the scan's output, the layer's; s (but the first) and the
        # norm's statistics; the last entry is the norm before the vocabulary
        self.layers = [dict(a=act(w), u=act(2 * w), h=act(w), v=act(w), states=vec(chunks), mean=vec(rows),
                            istd=vec(rows), s=act(w) if i else None) for i in range(spec.layers)]
        self.last = dict(a=act(w), mean=vec(rows), istd=vec(rows), s=act(w))
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
        need += [D.dbl_conv_workspace_bytes(s, p) for s in (self.in_shape, self.out_shape, self.vocab_shape)
                 for p in (D.DBL_PASS_FWD, D.DBL_PASS_DGRAD, D.DBL_PASS_WGRAD)]
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
        for i, d in enumerate(self.layers + [self.last]):
            pre = f"layer{i}.norm" if d is not self.last else "norm"
            # the stream takes up the layer before (x + v) as the norm reads it
            D.dbl_layer_norm_fwd(norm, x if v is None else v, None if v is None else x, pv(pre + ".g"), pv(pre + ".b"),
                                 None if v is None else d["s"], d["a"], d["mean"], d["istd"], s)
            if v is not None:
                x = d["s"]
            d["x"] = x
            if d is self.last:
                break
            D.dbl_conv_fwd(self.in_shape, d["a"], wv(f"layer{i}.in.w"), d["u"], None, None, ws, wsb, s)
            D.dbl_gated_scan_fwd(self.scan_shape, d["u"], gate(d["u"]), None, self.lengths, d["h"], self.h_last[i],
                                 d["states"], ws, wsb, s)
            D.dbl_conv_fwd(self.out_shape, d["h"], wv(f"layer{i}.out.w"), d["v"], None, None, ws, wsb, s)
            v = d["v"]
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
        for i in reversed(range(spec.layers)):
            d, pre, du = self.layers[i], f"layer{i}", self.du
            D.dbl_conv_wgrad(self.out_shape, d["h"], ds, gv(pre + ".out.w"), False, ws, wsb, s)
            D.dbl_conv_dgrad(self.out_shape, ds, wv(pre + ".out.w"), self.dh, ws, wsb, s)
            D.dbl_gated_scan_bwd(self.scan_shape, self.dh, None, d["u"], gate(d["u"]), d["states"], self.lengths, du,
                                 gate(du), None, ws, wsb, s)
            D.dbl_conv_wgrad(self.in_shape, d["a"], du, gv(pre + ".in.w"), False, ws, wsb, s)
            D.dbl_conv_dgrad(self.in_shape, du, wv(pre + ".in.w"), self.da, ws, wsb, s)
            # the gradient of the stream past the norm joins the one through it
            out = self.ds[1] if ds is self.ds[0] else self.ds[0]
            D.dbl_layer_norm_bwd(norm, self.da, ds, d["x"], pv(pre + ".norm.g"), d["mean"], d["istd"], out,
                                 gv(pre + ".norm.g"), gv(pre + ".norm.b"), ws, wsb, s)
            ds = out
        self.dfeatures = ds


def demo(iterations=30, precision="bf16", device="cuda"):
    """Dual-batch training of a student on a fixed random teacher over three lengths, shortest first: returns
    the losses (large worker, small worker) of every iteration."""
    gen = torch.Generator(device=device).manual_seed(0)
    spec, k = TokenSpec(256, 2, 500), 8
    normal = lambda *shape: torch.randn(shape, device=device, generator=gen)
    params = {e.name: (normal(*e.logical) / e.fan_in ** 0.5 if e.fan_in else
                       torch.ones(e.logical, device=device) if e.name.endswith(".g") else
                       torch.zeros(e.logical, device=device)) for e in spec.entries}
    server = ServerState(spec, params, precision=precision, device=device)
    mix = normal(spec.width, spec.classes) / 4.0
    losses = []
    for t in (64, 96, 128):
        workers = [TokenWorker(spec, n, t, k, precision=precision, device=device) for n in (16, 4)]
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
    for i, (large, small) in enumerate(demo()):
        print(f"iteration {i}: loss {large:.4f} (large worker), {small:.4f} (small)")
