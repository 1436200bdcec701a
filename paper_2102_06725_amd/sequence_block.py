"""A small gated sequence model on channel-last tokens, trained and served with libnnconv.

Each block is a pre-norm residual block:

    r = x + r;  u = norm(r);  p = projection to 3c of u;  y = gated recurrence of p's
    thirds (value, forget gate, output gate);  x = projection back to c of y

with 1x1 convolutions over NHWC images of height 1 and width t as the projections, and a last norm and
projection behind the blocks.  `SequenceModel` keeps fp32 masters, 16-bit working weights, gradients and
moments in flat arrays.  A training step is loss-scaled and stays on the device: forward, backward, AdamW
(8-bit moments for the matrices, 32-bit ones for gains and biases), the loss scaler's step.  It
queues kernels only, so it can be captured into a graph.  `Server` runs one token of every
sequence at a time, with the recurrence's states updated in place.

    python -m paper_2102_06725_amd.sequence_block      # trains on a leaky sum of its input, then serves
"""
from __future__ import annotations

import math

from . import nnconv as nc

ALIGN = 64  # elements: tensors of the flat arrays start at a block of 8-bit moments


class SequenceModel:
    """c_in input channels, `blocks` blocks of c channels, c_out outputs; channel counts in multiples of 8."""

    def __init__(self, n, t, c_in, c, c_out, blocks, dtype=nc.NNCONV_BF16, seed=0, loss_scale=1024.0, weight_decay=0.01,
                 device="cuda"):
        import torch
        self.n, self.t, self.c_in, self.c, self.c_out, self.blocks = n, t, c_in, c, c_out, blocks
        self.code, self.device = dtype, device
        self.dtype = torch.float16 if dtype == nc.NNCONV_F16 else torch.bfloat16
        self.layout = [("embed", (c, 1, 1, c_in), weight_decay)]
        for b in range(blocks):
            self.layout += [("gain%d" % b, (c,), 0.0), ("in%d" % b, (3 * c, 1, 1, c), weight_decay),
                            ("bias%d" % b, (c,), 0.0), ("out%d" % b, (c, 1, 1, c), weight_decay)]
        self.layout += [("gain", (c,), 0.0), ("head", (c_out, 1, 1, c), weight_decay)]
        self._parameters(torch.Generator().manual_seed(seed))
        self.scaler = torch.zeros(6, dtype=torch.int32, device=device)
        nc.check(nc.nnconv_loss_scaler_init(self.scaler.data_ptr(), loss_scale, 2.0, 2000, nc.current_stream()))
        self.loss_scale = self.scaler[:1].view(torch.float32)  # read on the device
        self.flag = torch.zeros(1, dtype=torch.int32, device=device)
        self.step_count = torch.zeros(1, dtype=torch.int32, device=device)

        conv = lambda k, cc: nc.Conv2d(n, cc, 1, t, k, 1, 1, layout=nc.NNCONV_NHWC, dtype=dtype)  # noqa: E731
        self.embed, self.head = conv(c, c_in), conv(c_out, c)
        self.into, self.back = [conv(3 * c, c) for _ in range(blocks)], [conv(c, c) for _ in range(blocks)]
        self.norm = nc.RMSNorm(n * t, c, dtype=dtype)
        self.rec = nc.GatedRecurrence(n, t, c, ld=3 * c, dtype=dtype)
        new = lambda k: torch.empty((n, t, k), dtype=self.dtype, device=device)  # noqa: E731
        f32 = lambda *s: torch.empty(s, dtype=torch.float32, device=device)  # noqa: E731
        # activations that the backward pass reads, one set a block
        self.acts = [dict(r=new(c), u=new(c), rstd=f32(n * t), p=new(3 * c), y=new(c), x=new(c), saved=self.rec.saved(device))
                     for _ in range(blocks)]
        self.x0, self.r, self.u, self.rstd, self.out = new(c), new(c), new(c), f32(n * t), new(c_out)
        self.grad = dict(out=new(c_out), u=new(c), r=new(c), y=new(c), p=new(3 * c))

    def _parameters(self, g):
        import torch
        starts, total = {}, 0
        for name, shape, _ in self.layout:
            starts[name] = total
            total += -(-math.prod(shape) // ALIGN) * ALIGN
        flat = {k: torch.zeros(total, dtype=d, device=self.device) for k, d in
                (("master", torch.float32), ("grad", torch.float32), ("w16", self.dtype), ("m", torch.float32), ("v", torch.float32),
                 ("m8", torch.uint8), ("v8", torch.uint8))}
        flat.update({k: torch.zeros(total // ALIGN, dtype=torch.uint8, device=self.device) for k in ("m_scale", "v_scale")})
        self.flat, tensors = flat, []

        def part(key, name, shape):
            return flat[key][starts[name]:starts[name] + math.prod(shape)].view(shape)

        self.master, self.w16, self.dw = {}, {}, {}
        for name, shape, decay in self.layout:
            m = self.master[name] = part("master", name, shape)
            self.dw[name] = part("grad", name, shape)
            if name.startswith("gain"):
                m.fill_(1.0)
            elif name.startswith("bias"):  # memories from 2 to about 150 tokens
                m.copy_(torch.linspace(0.0, 5.0, shape[0]))
            else:
                m.copy_(torch.randn(shape, generator=g) / math.sqrt(shape[-1]))
            entry = dict(master=m, grad=self.dw[name], weight_decay=decay)
            if len(shape) == 4:
                w = self.w16[name] = part("w16", name, shape)
                w.copy_(m)
                blocks = slice(starts[name] // ALIGN, -(-(starts[name] + m.numel()) // ALIGN))
                entry.update(w16=w, m=part("m8", name, shape), v=part("v8", name, shape), m_scale=flat["m_scale"][blocks],
                             v_scale=flat["v_scale"][blocks])
            else:
                entry.update(m=part("m", name, shape), v=part("v", name, shape))
            tensors.append(entry)
        self.solver = nc.AdamW(tensors, seed=1)

    def forward(self, x):
        """Outputs [n][t][c_out] of inputs [n][t][c_in]."""
        c = self.c
        self.embed.fwd(x, self.w16["embed"], self.x0)
        h, r = self.x0, None
        for b, a in enumerate(self.acts):
            self.norm.fwd(h, self.master["gain%d" % b], a["u"], residual=r, sum=a["r"], rstd=a["rstd"])
            self.into[b].fwd(a["u"], self.w16["in%d" % b], a["p"])
            v, f, g = (a["p"][..., i * c:(i + 1) * c] for i in range(3))
            self.rec.fwd(v, f, self.master["bias%d" % b], a["y"], g=g, saved=a["saved"])
            self.back[b].fwd(a["y"], self.w16["out%d" % b], a["x"])
            h, r = a["x"], a["r"]
        self.norm.fwd(h, self.master["gain"], self.u, residual=r, sum=self.r, rstd=self.rstd)
        self.head.fwd(self.u, self.w16["head"], self.out)
        return self.out

    def backward(self, x, dout):
        """Parameter gradients, loss-scaled as dout is, into the flat gradient array."""
        c, d, flag = self.c, self.grad, self.flag

        def weights(conv, inp, dy, name):
            conv.wgrad(inp, dy, self.dw[name], overflow_flag=flag)

        weights(self.head, self.u, dout, "head")
        self.head.dgrad(dout, self.w16["head"], d["u"])
        self.norm.bwd(self.r, d["u"], self.master["gain"], self.rstd, d["r"], dgain=self.dw["gain"], overflow_flag=flag)
        for b in range(self.blocks - 1, -1, -1):
            a = self.acts[b]
            weights(self.back[b], a["y"], d["r"], "out%d" % b)
            self.back[b].dgrad(d["r"], self.w16["out%d" % b], d["y"])
            v, f, g = (a["p"][..., i * c:(i + 1) * c] for i in range(3))
            dv, df, dg = (d["p"][..., i * c:(i + 1) * c] for i in range(3))
            self.rec.bwd(v, f, self.master["bias%d" % b], a["saved"], d["y"], dv, df, g=g, dg=dg, dbias=self.dw["bias%d" % b],
                         overflow_flag=flag)
            weights(self.into[b], a["u"], d["p"], "in%d" % b)
            self.into[b].dgrad(d["p"], self.w16["in%d" % b], d["u"])
            # the stream's own gradient joins in place
            self.norm.bwd(a["r"], d["u"], self.master["gain%d" % b], a["rstd"], d["r"], dgain=self.dw["gain%d" % b], dsum=d["r"],
                          overflow_flag=flag)
        weights(self.embed, x, d["r"], "embed")

    def train_step(self, x, target, lr, beta1=0.9, beta2=0.99):
        """One step on the mean squared error; returns the loss as a device scalar."""
        err = self.forward(x).float() - target
        self.grad["out"].copy_(err * (2.0 / err.numel()) * self.loss_scale)
        self.backward(x, self.grad["out"])
        self.solver.step(self.step_count, lr, beta1, beta2, state=self.scaler, overflow_flag=self.flag)
        nc.check(nc.nnconv_loss_scaler_update(self.scaler.data_ptr(), self.flag.data_ptr(), nc.current_stream()))
        return (err * err).mean()

    def features_q8(self, group=128):
        """The last forward's features (the last norm's output) in 8 bits: (codes, scales)."""
        import torch
        norm = nc.RMSNorm(self.n * self.t, self.c, dtype=self.code, group=group)
        q = torch.empty((self.n, self.t, self.c), dtype=torch.float8_e4m3fn, device=self.device)
        scales = torch.empty((self.n, self.t, -(-self.c // group)), dtype=torch.float32, device=self.device)
        norm.fwd_q8(self.r, self.master["gain"], q, scales)
        return q, scales


class Server:
    """One token of each of `n` sequences a call, from the model's present weights."""

    def __init__(self, model, n):
        import torch
        self.model, c = model, model.c
        conv = lambda k, cc: nc.Conv2d(n, cc, 1, 1, k, 1, 1, layout=nc.NNCONV_NHWC, dtype=model.code)  # noqa: E731
        self.embed, self.into, self.back, self.head = conv(c, model.c_in), conv(3 * c, c), conv(c, c), conv(model.c_out, c)
        self.norm = nc.RMSNorm(n, c, dtype=model.code)
        self.rec = nc.GatedRecurrence(n, 1, c, ld=3 * c, dtype=model.code)
        new = lambda k: torch.empty((n, k), dtype=model.dtype, device=model.device)  # noqa: E731
        self.h, self.r, self.u, self.p, self.y, self.out = new(c), new(c), new(c), new(3 * c), new(c), new(model.c_out)
        self.states = torch.zeros((model.blocks, n, c), dtype=torch.float32, device=model.device)

    def reset(self):
        self.states.zero_()

    def step(self, x):
        """Outputs [n][c_out] of one token [n][c_in] of each sequence; the states go on."""
        m, c = self.model, self.model.c
        self.embed.fwd(x, m.w16["embed"], self.h)
        r = None
        for b in range(m.blocks):
            self.norm.fwd(self.h, m.master["gain%d" % b], self.u, residual=r, sum=self.r)
            r = self.r  # from the second block on the stream is added to in place
            self.into.fwd(self.u, m.w16["in%d" % b], self.p)
            v, f, g = (self.p[:, i * c:(i + 1) * c] for i in range(3))
            self.rec.fwd(v, f, m.master["bias%d" % b], self.y, g=g, h0=self.states[b], ht=self.states[b])
            self.back.fwd(self.y, m.w16["out%d" % b], self.h)
        self.norm.fwd(self.h, m.master["gain"], self.u, residual=r, sum=self.r)
        self.head.fwd(self.u, m.w16["head"], self.out)
        return self.out


def leaky_sums(n, t, c_in, c_out, seed, device="cuda"):
    """Inputs, and targets that need a memory: sums of inputs that leak at a rate per output channel."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, t, c_in), generator=g)
    rate = torch.linspace(0.5, 0.95, c_out)
    y, s = torch.empty((n, t, c_out)), torch.zeros((n, c_out))
    for k in range(t):
        s = rate * s + (1.0 - rate ** 2).sqrt() * x[:, k, :1]
        y[:, k] = s
    return x.to(device), y.to(device)


def main(steps=200):
    import torch
    n, t, c_in, c, c_out = 16, 256, 8, 128, 16
    model = SequenceModel(n, t, c_in, c, c_out, blocks=2)
    for k in range(steps):
        x, y = leaky_sums(n, t, c_in, c_out, seed=k)
        loss = model.train_step(x.to(model.dtype), y, lr=2e-3)
        if k % 20 == 0 or k == steps - 1:
            print("step %3d  loss %.4f" % (k, float(loss)), flush=True)
    whole = model.forward(x.to(model.dtype)).float()
    server = Server(model, n)
    served = torch.stack([server.step(x[:, k].to(model.dtype).contiguous()).float().clone() for k in range(t)], dim=1)
    print("token by token: largest difference from the whole pass %.4f of %.4f" % (float((served - whole).abs().max()), float(whole.abs().max())))
    q, scales = model.features_q8()
    print("8-bit features: %d bytes of codes, %d of scales" % (q.numel(), scales.numel() * 4))


if __name__ == "__main__":
    main()
