"""Both ends of a sequence model over a vocabulary, as cases that can be timed and checked.

  embed      rows of a table by token number; `mode` "fwd" (lookup with a scale) or "bwd" (the table's
             gradient, summed over the tokens that name a row)
  loss       softmax cross entropy of x w^T against a label per row; `mode` "fwd" (loss and the
             log of the sum) or "train" (the loss and the gradients of x and w)
  distill    the same against a teacher's k largest logits of each row

Sizes are generic; channel counts are those of this repository's sequence cases where one fits.

The plain forms are elementary torch operations in 32 bits.  Definitions:

  embed      y[r] = scale * table[ids[r]], 0 for an id outside the table;
             dtable[j] = (what is there, where `tied`) + scale / S * sum of dy[r] over ids[r] = j
  loss       z[r][j] = logit_scale * <x[r], w[j]>, lse = log sum_j exp z; loss = lse - z[target];
             a row whose target is outside the vocabulary has loss, lse and gradients 0;
             dz = G (softmax(z) - onehot), dx = logit_scale * dz w, dw = logit_scale / S * dz^T x,
             with G = S / (rows that count), as a program takes the mean and scales it
  distill    q = softmax over the row's k entries of logit_scale * teacher, entries whose target is outside
             the vocabulary left out; loss = sum q (log q + lse - z[target]), dz = G (softmax(z) - q)
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
LOSS_SCALE = 1024.0
DY_STD = 1e-3


def listed():
    return [
        # a serving step of 8 sequences: one token each, the latency of one launch
        dict(name="embed-token", op="embed", mode="fwd", rows=8, c=2048, v=65536, dtype="bf16", out="bf16", pad=0.0, tied=False),
        # the prompts of a batch
        dict(name="embed-prompt", op="embed", mode="fwd", rows=16384, c=4096, v=65536, dtype="bf16", out="bf16", pad=0.0, tied=False),
        # an ordinary training batch: few tokens make up most of a text
        dict(name="embed-train", op="embed", mode="bwd", rows=32768, c=1152, v=32768, dtype="f16", out="f32", pad=0.0, tied=False),
        # a padded batch of odd sizes, added to the gradient of a head that shares the table
        dict(name="embed-tied-odd", op="embed", mode="bwd", rows=5003, c=771, v=10007, dtype="bf16", out="bf16", pad=0.3, tied=True),
        # scoring one token of each of 16 sequences: bound by the read of the head's weights
        dict(name="loss-score", op="loss", mode="fwd", rows=16, c=2048, v=65536, dtype="bf16", pad=0.0, scale=1.0),
        # evaluation of a batch
        dict(name="loss-eval", op="loss", mode="fwd", rows=4096, c=1152, v=32768, dtype="f16", pad=0.0, scale=1.0),
        # a small model's step: latency of the chain counts
        dict(name="loss-small-train", op="loss", mode="train", rows=512, c=512, v=8192, dtype="bf16", pad=0.0, scale=1.0),
        # the largest step
        dict(name="loss-train", op="loss", mode="train", rows=8192, c=2048, v=65536, dtype="bf16", pad=0.0, scale=1.0),
        # a padded batch of odd sizes
        dict(name="loss-odd-train", op="loss", mode="train", rows=1999, c=515, v=12345, dtype="f16", pad=0.2, scale=0.5),
        # how far a student is from its teacher
        dict(name="distill-eval", op="distill", mode="fwd", rows=2048, c=768, v=16384, dtype="f16", pad=0.0, scale=1.0, k=16, teacher="f32"),
        # a student's step
        dict(name="distill-train", op="distill", mode="train", rows=4096, c=1152, v=32768, dtype="bf16", pad=0.0, scale=0.5, k=32, teacher="bf16"),
        # a padded batch of odd sizes
        dict(name="distill-odd-train", op="distill", mode="train", rows=777, c=331, v=5003, dtype="f16", pad=0.2, scale=1.0, k=7, teacher="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _channels(rng, hi):
    """A channel count, six in ten of them multiples of 8."""
    c = _log(rng, 8, hi)
    return max(8, c // 8 * 8) if rng.random() < 0.6 else c


def draw(rng):
    op = rng.choice(["embed", "loss", "loss", "distill"])
    dtype = rng.choice(["f16", "bf16"])
    pad = rng.choice([0.0, 0.0, 0.1, 0.6])
    if op == "embed":
        c = _channels(rng, 4096)
        v = _log(rng, 100, min(131072, 134e6 // c))
        rows = _log(rng, 1, min(65536, 67e6 // c))
        mode = rng.choice(["fwd", "bwd"])
        out = dtype if mode == "fwd" else rng.choice([dtype, "f32"])
        return dict(op=op, mode=mode, rows=rows, c=c, v=v, dtype=dtype, out=out, pad=pad, tied=mode == "bwd" and rng.random() < 0.4)
    c = _channels(rng, 4096)
    v = _log(rng, 64, min(131072, 134e6 // c))
    rows = _log(rng, 1, min(8192, 536e6 // v, 1.0e12 // (v * c)))
    case = dict(op=op, mode=rng.choice(["fwd", "train", "train"]), rows=rows, c=c, v=v, dtype=dtype, pad=pad, scale=rng.choice([1.0, 0.5, 0.25]))
    return dict(case, k=_log(rng, 1, min(64, v)), teacher=rng.choice(["f32", dtype])) if op == "distill" else case


# --- what a program has in hand ---------------------------------------------------------


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, shape, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale)


def _rand(g, shape):
    return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)


def _tokens(g, rows, v, pad):
    """Tokens as texts have them: number j about as often as 1 / (j + 2), and -1 for padding."""
    ids = (2.0 * torch.exp(_rand(g, (rows,)) * math.log((v + 2.0) / 2.0)) - 2.0).to(torch.int32).clamp(0, v - 1)
    return torch.where(_rand(g, (rows,)) < pad, -1, ids)


def _embed_inputs(case, seed):
    g, t = _generator(seed), DTYPES[case["dtype"]]
    rows, c, v = case["rows"], case["c"], case["v"]
    s = {"ids": _tokens(g, rows, v, case["pad"]), "scale": math.sqrt(c)}
    if case["mode"] == "fwd":
        s["table"] = _randn(g, (v, c), c ** -0.5).to(t)
    else:
        s["dy"] = _randn(g, (rows, c), LOSS_SCALE * DY_STD).to(t)
        if case["tied"]:
            s["dtable"] = _randn(g, (v, c), 0.1).to(DTYPES[case["out"]])
    return s


def _loss_inputs(case, seed):
    g, t = _generator(seed), DTYPES[case["dtype"]]
    rows, c, v = case["rows"], case["c"], case["v"]
    s = {"w": _randn(g, (v, c), 1.5 * c ** -0.5).to(t)}
    label = _tokens(g, rows, v, case["pad"])
    x = _randn(g, (rows, c))
    # some rows are sure of their label, others have never seen it
    row = s["w"][label.clamp(min=0).long()].float()
    lift = 18.0 * _rand(g, (rows, 1)) * (_rand(g, (rows, 1)) < 0.8)
    s["x"] = x.add_(row * (lift / row.square().sum(1, keepdim=True).clamp(min=1e-3))).to(t)
    if case["op"] == "loss":
        s["target"] = label
    else:
        k = case["k"]  # distinct tokens, the label in front
        step = 1 + (_rand(g, (rows, 1)) * (v // k - 1)).long() if v // k > 1 else torch.ones((rows, 1), dtype=torch.int64, device="cuda")
        at = torch.arange(k, device="cuda") * step
        s["target"] = torch.where(label[:, None] < 0, -1, (label[:, None].clamp(min=0).long() + at) % v).to(torch.int32)
        s["teacher"] = (9.0 - 1.5 * torch.log1p(torch.arange(k, device="cuda").float()) + _randn(g, (rows, k), 0.4)).to(DTYPES[case["teacher"]])
    count = (label >= 0).sum().clamp(min=1)
    s["grad_scale"] = (LOSS_SCALE / count).float().view(1)
    return s


def prepare(case, seed):
    """The inputs, the arrays that outputs go to, and for the framework's calls the object that holds sizes and workspaces."""
    t = DTYPES[case["dtype"]]
    rows, c, v = case["rows"], case["c"], case["v"]
    if case["op"] == "embed":
        s = _embed_inputs(case, seed)
        if case["mode"] == "fwd":
            s["y"] = torch.empty((rows, c), dtype=t, device="cuda")
        else:
            s.setdefault("dtable", torch.empty((v, c), dtype=DTYPES[case["out"]], device="cuda"))
    else:
        s = _loss_inputs(case, seed)
        s["loss"], s["lse"] = (torch.empty(rows, dtype=torch.float32, device="cuda") for _ in range(2))
        if case["mode"] == "train":
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
    s["case"] = case
    if own:
        s["op"] = _framework_object(case, s)
    return s


def _framework_object(case, s):
    from paper_2102_06725_amd import nnconv as nc
    code = {"f16": nc.NNCONV_F16, "bf16": nc.NNCONV_BF16, "f32": nc.NNCONV_F32}
    sizes = (case["rows"], case["c"], case["v"])
    if case["op"] == "embed":
        return nc.Embedding(*sizes, dtype=code[case["dtype"]], scale=s["scale"])
    if case["op"] == "loss":
        return nc.CrossEntropy(*sizes, dtype=code[case["dtype"]], logit_scale=case["scale"])
    return nc.CrossEntropy(*sizes, dtype=code[case["dtype"]], logit_scale=case["scale"], k=case["k"], teacher_dtype=code[case["teacher"]])


# --- a pass -------------------------------------------------------------------------


def run(state):
    return _run_embed(state) if state["case"]["op"] == "embed" else _run_loss(state)


def _run_embed(s):
    case, ids = s["case"], s["ids"]
    forward = case["mode"] == "fwd"
    if own:
        if forward:
            s["op"].fwd(ids, s["table"], s["y"])
            return {"y": s["y"]}
        s["op"].bwd(ids, s["dy"], s["dtable"], inv_loss_scale=1.0 / LOSS_SCALE, accumulate=int(case["tied"]))
        return {"dtable": s["dtable"]}
    live = (ids >= 0) & (ids < case["v"])
    at = torch.where(live, ids, 0).long()
    if forward:
        y = torch.where(live[:, None], s["table"][at].float() * s["scale"], 0.0)
        return {"y": y.to(s["table"].dtype)}
    rows = torch.where(live[:, None], s["dy"].float() * (s["scale"] / LOSS_SCALE), 0.0)
    total = torch.zeros((case["v"], case["c"]), dtype=torch.float32, device="cuda").index_add_(0, at, rows)
    if case["tied"]:
        total += s["dtable"].float()
    s["dtable"].copy_(total)
    return {"dtable": s["dtable"]}


def _run_loss(s):
    case, train = s["case"], s["case"]["mode"] == "train"
    if own:
        if train:
            s["op"].train(s["x"], s["w"], s["target"], s["loss"], s["dx"], s["dw"], lse=s["lse"], teacher=s.get("teacher"),
                          grad_scale=s["grad_scale"], inv_loss_scale=1.0 / LOSS_SCALE)
        else:
            s["op"].fwd(s["x"], s["w"], s["target"], s["loss"], lse=s["lse"], teacher=s.get("teacher"))
        return {k: s[k] for k in (("loss", "lse", "dx", "dw") if train else ("loss", "lse"))}
    target = s["target"].view(case["rows"], -1)
    live = (target >= 0) & (target < case["v"])
    counts = live.any(1)
    at = torch.where(live, target, 0).long()
    x = torch.where(counts[:, None], s["x"].float(), 0.0)
    w = s["w"].float()
    z = (x @ w.t()).mul_(case["scale"])
    top = z.amax(1)
    p = torch.exp(z - top[:, None])
    total = p.sum(1)
    lse = top + torch.log(total)
    if case["op"] == "loss":
        q, log_q = live.float(), torch.zeros_like(target, dtype=torch.float32)
    else:
        a = torch.where(live, s["teacher"].float() * case["scale"], -torch.inf)
        a = a - torch.where(counts, a.amax(1), 0.0)[:, None]
        e = torch.exp(a)
        q = e / e.sum(1, keepdim=True).clamp(min=1e-30)
        log_q = torch.where(q > 0, a - torch.log(e.sum(1, keepdim=True).clamp(min=1e-30)), 0.0)
    loss = torch.where(q > 0, q * (log_q + lse[:, None] - z.gather(1, at)), 0.0).sum(1)
    out = {"loss": loss, "lse": torch.where(counts, lse, 0.0)}
    if not train:
        return out
    p = p.mul_((counts / total)[:, None]).scatter_add_(1, at, torch.where(live, -q, 0.0))
    p = p.mul_(s["grad_scale"] * case["scale"])
    out["dx"] = (p @ w).to(s["x"].dtype)
    out["dw"] = ((p.t() @ x) / LOSS_SCALE).to(s["w"].dtype)
    return out


# --- work ------------------------------------------------------------------------------


def work(case):
    rows, c, v = case["rows"], case["c"], case["v"]
    if case["op"] == "embed":
        if case["mode"] == "fwd":
            return {"bytes": 4 * rows + 4 * rows * c, "flops": rows * c}
        size = 4 if case["out"] == "f32" else 2
        # added to what is there only the rows that tokens name are read and written
        table = 2 * min(v, rows) * c * size if case["tied"] else v * c * size
        return {"bytes": 4 * rows + 2 * rows * c + table, "flops": rows * c}
    k = case.get("k", 1)
    io = 2 * c * (rows + v) + rows * (4 * k + 8)
    if case["op"] == "distill":
        io += rows * k * (4 if case["teacher"] == "f32" else 2)
    if case["mode"] == "fwd":
        return {"bytes": io, "flops": 2 * rows * v * c}
    return {"bytes": io + 2 * c * (rows + v), "flops": 6 * rows * v * c}


# --- in 64 bits ----------------------------------------------------------------------------


def exact(case, seed):
    return _exact_embed(case, seed) if case["op"] == "embed" else _exact_loss(case, seed)


def _exact_embed(case, seed):
    s = _embed_inputs(case, seed)
    ids, c, v = s["ids"].long(), case["c"], case["v"]
    kept = torch.nonzero(ids >= 0).view(-1)
    if case["mode"] == "fwd":
        y = torch.zeros((case["rows"], c), dtype=torch.float64, device="cuda")
        y[kept] = s["scale"] * s["table"][ids[kept]].double()
        return {"y": y}
    # sums of runs of equal tokens, as differences of running sums
    order = kept[torch.argsort(ids[kept], stable=True)]
    n = torch.bincount(ids[kept], minlength=v)
    out = torch.empty((v, c), dtype=torch.float64, device="cuda")
    for at in range(0, c, 256):
        run_sum = torch.cumsum(s["dy"][:, at:at + 256][order].double(), 0)
        run_sum = torch.cat([torch.zeros_like(s["dy"][:1, at:at + 256], dtype=torch.float64), run_sum])
        end = torch.cumsum(n, 0)
        out[:, at:at + 256] = run_sum[end] - run_sum[end - n]
    out *= s["scale"] / LOSS_SCALE
    return {"dtable": out + s["dtable"].double() if case["tied"] else out}


def _exact_loss(case, seed):
    s = _loss_inputs(case, seed)
    rows, v, scale = case["rows"], case["v"], case["scale"]
    w, target = s["w"].double(), s["target"].view(rows, -1).long()
    train = case["mode"] == "train"
    loss, lse = (torch.zeros(rows, dtype=torch.float64, device="cuda") for _ in range(2))
    dx = torch.zeros((rows, case["c"]), dtype=torch.float64, device="cuda")
    dw = torch.zeros_like(w)
    step = max(1, min(rows, int(2e8) // v))
    for at in range(0, rows, step):
        kept = at + torch.nonzero(target[at:at + step, 0] >= 0).view(-1)  # a row's targets are all there, or none
        if not len(kept):
            continue
        x, t = s["x"][kept].double(), target[kept]
        z = x @ w.t() * scale
        lse[kept] = torch.logsumexp(z, 1)
        if case["op"] == "loss":
            q = torch.ones_like(t, dtype=torch.float64)
            loss[kept] = lse[kept] - z[torch.arange(len(kept), device="cuda"), t[:, 0]]
        else:
            log_q = torch.log_softmax(s["teacher"][kept].double() * scale, 1)
            q = log_q.exp()
            loss[kept] = (q * (log_q - torch.gather(z - lse[kept, None], 1, t))).sum(1)
        if train:
            dz = torch.exp(z - lse[kept, None])
            dz[torch.arange(len(kept), device="cuda")[:, None], t] -= q
            dz *= s["grad_scale"].double() * scale
            dx[kept] = dz @ w
            dw += dz.t() @ x
    out = {"loss": loss, "lse": lse}
    return dict(out, dx=dx, dw=dw / LOSS_SCALE) if train else out
