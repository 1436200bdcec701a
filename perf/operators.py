"""The operators of a gated sequence block and its training step, as cases that can be timed and checked.

  norm       root-mean-square norm over the channels of channel-last rows, with the residual's
             addition; `mode` "fwd" (y and the stored sum), "q8" (an 8-bit output with a scale per
             row or per `group` channels) or "train" (forward and backward)
  recur      the gated linear recurrence over the tokens of each sequence, on the packed output
             [n][t][3c] of one projection (value, forget gate, output gate); `mode` "fwd" or "train"
  adamw      one AdamW step over many tensors, moments in 32 bits or in 8

Sizes are those of this repository's own layers (`paper_2102_06725_amd/inputs.py`) or generic.

The plain forms are elementary torch operations in 32 bits.  Definitions:

  norm       r = round16(x + residual) is the stored residual stream (x itself without one),
             rstd = 1 / sqrt(mean(r^2) + eps), y = gain * r * rstd; in 8 bits q = e4m3(y / s) with
             s = max|y| / 448 over the row or the group.
             dx = dsum + rstd * (dy * gain - xh * mean(dy * gain * xh)) with xh = r * rstd;
             dgain = inv_loss_scale * sum over rows of dy * xh
  recur      z = clamp(f + bias, -80, 80), a = sigmoid(z), h_t = a_t h_(t-1) + (1 - a_t) x_t,
             y_t = h_t * g_t * sigmoid(g_t); tokens from a sequence's length on leave h as it is
             and have y = 0
  adamw      g = grad / S, m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2,
             w -= lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay w).
             8-bit moments are e4m3 (m) and e5m2 (v) codes times a power of two per 64 elements;
             codes are rounded at random, by a hash of (seed, step, tensor, element), so that
             changes far below a code's spacing survive on average, and a v above 0 stays above 0
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
LOSS_SCALE = 1024.0
DY_STD = 1e-3
EPS_NORM = 1e-6
GATE_LIMIT = 80.0
F8_MAX = 448.0
f32 = lambda v: float(np.float32(v))  # noqa: E731  what a C float holds
LR, BETA1, BETA2, EPS, DECAY = f32(1e-3), f32(0.9), f32(0.999), f32(1e-8), f32(0.1)
STEPS_DONE = 1000  # steps before the one that is measured
SEED8 = 20240229
BLOCK = 64  # elements with one scale


def listed():
    return [
        # a serving step of 8 sequences: one token each, the latency of one launch
        dict(name="norm-token", op="norm", mode="fwd", rows=8, c=2048, dtype="bf16", residual=True, group=0),
        # a prefill of 16 Ki tokens in front of an 8-bit product, a scale per 128 channels
        dict(name="norm-q8", op="norm", mode="q8", rows=16384, c=4096, dtype="bf16", residual=True, group=128),
        # the pixels of a 56x56 stage with 256 channels, batch 64, in training
        dict(name="norm-pixels-train", op="norm", mode="train", rows=64 * 56 * 56, c=256, dtype="f16", residual=True, group=0),
        # an odd channel count: rows start at every alignment
        dict(name="norm-odd-train", op="norm", mode="train", rows=12345, c=771, dtype="bf16", residual=True, group=0),
        # a serving step of 64 sequences: one token each, the state updated in place
        dict(name="recur-token", op="recur", mode="fwd", n=64, t=1, c=1152, dtype="bf16", ragged=False, carry=True),
        # an ordinary training batch
        dict(name="recur-train", op="recur", mode="train", n=8, t=2048, c=1152, dtype="bf16", ragged=False, carry=False),
        # two long sequences: the work has to be split over the tokens
        dict(name="recur-long", op="recur", mode="fwd", n=2, t=32768, c=768, dtype="f16", ragged=False, carry=True),
        # sequences of 0, 1 and more tokens, an odd channel count, with carried states
        dict(name="recur-ragged-train", op="recur", mode="train", n=6, t=1501, c=331, dtype="f16", ragged=True, carry=True),
        # the tensors of one small block
        dict(name="adamw-block", op="adamw", set="block", width=256, blocks=1, bits=32, dtype="bf16"),
        # all convolution weights of ResNet-50, with norm gains
        dict(name="adamw-resnet50", op="adamw", set="resnet50", width=0, blocks=0, bits=32, dtype="f16"),
        # a stack of wide blocks with 8-bit moments: the largest update
        dict(name="adamw8-stack", op="adamw", set="block", width=2048, blocks=6, bits=8, dtype="bf16"),
        # many tensors of odd sizes, 8-bit moments
        dict(name="adamw8-odd", op="adamw", set="odd", width=777, blocks=40, bits=8, dtype="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _channels(rng, hi):
    """A channel count, six in ten of them multiples of 8."""
    c = _log(rng, 8, hi)
    c = max(8, c // 8 * 8) if rng.random() < 0.6 else c
    return c + 8 if c in (1024, 3072) else c


def draw(rng):
    op = rng.choice(["norm", "recur", "adamw"])
    dtype = rng.choice(["f16", "bf16"])
    if op == "norm":
        c = _channels(rng, 8192)
        rows = _log(rng, 1, min(400000, 67e6 // c))
        mode = rng.choice(["fwd", "q8", "train"])
        return dict(op=op, mode=mode, rows=rows, c=c, dtype=dtype, residual=rng.random() < 0.7,
                    group=rng.choice([0, 32, 64, 128]) if mode == "q8" else 0)
    if op == "recur":
        c = _channels(rng, 2048)
        t = _log(rng, 1, 65536)
        n = _log(rng, 1, max(1, min(64, 16e6 // (c * t))))
        return dict(op=op, mode=rng.choice(["fwd", "train"]), n=n, t=min(t, int(16e6 // c)), c=c, dtype=dtype,
                    ragged=rng.random() < 0.5, carry=rng.random() < 0.5)
    if rng.random() < 0.5:
        return dict(op=op, set="odd", width=_log(rng, 8, 2000), blocks=_log(rng, 1, 200), bits=rng.choice([8, 32]), dtype=dtype)
    width = _log(rng, 16, 1000)
    return dict(op=op, set="block", width=width, blocks=_log(rng, 1, 14), bits=rng.choice([8, 32]), dtype=dtype)


# --- what a program has in hand ---------------------------------------------------------


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, shape, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale)


def _norm_inputs(case, seed):
    g, t = _generator(seed), DTYPES[case["dtype"]]
    rows, c = case["rows"], case["c"]
    loud = 1.0 + 9.0 * (torch.rand(c, generator=g, device="cuda") < 0.01)  # a few channels of a residual stream are large
    s = {"x": _randn(g, (rows, c)).to(t), "gain": 1.0 + _randn(g, (c,), 0.2)}
    s["residual"] = (_randn(g, (rows, c), 2.0) * loud).to(t) if case["residual"] else None
    if case["mode"] == "train":
        s["dy"] = _randn(g, (rows, c), LOSS_SCALE * DY_STD).to(t)
        s["dsum"] = _randn(g, (rows, c), LOSS_SCALE * DY_STD).to(t)
    return s


def _groups(case):
    return 1 if case["group"] == 0 else -(-case["c"] // case["group"])


def _lengths(case):
    """Ragged: the first sequence is empty, the second has one token, the rest reach up to all t."""
    n, t = case["n"], case["t"]
    return [0 if i == 0 and n > 1 else min(1, t) if i == 1 else t * (i + 1) // n for i in range(n)] if case["ragged"] else [t] * n


def _recur_inputs(case, seed):
    g, dt = _generator(seed), DTYPES[case["dtype"]]
    n, t, c = case["n"], case["t"], case["c"]
    s = {"proj": _randn(g, (n, t, 3 * c)).to(dt)}  # value, forget gate, output gate, as one projection writes them
    s["bias"] = torch.rand(c, generator=g, device="cuda") * 7.0  # memories from 2 tokens to about 1000
    s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
    s["h"] = _randn(g, (n, c), 0.5) if case["carry"] else None
    if case["mode"] == "train":
        s["dy"] = _randn(g, (n, t, c), LOSS_SCALE * DY_STD).to(dt)
        s["dht"] = _randn(g, (n, c), LOSS_SCALE * DY_STD) if case["carry"] else None
    return s


def _adamw_sizes(case):
    """[(elements, weight decay)] of the tensors."""
    if case["set"] == "resnet50":  # the convolutions' weights [k][r][s][c], and a gain and a bias per output channel
        convs = [(64, 7, 4)] + [s for c, mid, count in ((64, 64, 3), (256, 128, 4), (512, 256, 6), (1024, 512, 3)) for i in range(count)
                                for s in ([(mid, 1, c if i == 0 else 4 * mid), (mid, 3, mid), (4 * mid, 1, mid)] + [(4 * mid, 1, c)] * (i == 0))]
        return [s for k, r, c in convs for s in ((k * r * r * c, DECAY), (k, 0.0), (k, 0.0))]
    w, got = case["width"], []
    for b in range(case["blocks"]):
        if case["set"] == "odd":
            got += [(1 + w * (b * 37 % 101), DECAY if b % 3 else 0.0)]
        else:  # norm gain, projection to three, gate bias, projection back, and two of a wider product
            got += [(w, 0.0), (3 * w * w, DECAY), (w, 0.0), (w * w, DECAY), (4 * w * w, DECAY), (4 * w * w, DECAY)]
    return got


def _arena(case):
    """Where each tensor begins in the flat arrays, and their size: tensors start at multiples of BLOCK, as allocations do."""
    sizes = _adamw_sizes(case)
    padded = [-(-n // BLOCK) * BLOCK for n, _ in sizes]
    starts = [0] + list(np.cumsum(padded))
    return sizes, [int(v) for v in starts[:-1]], int(starts[-1]), padded


def _adamw_inputs(case, seed):
    g = _generator(seed)
    sizes, starts, total, padded = _arena(case)
    count = torch.tensor([n for n, _ in sizes], device="cuda")
    at = torch.arange(total, device="cuda", dtype=torch.int64)
    pad = torch.tensor(padded, device="cuda")
    live = at - torch.tensor(starts, device="cuda").repeat_interleave(pad) < count.repeat_interleave(pad)
    s = {"master": _randn(g, (total,), 0.05).mul_(live)}
    size = torch.exp(_randn(g, (total,), 1.5)).mul_(live)  # gradients of one tensor span several orders
    s["grad"] = _randn(g, (total,), LOSS_SCALE * 1e-3).mul_(size)
    m, v = _randn(g, (total,), 3e-4).mul_(size), size.square().mul_(1e-6).mul_(torch.rand(total, generator=g, device="cuda") + 0.5)
    s["step"] = torch.full((1,), STEPS_DONE, dtype=torch.int32, device="cuda")
    s["flag"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    # the device-resident loss scaler: scale, growth factor, and its counters
    s["scaler"] = torch.cat([torch.tensor([LOSS_SCALE, 2.0]).view(torch.int32), torch.tensor([2000, 0, 0, 0], dtype=torch.int32)]).cuda()
    if case["bits"] == 8:
        half = torch.full((total,), 0.5, device="cuda")
        s["m"], s["m_scale"] = _encode(m, half, "m")
        s["v"], s["v_scale"] = _encode(v, half, "v")
    else:
        s["m"], s["v"] = m, v
    return s


def prepare(case, seed):
    """The inputs, the arrays that outputs go to, and for the framework's calls the object that holds sizes and workspaces."""
    dt = DTYPES[case["dtype"]]
    if case["op"] == "norm":
        s = _norm_inputs(case, seed)
        x = s["x"]
        s["sum"] = torch.empty_like(x) if case["residual"] else x
        s["rstd"] = torch.empty(case["rows"], dtype=torch.float32, device="cuda")
        s["y"] = torch.empty_like(x) if case["mode"] != "q8" else torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda")
        s["scales"] = torch.empty((case["rows"], _groups(case)), dtype=torch.float32, device="cuda")
        s["dx"], s["dgain"] = torch.empty_like(x), torch.empty(case["c"], dtype=torch.float32, device="cuda")
    elif case["op"] == "recur":
        s = _recur_inputs(case, seed)
        n, t, c = case["n"], case["t"], case["c"]
        s["y"] = torch.empty((n, t, c), dtype=dt, device="cuda")
        s["dproj"] = torch.empty_like(s["proj"])
        s["dbias"] = torch.empty(c, dtype=torch.float32, device="cuda")
        s["ht"] = torch.empty((n, c), dtype=torch.float32, device="cuda")
        s["dh0"] = torch.empty((n, c), dtype=torch.float32, device="cuda")
    else:
        s = _adamw_inputs(case, seed)
        s["w16"] = s["master"].to(dt)
    s["case"] = case
    if own:
        s["op"] = _framework_object(case, s)
    return s


def _code(case):
    from paper_2102_06725_amd import nnconv as nc
    return nc.NNCONV_F16 if case["dtype"] == "f16" else nc.NNCONV_BF16


def _framework_object(case, s):
    from paper_2102_06725_amd import nnconv as nc
    if case["op"] == "norm":
        return nc.RMSNorm(case["rows"], case["c"], dtype=_code(case), eps=EPS_NORM, group=case["group"])
    if case["op"] == "recur":
        op = nc.GatedRecurrence(case["n"], case["t"], case["c"], ld=3 * case["c"], dtype=_code(case))
        s["saved"] = op.saved() if case["mode"] == "train" else None
        return op
    sizes, starts, _, _ = _arena(case)
    tensors = []
    for (n, decay), at in zip(sizes, starts):
        t = {k: s[k][at:at + n] for k in ("master", "grad", "w16", "m", "v")}
        if case["bits"] == 8:
            t.update({k: s[k][at // BLOCK:-(-(at + n) // BLOCK)] for k in ("m_scale", "v_scale")})
        tensors.append(dict(t, weight_decay=decay))
    return nc.AdamW(tensors, seed=SEED8)


# --- a pass -------------------------------------------------------------------------


def run(state):
    return {"norm": _run_norm, "recur": _run_recur, "adamw": _run_adamw}[state["case"]["op"]](state)


def _run_norm(s):
    case = s["case"]
    keep = s["sum"] if case["residual"] else None
    if case["mode"] == "q8":
        if own:
            s["op"].fwd_q8(s["x"], s["gain"], s["y"], s["scales"], residual=s["residual"], sum=keep)
            out = {"q": s["y"], "scales": s["scales"]}
        else:
            r, _, y = _plain_norm(s)
            q, scales = _plain_q8(y, case)
            out = {"q": q, "scales": scales, "sum": r}
    elif case["mode"] == "fwd":
        if own:
            s["op"].fwd(s["x"], s["gain"], s["y"], residual=s["residual"], sum=keep)
            out = {"y": s["y"]}
        else:
            r, _, y = _plain_norm(s)
            out = {"y": y.to(r.dtype), "sum": r}
    elif own:
        s["op"].fwd(s["x"], s["gain"], s["y"], residual=s["residual"], sum=keep, rstd=s["rstd"])
        s["op"].bwd(s["sum"], s["dy"], s["gain"], s["rstd"], s["dx"], s["dgain"], dsum=s["dsum"], inv_loss_scale=1.0 / LOSS_SCALE)
        out = {k: s[k] for k in ("y", "rstd", "dx", "dgain")}
    else:
        r, rstd, y = _plain_norm(s)
        xh, dy = r.float() * rstd, s["dy"].float()
        p = dy * s["gain"]
        dx = s["dsum"].float() + rstd * (p - xh * (p * xh).mean(1, keepdim=True))
        out = {"y": y.to(r.dtype), "rstd": rstd.view(-1), "dx": dx.to(r.dtype), "dgain": (dy * xh).sum(0) / LOSS_SCALE, "sum": r}
    if case["residual"]:
        out.setdefault("sum", s["sum"])
    else:
        out.pop("sum", None)
    return out


def _plain_norm(s):
    r = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
    v = r.float()
    rstd = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS_NORM)
    return r, rstd, v * rstd * s["gain"]


def _plain_q8(y, case):
    rows, c = y.shape
    n = _groups(case)
    y = torch.nn.functional.pad(y, (0, n * case["group"] - c)) if case["group"] else y
    y = y.view(rows, n, -1)
    scales = y.abs().amax(2) / F8_MAX
    q = (y / scales.unsqueeze(2)).nan_to_num(0.0).view(rows, -1)[:, :c]
    return q.to(torch.float8_e4m3fn), scales


def _run_recur(s):
    case = s["case"]
    n, t, c = case["n"], case["t"], case["c"]
    x, f, g = (s["proj"][..., i * c:(i + 1) * c] for i in range(3))
    if own:
        carry, train = case["carry"], case["mode"] == "train"
        # serving updates the state in place; training keeps the first state for the backward pass
        ht = s["ht"] if train else s["h"] if carry else None
        s["op"].fwd(x, f, s["bias"], s["y"], g=g, lengths=s["lengths"], h0=s["h"], ht=ht, saved=s.get("saved"))
        if not train:
            return {"y": s["y"], "h": s["h"]} if carry else {"y": s["y"]}
        dx, df, dg = (s["dproj"][..., i * c:(i + 1) * c] for i in range(3))
        s["op"].bwd(x, f, s["bias"], s["saved"], s["dy"], dx, df, g=g, dg=dg, lengths=s["lengths"], dht=s["dht"],
                    dh0=s["dh0"] if carry else None, dbias=s["dbias"], inv_loss_scale=1.0 / LOSS_SCALE)
        out = {"y": s["y"], "ht": s["ht"], "dproj": s["dproj"], "dbias": s["dbias"]}
        return dict(out, dh0=s["dh0"]) if carry else out
    dt = s["proj"].dtype
    x, f, g = x.float(), f.float(), g.float()
    z = (f + s["bias"]).clamp(-GATE_LIMIT, GATE_LIMIT)
    a, b, gate = torch.sigmoid(z), torch.sigmoid(-z), torch.sigmoid(g)
    live = None
    if s["lengths"] is not None:
        live = (torch.arange(t, device="cuda") < s["lengths"].view(n, 1)).unsqueeze(2)
        a, b = torch.where(live, a, 1.0), torch.where(live, b, 0.0)
    u = b * x
    if s["h"] is not None:
        u[:, 0] += a[:, 0] * s["h"]
    h = _scan(a, u)
    y = h * g * gate
    y = y if live is None else torch.where(live, y, 0.0)
    if case["mode"] == "fwd":
        if s["h"] is None:
            return {"y": y.to(dt)}
        s["h"].copy_(h[:, -1])
        return {"y": y.to(dt), "h": s["h"]}
    dy = s["dy"].float()
    dy = dy if live is None else torch.where(live, dy, 0.0)
    dh = dy * g * gate
    if s["dht"] is not None:
        dh[:, -1] += s["dht"]
    after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    dh = _scan(after.flip(1), dh.flip(1)).flip(1)
    first = torch.zeros_like(h[:, :1]) if s["h"] is None else s["h"].unsqueeze(1)
    before = torch.cat([first, h[:, :-1]], 1)
    dz = dh * (before - x) * a * b
    dg = dy * h * gate * (1.0 + g * (1.0 - gate))
    out = {"y": y.to(dt), "ht": h[:, -1].clone(), "dproj": torch.cat([dh * b, dz, dg], 2).to(dt), "dbias": dz.sum((0, 1)) / LOSS_SCALE}
    return dict(out, dh0=a[:, 0] * dh[:, 0]) if case["carry"] else out


def _scan(a, u):
    """h_t = a_t h_(t-1) + u_t over dimension 1, by doubling: after a step of k, each place holds the sum over its last 2k tokens."""
    k, t = 1, a.shape[1]
    while k < t:
        u = torch.cat([u[:, :k], u[:, k:] + a[:, k:] * u[:, :-k]], 1)
        a = torch.cat([a[:, :k], a[:, k:] * a[:, :-k]], 1)
        k *= 2
    return u


def _power(e):
    """2^e for whole e from -126 to 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _encode(x, u, which):
    """8-bit codes of x with one power of two per BLOCK elements; u in (0, 1) says where each element is rounded."""
    top, low, bits, kind = (8, -6, 3, torch.float8_e4m3fn) if which == "m" else (15, -14, 2, torch.float8_e5m2)
    x, u = x.view(-1, BLOCK), u.view(-1, BLOCK)
    most = x.abs().amax(1, keepdim=True)
    mant, e = torch.frexp(most)
    k = torch.where(most > 0, e - 1 - top + (mant > 0.875), -127).clamp(-127, 127)
    y = (x * _power(-k)).abs()
    ulp = _power(torch.frexp(y)[1].sub(1).clamp(min=low) - bits)
    r = torch.floor(y / ulp + u)
    if which == "v":
        r = torch.where((r == 0) & (y > 0), 1.0, r)
    r = (r * ulp).clamp(max=1.75 * 2.0 ** top)
    code = torch.copysign(r, x).to(kind).view(-1)
    return code, (k + 127).to(torch.uint8).view(torch.float8_e8m0fnu).view(-1)


def _decode(code, scale):
    return (code.float().view(-1, BLOCK) * scale.float().view(-1, 1)).view(-1)


def _dither(case, step):
    """Two numbers in (0, 1) for every element, 16 bits each of one hash of (seed, step, tensor, element)."""
    _, starts, total, padded = _arena(case)
    low = 0xFFFFFFFF
    tensor = torch.arange(len(padded), device="cuda").repeat_interleave(torch.tensor(padded, device="cuda"))
    index = torch.arange(total, device="cuda") - torch.tensor(starts, device="cuda")[tensor]
    h = (index * 0x9E3779B1 + tensor * 0x6C8E9CF5 + step.long() * 0xB5297A4D + SEED8 * 0x68E31DA4) & low
    h = ((h ^ (h >> 16)) * 0x2C1B3C6D) & low
    h = ((h ^ (h >> 15)) * 0x297A2D39) & low
    h = h ^ (h >> 16)
    return [((v.float() + 0.5) * 2.0 ** -16) for v in (h & 0xFFFF, h >> 16)]


def _run_adamw(s):
    case = s["case"]
    names = ("master", "w16", "m", "v", "step") + (("m_scale", "v_scale") if case["bits"] == 8 else ())
    if own:
        s["op"].step(s["step"], LR, BETA1, BETA2, EPS, state=s["scaler"], overflow_flag=s["flag"])
        return {k: s[k] for k in names}
    sizes, _, _, padded = _arena(case)
    decay = torch.tensor([d for _, d in sizes], device="cuda").repeat_interleave(torch.tensor(padded, device="cuda"))
    go = s["flag"] == 0  # a step with an inf or NaN gradient changes nothing
    step = s["step"] + go
    eight = case["bits"] == 8
    m = _decode(s["m"], s["m_scale"]) if eight else s["m"]
    v = _decode(s["v"], s["v_scale"]) if eight else s["v"]
    g = s["grad"] / s["scaler"][:1].view(torch.float32)
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    left1, left2 = ((1.0 - torch.pow(b, step.double())).float() for b in (BETA1, BETA2))
    w = s["master"] - LR * (m / left1 / (torch.sqrt(v / left2) + EPS) + decay * s["master"])
    new = {"master": w, "w16": w.to(DTYPES[case["dtype"]]), "m": m, "v": v}
    if eight:
        um, uv = _dither(case, step)
        new["m"], new["m_scale"] = _encode(m, um, "m")
        new["v"], new["v_scale"] = _encode(v, uv, "v")
    s.update({k: torch.where(go, x.view(torch.uint8), s[k].view(torch.uint8)).view(x.dtype) if x.element_size() == 1 else torch.where(go, x, s[k])
              for k, x in new.items()})
    s["step"] = step.to(torch.int32)
    return {k: s[k] for k in names}


# --- work ------------------------------------------------------------------------------


def work(case):
    if case["op"] == "norm":
        e, rows, c = case["rows"] * case["c"], case["rows"], case["c"]
        io = e * (2 + (4 if case["residual"] else 0)) + 4 * c  # x, and the residual and the sum
        if case["mode"] == "q8":
            return {"bytes": io + e + 4 * rows * _groups(case), "flops": 7 * e}
        if case["mode"] == "fwd":
            return {"bytes": io + 2 * e, "flops": 5 * e}
        return {"bytes": io + 2 * e + 4 * rows + 6 * e + 4 * c, "flops": 15 * e}  # and dy, dsum, dx, dgain
    if case["op"] == "recur":
        c, n, t = case["c"], case["n"], case["t"]
        live, every = sum(_lengths(case)) * c, n * t * c
        state = 4 * n * c * ((1 if case["carry"] else 0) + (1 if case["carry"] or case["mode"] == "train" else 0))
        if case["mode"] == "fwd":
            return {"bytes": 6 * live + 2 * every + state + 4 * c, "flops": 16 * live}
        return {"bytes": 8 * live + 8 * every + state + (8 * n * c if case["carry"] else 0) + 8 * c, "flops": 50 * live}
    sizes = _adamw_sizes(case)
    e, blocks = sum(n for n, _ in sizes), sum(-(-n // BLOCK) for n, _ in sizes)
    # read grad, master, m, v; write master, its 16-bit copy, m, v
    return {"bytes": 14 * e + (4 * e + 4 * blocks if case["bits"] == 8 else 16 * e), "flops": (60 if case["bits"] == 8 else 15) * e}


# --- in 64 bits ----------------------------------------------------------------------------


def exact(case, seed):
    return {"norm": _exact_norm, "recur": _exact_recur, "adamw": _exact_adamw}[case["op"]](case, seed)


def _exact_norm(case, seed):
    s = _norm_inputs(case, seed)
    gain = s["gain"].double()
    r = s["x"] if s["residual"] is None else (s["x"].double() + s["residual"].double()).to(s["x"].dtype)
    v = r.double()
    rstd = (v.square().sum(1) / case["c"] + EPS_NORM).pow(-0.5)
    xh = v * rstd[:, None]
    y = xh * gain
    out = {}
    if case["mode"] == "q8":
        n, width = _groups(case), case["group"] or case["c"]
        most = torch.zeros((case["rows"], n), dtype=torch.float64, device="cuda")
        for i in range(n):
            most[:, i] = y[:, i * width:(i + 1) * width].abs().amax(1)
        out["q"] = y * F8_MAX / most.repeat_interleave(width, 1)[:, :case["c"]]  # before the rounding to 8 bits
        out["scales"] = most / F8_MAX
    else:
        out["y"] = y
    if case["mode"] == "train":
        dy = s["dy"].double()
        out["rstd"] = rstd
        out["dgain"] = torch.einsum("rc,rc->c", dy, xh) / LOSS_SCALE
        along = torch.einsum("rc,rc->r", dy * gain, xh) / case["c"]
        out["dx"] = s["dsum"].double() + (dy * gain - xh * along[:, None]) * rstd[:, None]
    if case["residual"]:
        out["sum"] = r.double()
    return out


def _exact_recur(case, seed):
    s = _recur_inputs(case, seed)
    n, t, c = case["n"], case["t"], case["c"]
    x, f, g = (v.double() for v in s["proj"].split(c, 2))
    z = (f + s["bias"].double()).clamp(-GATE_LIMIT, GATE_LIMIT)
    a = 1.0 / (1.0 + torch.exp(-z))
    b = 1.0 / (1.0 + torch.exp(z))
    lengths = _lengths(case)
    for i, k in enumerate(lengths):
        a[i, k:], b[i, k:] = 1.0, 0.0
    h = torch.empty((n, t + 1, c), dtype=torch.float64, device="cuda")
    h[:, 0] = 0.0 if s["h"] is None else s["h"].double()
    u = b * x
    for k in range(t):
        torch.addcmul(u[:, k], a[:, k], h[:, k], out=h[:, k + 1])
    gate = 1.0 / (1.0 + torch.exp(-g))
    y = h[:, 1:] * (g * gate)
    for i, k in enumerate(lengths):
        y[i, k:] = 0.0
    if case["mode"] == "fwd":
        return {"y": y, "h": h[:, t]} if case["carry"] else {"y": y}
    dy = s["dy"].double()
    for i, k in enumerate(lengths):
        dy[i, k:] = 0.0
    own_part = dy * (g * gate)
    d = torch.empty_like(own_part)  # the gradient of each h
    into = torch.zeros((n, c), dtype=torch.float64, device="cuda") if s["dht"] is None else s["dht"].double()
    for k in range(t - 1, -1, -1):
        torch.add(own_part[:, k], into, out=d[:, k])
        into = d[:, k] * a[:, k]
    dproj = torch.empty((n, t, 3 * c), dtype=torch.float64, device="cuda")
    dproj[..., :c] = d * b
    dproj[..., c:2 * c] = d * (h[:, :-1] - x) * a * b
    dproj[..., 2 * c:] = dy * h[:, 1:] * (gate + g * gate * (1.0 - gate))
    out = {"y": y, "ht": h[:, t], "dproj": dproj, "dbias": dproj[..., c:2 * c].sum((0, 1)) / LOSS_SCALE}
    return dict(out, dh0=into) if case["carry"] else out


def _exact_adamw(case, seed):
    s = _adamw_inputs(case, seed)
    sizes, starts, _, _ = _arena(case)
    m, v = s["m"].double(), s["v"].double()
    if case["bits"] == 8:
        m = m * s["m_scale"].double().repeat_interleave(BLOCK)
        v = v * s["v_scale"].double().repeat_interleave(BLOCK)
    g = s["grad"].double() / LOSS_SCALE
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * g ** 2
    k = STEPS_DONE + 1
    w = s["master"].double()
    change = (m / (1.0 - BETA1 ** k)) / ((v / (1.0 - BETA2 ** k)) ** 0.5 + EPS)
    for (n, decay), at in zip(sizes, starts):
        change[at:at + n] += decay * w[at:at + n]
    w = w - LR * change
    if case["bits"] == 8:  # the moments' codes depend on the rounding
        return {"master": w, "w16": w, "m": None, "v": None, "step": None, "m_scale": None, "v_scale": None}
    return {"master": w, "w16": w, "m": m, "v": v, "step": None}
