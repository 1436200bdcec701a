"""The model over a vocabulary, which runs embedding, blocks, cross entropy or distillation and AdamW together:
its gradients against automatic differentiation in 64 bits, serving against the whole pass, a captured training
step against the same step queued call by call."""
import math

import numpy as np
import pytest

import sequence_util as U

pytestmark = pytest.mark.gpu


def make(n, t, dtype, v=203, c=64, blocks=2, k=None, seed=3):
    from paper_2102_06725_amd.token_model import TokenModel, counting
    m = TokenModel(n, t, v, c, blocks, dtype=U.CODE[dtype], seed=seed, k=k)
    ids, targets = counting(n, t, v, seed=4)
    targets[0, t // 3:] = -1
    return m, ids, targets


def reference(model, ids, targets, teacher=None):
    """Token losses and parameter gradients of the model's 16-bit weights, by torch's autograd in float64 on the CPU."""
    t = U.torch()
    p = {k: (model.w16[k] if k in model.w16 else m).detach().double().cpu().clone().requires_grad_(True) for k, m in model.master.items()}
    c = model.c
    lin = lambda v, w: v @ w.reshape(w.shape[0], -1).T  # noqa: E731

    def norm(v, gain):
        return v * t.rsqrt((v * v).mean(-1, keepdim=True) + 1e-6) * gain
    ids, targets = ids.cpu().long(), targets.cpu().long()
    h = p["table"][ids.clamp(min=0)] * math.sqrt(c) * (ids >= 0)[..., None]
    r = 0.0
    for b in range(model.blocks):
        r = h + r
        q = lin(norm(r, p["gain%d" % b]), p["in%d" % b])
        v, f, g = q[..., :c], q[..., c:2 * c], q[..., 2 * c:]
        a = t.sigmoid(f + p["bias%d" % b])
        s, ys = t.zeros_like(v[:, 0]), []
        for k in range(v.shape[1]):
            s = a[:, k] * s + (1.0 - a[:, k]) * v[:, k]
            ys.append(s * t.nn.functional.silu(g[:, k]))
        h = lin(t.stack(ys, 1), p["out%d" % b])
    z = t.log_softmax(lin(norm(h + r, p["gain"]), p["table"]), -1)
    if teacher is None:
        losses = -z.gather(-1, targets.clamp(min=0)[..., None])[..., 0] * (targets >= 0)
    else:
        q = t.log_softmax(teacher.double().cpu(), -1)
        losses = (q.exp() * (q - z.gather(-1, targets.clamp(min=0)))).sum(-1) * (targets[..., 0] >= 0)
    (losses.sum() / losses.numel()).backward()
    return losses.detach().numpy(), {k: v.grad.numpy() for k, v in p.items()}


# the longest way from a loss to a parameter passes about 22 roundings to 16 bits, each of at most half a unit in the
# last place of a value; gradients add such errors of both signs
@pytest.mark.parametrize("dtype,bound", [("f16", 22 * 2.0 ** -11), ("bf16", 22 * 2.0 ** -8)])
@pytest.mark.parametrize("n,t,k", [(2, 150, None), (3, 33, None), (2, 70, 9)])
def test_gradients(nnlib, n, t, k, dtype, bound):
    tt = U.torch()
    m, ids, targets = make(n, t, dtype, k=k)
    teacher = None
    if k is not None:
        g = tt.Generator(device="cuda").manual_seed(1)
        at = tt.stack([tt.randperm(m.v, generator=g, device="cuda")[:k] for _ in range(n * t)]).view(n, t, k)
        targets = tt.where((targets >= 0)[..., None], at.int(), -1)
        teacher = tt.randn((n, t, k), generator=g, device="cuda")
    m.forward(ids)
    losses = m.backward(ids, targets, teacher).double().cpu().numpy()
    tt.cuda.synchronize()
    ref, grads = reference(m, ids, targets, teacher)
    assert np.linalg.norm(losses - ref) <= bound * np.linalg.norm(ref)
    for name, want in grads.items():
        got = m.dw[name].double().cpu().numpy().reshape(want.shape) / 1024.0
        assert np.linalg.norm(got - want) <= bound * np.linalg.norm(want), name
    assert int(m.flag.item()) == 0


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_serving(nnlib, dtype):
    """Token by token the logits are those of the whole pass, and the score the loss of the logits."""
    from paper_2102_06725_amd.token_model import TokenServer
    tt = U.torch()
    n, t = 6, 40
    m, ids, targets = make(n, t, dtype)
    for _ in range(3):
        m.train_step(ids, targets, lr=3e-3)
    whole = m.logits(ids).double().cpu()
    server = TokenServer(m, n)
    for _ in range(2):
        server.reset()
        served = tt.stack([server.step(ids[:, i].contiguous()).double().cpu().clone() for i in range(t)], 1)
        # both are about 20 roundings from the exact logits
        assert float((served - whole).norm() / whole.norm()) <= 2 * 20 * U.HALF_ULP[dtype]
    score = m.score(ids, targets).double().cpu()
    live = (targets >= 0).cpu()
    want = -tt.log_softmax(whole, -1).gather(-1, targets.cpu().long().clamp(min=0)[..., None])[..., 0] * live
    # the whole pass's logits are rounded to 16 bits
    assert float((score - want).abs().max()) <= 4 * U.HALF_ULP[dtype] * float(whole.abs().max())
    assert bool((score[~live] == 0).all())


@pytest.mark.parametrize("k", [None, 5])
def test_captured_step_is_the_same_step(nnlib, k):
    tt = U.torch()
    a, ids, targets = make(3, 60, "bf16", k=k)
    b, _, _ = make(3, 60, "bf16", k=k)
    teacher = None
    if k is not None:
        targets, teacher = a.largest_logits(ids, k)
    s = tt.cuda.Stream()
    for m in (a, b):  # workspaces exist before the capture
        with tt.cuda.stream(s):
            s.wait_stream(tt.cuda.default_stream())
            m.train_step(ids, targets, lr=1e-3, teacher=teacher)
    tt.cuda.synchronize()
    graph = tt.cuda.CUDAGraph()
    with tt.cuda.graph(graph, stream=s):
        b.train_step(ids, targets, lr=1e-3, teacher=teacher)
    for i in range(3):
        with tt.cuda.stream(s):
            a.train_step(ids, targets, lr=1e-3, teacher=teacher)
        tt.cuda.synchronize()
        graph.replay()
        tt.cuda.synchronize()
        assert int(a.step_count.item()) == int(b.step_count.item()) == i + 2
        assert tt.equal(a.losses, b.losses)
        for key in a.flat:
            assert bool((a.flat[key].view(tt.uint8) == b.flat[key].view(tt.uint8)).all()), (i, key)


def test_an_overflow_skips_the_step(nnlib):
    tt = U.torch()
    m, ids, targets = make(2, 64, "f16")
    m.train_step(ids, targets, lr=1e-3)
    before = {k: v.clone() for k, v in m.flat.items() if k != "grad"}
    m.loss_scale.fill_(2.0 ** 40)  # the gradients pass fp16's range
    m.train_step(ids, targets, lr=1e-3)
    assert int(m.step_count.item()) == 1 and float(m.loss_scale.item()) == 2.0 ** 39 and int(m.flag.item()) == 0
    for k, v in before.items():
        assert bool((m.flat[k].view(tt.uint8) == v.view(tt.uint8)).all()), k


def test_the_example_runs(nnlib, capsys):
    from paper_2102_06725_amd import token_model
    token_model.main(steps=3)
    assert "served token by token" in capsys.readouterr().out
