"""The fp64 oracle of embedding, cross entropy and distillation against torch's float64 on the CPU and against
differences; plants of plausible mistakes have to be seen."""
import numpy as np
import pytest

from oracle import vocabulary as V


def inputs(rows=7, c=5, v=11, k=None, seed=0):
    rng = np.random.default_rng(seed)
    x, w = rng.standard_normal((rows, c)), rng.standard_normal((v, c))
    targets = rng.integers(0, v, (rows, 1)) if k is None else np.stack([rng.permutation(v)[:k] for _ in range(rows)])
    return x, w, targets, None if k is None else rng.standard_normal((rows, k))


def test_embedding_against_torch():
    import torch
    rng = np.random.default_rng(1)
    table, dy, ids = rng.standard_normal((6, 4)), rng.standard_normal((9, 4)), rng.integers(0, 6, 9)
    t = torch.tensor(table, requires_grad=True)
    y = 1.5 * torch.nn.functional.embedding(torch.tensor(ids), t)
    y.backward(torch.tensor(dy))
    assert np.allclose(V.embedding_fwd(ids, table, 1.5), y.detach().numpy(), rtol=1e-15)
    d, mag, n = V.embedding_bwd(ids, dy, 6, 1.5)
    assert np.allclose(d, t.grad.numpy(), rtol=1e-13, atol=1e-13) and np.all(mag >= np.abs(d) - 1e-12) and n.sum() == 9
    ids[3], ids[4] = -1, 6  # padding
    assert not V.embedding_fwd(ids, table, 1.5)[3:5].any() and V.embedding_bwd(ids, dy, 6, 1.5)[2].sum() == 7


@pytest.mark.parametrize("scale", [1.0, 0.3])
def test_labels_against_torch(scale):
    import torch
    x, w, targets, _ = inputs()
    targets[2], targets[5] = -1, 11
    X, W = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
    label = torch.tensor(np.where((targets < 0) | (targets > 10), -100, targets)[:, 0])
    loss = torch.nn.functional.cross_entropy(scale * X @ W.t(), label, reduction="none")
    (2.0 * loss.sum()).backward()
    o = V.cross_entropy(x, w, targets, scale)
    dx, dw = V.gradients(o, w, scale, 2.0)
    assert np.allclose(o["loss"], loss.detach().numpy(), atol=1e-13)
    assert np.allclose(dx, X.grad.numpy(), atol=1e-13) and np.allclose(dw, W.grad.numpy(), atol=1e-13)


def test_teacher_against_torch():
    import torch
    x, w, targets, teacher = inputs(k=4)
    targets[1, 2], teacher[3, 0] = -1, -np.inf
    X, W = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
    z = torch.log_softmax(0.5 * X @ W.t(), 1)
    total = 0.0
    for r in range(7):
        live = [i for i in range(4) if targets[r, i] >= 0 and teacher[r, i] != -np.inf]
        q = torch.softmax(0.5 * torch.tensor(teacher[r, live]), 0)
        total = total + torch.nn.functional.kl_div(z[r, targets[r, live]], q, reduction="sum")
    total.backward()
    o = V.cross_entropy(x, w, targets, 0.5, teacher)
    dx, dw = V.gradients(o, w, 0.5, 1.0)
    assert np.isclose(o["loss"].sum(), total.item(), atol=1e-13)
    assert np.allclose(dx, X.grad.numpy(), atol=1e-13) and np.allclose(dw, W.grad.numpy(), atol=1e-13)


@pytest.mark.parametrize("k", [None, 3])
def test_gradients_by_differences(k):
    x, w, targets, teacher = inputs(k=k, seed=3)
    if k is not None:
        targets[0] = targets[0, 0]  # one target, three times
    o = V.cross_entropy(x, w, targets, 0.7, teacher)
    dx, dw = V.gradients(o, w, 0.7, 1.0)
    rng = np.random.default_rng(4)
    ux, uw, h = rng.standard_normal(x.shape), rng.standard_normal(w.shape), 1e-5
    at = lambda s: V.cross_entropy(x + s * ux, w + s * uw, targets, 0.7, teacher)["loss"].sum()  # noqa: E731
    # central differences: the step's square times a third derivative of order 100, and rounding over the step
    assert abs((at(h) - at(-h)) / (2 * h) - (dx * ux).sum() - (dw * uw).sum()) < 1e-7


def test_rows_that_do_not_count():
    x, w, targets, teacher = inputs(k=3)
    x[4], targets[4] = np.nan, -1
    teacher[2] = -np.inf
    o = V.cross_entropy(x, w, targets, 1.0, teacher)
    dx, dw = V.gradients(o, w, 1.0, 1.0)
    assert not o["counts"][[2, 4]].any() and np.isfinite(dw).all()
    for v in (o["loss"], o["lse"], dx):
        assert not v[[2, 4]].any()


def test_plants():
    """Mistakes that the bounds of the GPU tests have to see, on an ordinary case: they are planted in the oracle's
    results."""
    import vocabulary_util as W
    rng = np.random.default_rng(5)
    x, w, targets, _ = W.loss_inputs(rng, 40, 24, 130, "bf16")
    o = V.cross_entropy(x, w, targets, 1.0)
    eloss, elast, edz = W.bounds(o, x, w, targets, "bf16", 1.0)
    dx, dw = V.gradients(o, w, 1.0, 1.0)
    sum_x = edz @ np.abs(w) + 2.0 ** -8 * np.abs(dx)
    sum_w = edz.T @ np.abs(x) + 2.0 ** -8 * np.abs(dw)
    no_target = np.where(o["dz"] < 0, o["p"], o["dz"])
    shifted = np.roll(o["dz"], 1, axis=1)
    last_tile = o["dz"].copy()
    last_tile[:, 128:] = 0.0
    for name, dz in (("no target", no_target), ("shifted", shifted), ("a tile less", last_tile), ("twice", 2 * o["dz"])):
        assert (np.abs(dz @ w - dx) > sum_x).any(), name
        assert (np.abs(dz.T @ x - dw) > sum_w).any(), name
    assert (np.abs(np.log(np.exp(o["z"][:, :128]).sum(1)) - o["lse"]) > elast).any()
    assert (np.abs(o["loss"] + 2.0 ** -12 - o["loss"]) > eloss).any()
