"""Tables and gradients of more than 2^32 bytes: rows at both ends are found."""
import numpy as np
import pytest

from paper_2102_06725_amd import nnconv as nc

import sequence_util as U

pytestmark = pytest.mark.gpu
V, C = 2 ** 21, 1040  # 4.4 GB in 16 bits


@pytest.fixture(scope="module")
def table():
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(1)
    return t.randn((V, C), generator=g, device="cuda", dtype=t.bfloat16) * 0.05


def test_embedding(nnlib, table):
    t = U.torch()
    ids = t.tensor([0, V - 1, 5, V - 1, V // 2, V], dtype=t.int32, device="cuda")
    op = nc.Embedding(6, C, V, dtype=nc.NNCONV_BF16, scale=2.0)
    y = t.empty((6, C), dtype=t.bfloat16, device="cuda")
    op.fwd(ids, table, y)
    at = ids[:5].long()
    assert t.equal(y[:5], table[at] * 2.0) and not bool(y[5].any())
    grad = t.zeros((V, C), dtype=t.bfloat16, device="cuda")
    dy = t.ones_like(y)
    for accumulate in (1, 0):
        grad[V - 2] = 3.0
        op.bwd(ids, dy, grad, accumulate=accumulate)
        rows = [(0, 2.0), (5, 2.0), (V // 2, 2.0), (V - 1, 4.0), (V - 2, 3.0 if accumulate else 0.0), (1, 0.0)]
        for row, value in rows:
            assert bool((grad[row] == value).all()), (row, accumulate)
        assert float(grad.float().sum()) == C * (10.0 + (3.0 if accumulate else 0.0))


@pytest.mark.parametrize("k", [None, 3])
def test_loss(nnlib, table, k):
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(2)
    rows = 5
    x = t.randn((rows, C), generator=g, device="cuda").bfloat16()
    targets = t.randint(0, V, (rows, k or 1), generator=g, device="cuda", dtype=t.int32)
    targets[0, 0], targets[1, 0], targets[2, 0] = V - 1, 0, V // 2 + 1
    teacher = None if k is None else t.randn((rows, k), generator=g, device="cuda")
    op = nc.CrossEntropy(rows, C, V, dtype=nc.NNCONV_BF16, k=k)
    loss, dx, dw = t.empty(rows, device="cuda"), t.empty_like(x), t.empty_like(table)
    op.train(x, table, targets if k else targets[:, 0].contiguous(), loss, dx, dw, teacher=teacher)
    z = t.cat([(x.double() @ table[i:i + V // 16].double().t()) for i in range(0, V, V // 16)], 1)
    p = t.log_softmax(z, 1)
    log_q = t.zeros((rows, 1), device="cuda", dtype=t.float64) if k is None else t.log_softmax(teacher.double(), 1)
    want = (log_q.exp() * (log_q - p.gather(1, targets.long()))).sum(1)
    # z of 1040 products (2^-13 of their magnitudes' sum at most), lse, shares
    assert float((loss - want).abs().max()) < 2.0 ** -12
    dz = p.exp_().scatter_add_(1, targets.long(), -log_q.exp())
    ref = sum(dz[:, i:i + V // 16] @ table[i:i + V // 16].double() for i in range(0, V, V // 16))
    # one rounding of dz and one of the result, in each term at most
    mag = sum(dz[:, i:i + V // 16].abs() @ table[i:i + V // 16].double().abs() for i in range(0, V, V // 16))
    assert bool(((dx.double() - ref).abs() <= 1.2 * 2.0 ** -8 * mag + 2.0 ** -8 * ref.abs()).all())
    for row in (0, 1, V // 2 + 1, V - 2, V - 1):
        got, want = dw[row].double(), dz[:, row] @ x.double()
        assert bool(((got - want).abs() <= 1.2 * 2.0 ** -8 * (dz[:, row].abs() @ x.double().abs()) + 2.0 ** -8 * want.abs() + 2.0 ** -20).all()), row


def test_many_rows(nnlib):
    """x, dx and y of more than 2^32 bytes."""
    t = U.torch()
    rows, c, v = 2 ** 21 + 3, 1032, 3
    g = t.Generator(device="cuda").manual_seed(3)
    ids = t.randint(0, v, (rows,), generator=g, device="cuda", dtype=t.int32)
    w = t.randn((v, c), generator=g, device="cuda").half()
    x = t.empty((rows, c), dtype=t.float16, device="cuda")
    nc.Embedding(rows, c, v, scale=0.25).fwd(ids, w, x)
    for r in (0, 1, rows // 2, rows - 1):
        assert t.equal(x[r], w[ids[r].long()] * 0.25)
    loss, dx, dw = t.empty(rows, device="cuda"), t.empty_like(x), t.empty((v, c), device="cuda")
    op = nc.CrossEntropy(rows, c, v)
    target = (ids + 1) % v
    op.train(x, w, target, loss, dx, dw)
    logits = 0.25 * (w.double() @ w.double().t())  # rows are one of three
    dz = t.softmax(logits, 1)
    want = t.log_softmax(logits, 1)
    for r in (0, 1, rows // 3, rows - 2, rows - 1):
        i, j = int(ids[r]), int(target[r])
        assert abs(float(loss[r] + want[i, j])) < 2.0 ** -10 + 2.0 ** -20 * abs(float(want[i, j]))
        d = dz[i].clone()
        d[j] -= 1.0
        ref, mag = d @ w.double(), d.abs() @ w.double().abs()
        assert bool(((dx[r].double() - ref).abs() <= 1.3 * 2.0 ** -11 * mag + 2.0 ** -11 * ref.abs() + 2.0 ** -20).all())
    grad = t.empty((v, c), device="cuda")
    nc.Embedding(rows, c, v, scale=1.0).bwd(ids, x, grad)
    n = np.bincount(ids.cpu().numpy(), minlength=v)
    ref = t.from_numpy(n).double().cuda()[:, None] * (w * 0.25).double()
    # chains of 32 tokens of a span and up to 2^16 spans
    assert bool(((grad.double() - ref).abs() <= 2.0 ** -24 * (2 ** 16 + 40) * ref.abs()).all())
