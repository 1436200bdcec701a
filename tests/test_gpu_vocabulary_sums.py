"""Sums over very many rows, exact: small integers, in any order."""
import pytest

from paper_2102_06725_amd import nnconv as nc

import sequence_util as U

pytestmark = pytest.mark.gpu


def integers(shape, dtype, seed, most=3):
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(seed)
    return t.randint(-most, most + 1, shape, generator=g, device="cuda", dtype=t.int8).to(dtype)


def sums(ids, dy, v):
    """Exact sums of the rows that each number names: differences of each column's running sums (additions to a place
    of their own would wait for each other where one number is common)."""
    t = U.torch()
    at = t.where((ids >= 0) & (ids < v), ids, v).long()
    at, order = t.sort(at)
    end = t.searchsorted(at, t.arange(v, device="cuda"), right=True)
    out = t.empty((v, dy.shape[1]), dtype=t.float64, device="cuda")
    for c in range(dy.shape[1]):
        run = t.cat([t.zeros(1, dtype=t.float64, device="cuda"), t.cumsum(dy[:, c][order].double(), 0)])[end]
        out[:, c] = run.diff(prepend=run.new_zeros(1))
    return out


def test_a_heads_gradient(nnlib):
    """x of more than 2^32 bytes, all logits equal: dw is a fourth of the sum of all rows less the sum of its own."""
    t = U.torch()
    rows, c, v = 2 ** 21 + 3, 1032, 4
    x = integers((rows, c), t.float16, 1)
    w = t.zeros((v, c), dtype=t.float16, device="cuda")
    targets = t.randint(0, v, (rows,), generator=t.Generator(device="cuda").manual_seed(2), device="cuda", dtype=t.int32)
    loss, dx, dw = t.empty(rows, device="cuda"), t.empty_like(x), t.empty((v, c), device="cuda")
    nc.CrossEntropy(rows, c, v).train(x, w, targets, loss, dx, dw)
    own = sums(targets, x, v)
    assert t.equal(dw.double(), own.sum(0) / v - own)


@pytest.mark.parametrize("rows,c,v,common", [
    (2 ** 21 + 3, 1032, 3, 0.0),          # dy of more than 2^32 bytes, runs of 700000
    (2 ** 22 + 77, 8, 5000, 0.9),         # nine in ten are one number
    (2 ** 24 + 5, 3, 70000, 0.0),         # three sorting passes
    (2 ** 26, 1, 1000, 0.5),              # the most tokens
    (2 ** 20 + 1, 40, 2 ** 20 + 9, 0.2)])
def test_an_embeddings_gradient(nnlib, rows, c, v, common):
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(rows)
    ids = t.randint(-1, v + 1, (rows,), generator=g, device="cuda", dtype=t.int32)
    if common:
        ids[t.rand(rows, generator=g, device="cuda") < common] = v // 2
    dy = integers((rows, c), t.float16, 3)
    want = sums(ids, dy, v)
    op = nc.Embedding(rows, c, v)
    new, added = t.empty((v, c), device="cuda"), t.full((v, c), 7.0, device="cuda")
    op.bwd(ids, dy, new)
    op.bwd(ids, dy, added, accumulate=1)
    assert t.equal(new.double(), want) and t.equal(added.double(), want + 7.0)
