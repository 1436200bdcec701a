"""nnconv_xent_* against the fp64 oracle; vocabulary_util.bounds has the error bounds."""
import numpy as np
import pytest

from oracle import vocabulary as V
from paper_2102_06725_amd import nnconv as nc

import sequence_util as U
import vocabulary_util as W

pytestmark = pytest.mark.gpu

SIZES = [  # rows, c, v, dtype, padding, elements past 16-byte alignment
    (1, 1, 1, "f16", 0.0, 0), (1, 8, 2, "bf16", 0.0, 0), (3, 7, 5, "f16", 0.0, 1), (2, 64, 64, "bf16", 0.0, 0),
    (16, 72, 65, "f16", 0.2, 0), (33, 100, 127, "bf16", 0.3, 0), (64, 33, 129, "f16", 0.0, 1), (127, 256, 255, "bf16", 0.0, 0),
    (128, 40, 256, "f16", 0.1, 0), (129, 520, 257, "bf16", 0.2, 0), (257, 129, 1000, "f16", 0.3, 3), (300, 48, 2049, "bf16", 0.0, 0),
    (130, 8, 5003, "f16", 0.5, 0), (40, 1000, 300, "bf16", 1.0, 0), (513, 264, 700, "f16", 0.1, 0), (1, 24, 9001, "bf16", 0.0, 0),
]


@pytest.mark.parametrize("rows,c,v,dtype,pad,shift", SIZES)
def test_labels(nnlib, rows, c, v, dtype, pad, shift):
    rng = np.random.default_rng(rows + c + v)
    x, w, targets, _ = W.loss_inputs(rng, rows, c, v, dtype, pad=pad)
    W.check_loss(W.loss_call(x, w, targets, None, dtype, 0.75, train=False, shift=shift), x, w, targets, None, dtype, 0.75)
    got = W.loss_call(x, w, targets, None, dtype, 0.75, alpha=0.5, grad_scale=16.0, inv=2.0 ** -3, shift=shift)
    W.check_loss(got, x, w, targets, None, dtype, 0.75, factor=8.0, inv=2.0 ** -3)


@pytest.mark.parametrize("k,dup", [(1, False), (2, False), (7, False), (64, False), (65, True), (300, True)])
@pytest.mark.parametrize("rows,c,v,dtype,pad,shift", SIZES[3:14:2])
def test_teacher(nnlib, rows, c, v, dtype, pad, shift, k, dup):
    rng = np.random.default_rng(rows + c + v + k)
    x, w, targets, teacher = W.loss_inputs(rng, rows, c, v, dtype, k=k, pad=pad, dup=dup)
    kind = "f32" if k % 2 else dtype
    got = W.loss_call(x, w, targets, teacher, dtype, 0.5, teacher_dtype=kind, alpha=4.0, shift=shift)
    W.check_loss(got, x, w, targets, teacher, dtype, 0.5, factor=4.0)
    got = W.loss_call(x, w, targets, teacher, dtype, 0.5, train=False, teacher_dtype=kind, shift=shift)
    W.check_loss(got, x, w, targets, teacher, dtype, 0.5)


@pytest.mark.parametrize("rows,c,v,dtype,pad,shift", [SIZES[5], SIZES[8], SIZES[10]])
@pytest.mark.parametrize("wide", [True, False], ids=["f32", "16 bits"])
def test_added_to_dw(nnlib, rows, c, v, dtype, pad, shift, wide):
    rng = np.random.default_rng(rows)
    x, w, targets, _ = W.loss_inputs(rng, rows, c, v, dtype, pad=pad)
    kind = "f32" if wide else dtype
    dw0 = U.normal(rng, (v, c), dtype, 0.1)
    got = W.loss_call(x, w, targets, None, dtype, dw_dtype=kind, dw0=dw0, shift=shift)
    W.check_loss(got, x, w, targets, None, dtype, dw_dtype=kind, dw0=dw0)
    W.check_loss(W.loss_call(x, w, targets, None, dtype, dw_dtype=kind, shift=shift), x, w, targets, None, dtype, dw_dtype=kind)


def test_without_dw_and_in_place(nnlib):
    rng = np.random.default_rng(2)
    x, w, targets, _ = W.loss_inputs(rng, 70, 48, 333, "f16", pad=0.2)
    W.check_loss(W.loss_call(x, w, targets, None, "f16", want_dw=False), x, w, targets, None, "f16")
    W.check_loss(W.loss_call(x, w, targets, None, "f16", in_place=True), x, w, targets, None, "f16")


def test_rows_that_do_not_count_hold_anything(nnlib):
    """NaN and inf in the x of padded rows and in a teacher's logits for padding touch nothing."""
    rng = np.random.default_rng(3)
    x, w, targets, teacher = W.loss_inputs(rng, 90, 40, 500, "bf16", k=6, pad=0.3)
    idle = targets[:, 0] != np.clip(targets[:, 0], 0, 499)
    assert idle.any()
    x[idle] = np.nan
    teacher[idle] = np.inf
    teacher[~idle, 3] = -np.inf  # one entry is masked
    teacher[5] = -np.inf         # a row's are all
    x[5] = np.inf
    got = W.loss_call(x, w, targets, teacher, "bf16")
    masked = np.where(idle[:, None], 0.0, teacher)
    W.check_loss(got, x, w, targets, masked, "bf16")
    assert np.isfinite(got["dw"].f64()).all()
    x, w, targets, _ = W.loss_inputs(rng, 90, 40, 500, "f16", pad=0.3)
    idle = targets[:, 0] != np.clip(targets[:, 0], 0, 499)
    x[idle] = np.inf
    W.check_loss(W.loss_call(x, w, targets, None, "f16"), x, w, targets, None, "f16")


def test_nan_and_infinite_logits(nnlib):
    """A NaN in a row that counts: its loss and gradients are NaN, the other rows' are not."""
    rng = np.random.default_rng(4)
    x, w, targets, _ = W.loss_inputs(rng, 20, 16, 300, "f16")
    clean = W.loss_call(x, w, targets, None, "f16")
    x[7, 3] = np.nan
    t = U.torch()
    flag = t.zeros(1, dtype=t.int32, device="cuda")
    got = W.loss_call(x, w, targets, None, "f16", flag=flag)
    assert np.isnan(got["loss"].f64()[7]) and np.isnan(got["dx"].f64()[7]).all() and int(flag) == 1
    rest = np.arange(20) != 7
    for key in ("loss", "lse", "dx"):
        assert np.array_equal(got[key].f64()[rest], clean[key].f64()[rest])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_sure_rows(nnlib, dtype):
    """Logits hundreds apart: p is 1 or 0, and the loss 0 or the difference."""
    c, v = 8, 600
    w = np.zeros((v, c))
    w[:, 0] = np.linspace(-1, 1, v)
    w = U.round16(dtype)(w)
    x = np.zeros((5, c))
    x[:, 0] = [0.0, 200.0, -200.0, 3.0, 200.0]
    targets = np.array([[3], [v - 1], [0], [v // 2], [0]])
    got = W.loss_call(x, w, targets, None, dtype)
    W.check_loss(got, x, w, targets, None, dtype)


def test_small_gradients_keep_their_bits(nnlib):
    """In fp16 a softmax value of 1 / v lies far below the smallest normal number."""
    rng = np.random.default_rng(9)
    v, c, rows = 60000, 16, 8
    w, x = U.normal(rng, (v, c), "f16", 0.01), U.normal(rng, (rows, c), "f16", 0.01)
    targets = np.full((rows, 1), 5)
    got = W.loss_call(x, w, targets, None, "f16", dw_dtype="f32", grad_scale=1024.0, inv=2.0 ** -10)
    o = V.cross_entropy(x, w, targets)
    _, dw = V.gradients(o, w, 1.0, 1.0)
    others = np.arange(v) != 5
    err = np.linalg.norm(got["dw"].f64()[others] - dw[others]) / np.linalg.norm(dw[others])
    assert err <= 2.0 ** -11 * 1.2  # one rounding of each p, and the exponentials' storage


def test_same_bits(nnlib):
    rng = np.random.default_rng(10)
    x, w, targets, _ = W.loss_inputs(rng, 500, 72, 3000, "bf16")
    first = W.loss_call(x, w, targets, None, "bf16")
    for _ in range(3):
        again = W.loss_call(x, w, targets, None, "bf16")
        for key in ("loss", "lse", "dx", "dw"):
            assert U.torch().equal(first[key].host(), again[key].host())


def test_flag(nnlib):
    """dx past fp16's range sets the flag; so does dw; finite ones do not."""
    t = U.torch()
    rng = np.random.default_rng(11)
    x, w, targets, _ = W.loss_inputs(rng, 30, 24, 100, "f16")
    for scale, kind, want in ((1.0, "f16", 0), (2.0 ** 20, "f32", 1)):
        flag = t.zeros(1, dtype=t.int32, device="cuda")
        W.loss_call(x, w, targets, None, "f16", grad_scale=scale, dw_dtype=kind, flag=flag)
        assert int(flag) == want
    flag = t.zeros(1, dtype=t.int32, device="cuda")
    W.loss_call(x * 0.0, w * 0.0, targets, None, "f16", dw0=np.full((100, 24), np.inf), dw_dtype="f16", flag=flag)
    assert int(flag) == 1


def test_gradient_by_differences(nnlib):
    """d loss / d w and d loss / d x along a random direction, from the kernel's own losses (fp32, the step's error is
    its square times a third derivative below 1)."""
    rng = np.random.default_rng(12)
    rows, c, v = 40, 24, 200
    x, w, targets, teacher = W.loss_inputs(rng, rows, c, v, "f16", k=5)
    got = W.loss_call(x, w, targets, teacher, "f16", dw_dtype="f32")
    gx, gw = got["dx"].f64(), got["dw"].f64()
    h = 2.0 ** -4
    # directions whose steps are exact in fp16
    ux, uw = rng.integers(-1, 2, x.shape) * 2.0 ** -3, rng.integers(-1, 2, w.shape) * 2.0 ** -5
    x, w = np.round(x * 256) / 256, np.round(w * 1024) / 1024
    got = W.loss_call(x, w, targets, teacher, "f16", dw_dtype="f32")
    gx, gw = got["dx"].f64(), got["dw"].f64()

    def loss(a, b):
        return W.loss_call(x + a * ux, w + b * uw, targets, teacher, "f16", train=False)["loss"].f64().sum()

    for a, b, along in ((h, 0.0, (gx * ux).sum()), (0.0, h, (gw * uw).sum())):
        slope = (loss(a, b) - loss(-a, -b)) / (2 * h)
        # curvature of third order: each row's logits move by s = h |u . w| at most, the remainder is s^3 / 6 / h
        s = h * (np.abs(ux) @ np.abs(w).T).max() if a else h * (np.abs(x) @ np.abs(uw).T).max()
        rounding = rows * 2.0 ** -18 / h + 2.0 ** -10 * (np.abs(gx * ux).sum() if a else np.abs(gw * uw).sum())
        assert abs(slope - along) <= rows * s ** 3 / 6 / h + rounding


def test_nothing(nnlib):
    t = U.torch()
    none = np.zeros((0, 8))
    w = np.ones((20, 8))
    got = W.loss_call(none, w, np.zeros((0, 1)), None, "f16")
    assert np.all(got["dw"].f64() == 0)
    got = W.loss_call(none, w, np.zeros((0, 1)), None, "f16", dw0=np.ones((20, 8)))
    assert np.all(got["dw"].f64() == 1)
    t.cuda.synchronize()


@pytest.mark.parametrize("rows,c,v", [(700, 136, 1500), (1100, 64, 700)])
def test_handle(nnlib, rows, c, v):
    """The handle's calls are the C entry points', on another stream too."""
    t = U.torch()
    rng = np.random.default_rng(rows)
    x, w, targets, teacher = W.loss_inputs(rng, rows, c, v, "bf16", k=3, pad=0.1)
    ref = W.loss_call(x, w, targets, teacher, "bf16", 0.5)
    bf = lambda a: t.from_numpy(a).to(t.bfloat16).cuda()  # noqa: E731
    op = nc.CrossEntropy(rows, c, v, dtype=nc.NNCONV_BF16, logit_scale=0.5, k=3)
    X, Wt, T, Q = bf(x), bf(w), t.from_numpy(targets.astype(np.int32)).cuda(), t.from_numpy(teacher).float().cuda()
    loss, lse, dx, dw = t.empty(rows, device="cuda"), t.empty(rows, device="cuda"), t.empty_like(X), t.empty_like(Wt)
    other = t.cuda.Stream()
    t.cuda.synchronize()
    with t.cuda.stream(other):
        op.train(X, Wt, T, loss, dx, dw, lse=lse, teacher=Q)
    other.synchronize()
    for a, key in ((loss, "loss"), (lse, "lse"), (dx, "dx"), (dw, "dw")):
        assert t.equal(a.cpu(), ref[key].host())
    op.fwd(X, Wt, T, loss, teacher=Q)
    assert t.allclose(loss.cpu(), ref["loss"].host(), rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("rows,c,v,dtype,k", [(600, 520, 20000, "bf16", None), (2100, 1100, 8300, "f16", None), (1500, 300, 3000, "f16", 9),
                                              (1100, 64, 2001, "bf16", None), (1409, 77, 1500, "f16", None)])
def test_large_tiles(nnlib, rows, c, v, dtype, k):
    """Sizes whose products take 256 x 256 and 128 x 128 tiles, one and several a compute unit, and split reductions."""
    rng = np.random.default_rng(rows)
    x, w, targets, teacher = W.loss_inputs(rng, rows, c, v, dtype, k=k, pad=0.1)
    got = W.loss_call(x, w, targets, teacher, dtype, 1.0)
    W.check_loss(got, x, w, targets, teacher, dtype, 1.0)
    again = W.loss_call(x, w, targets, teacher, dtype, 1.0, train=False)
    assert np.allclose(again["loss"].f64(), got["loss"].f64(), rtol=1e-6, atol=1e-5)


@pytest.mark.parametrize("scale", [-0.75, 2.0 ** -20, 3.0])
def test_logit_scales(nnlib, scale):
    rng = np.random.default_rng(14)
    x, w, targets, teacher = W.loss_inputs(rng, 60, 40, 300, "f16", k=4)
    W.check_loss(W.loss_call(x, w, targets, teacher, "f16", scale), x, w, targets, teacher, "f16", scale)
    W.check_loss(W.loss_call(x, w, targets[:, :1], None, "f16", scale), x, w, targets[:, :1], None, "f16", scale)


def test_pieces(nnlib):
    """A vocabulary of which 256 rows fill the workspace's exponentials: dw joins over two pieces."""
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(3)
    rows, c, v = 300, 8, 2 ** 21
    w = t.randn((v, c), generator=g, device="cuda").half()
    x = t.randn((rows, c), generator=g, device="cuda").half()
    target = t.randint(0, v, (rows,), generator=g, device="cuda", dtype=t.int32)
    target[7], target[299] = -1, v - 1
    op = nc.CrossEntropy(rows, c, v)
    loss, lse, dx = t.empty(rows, device="cuda"), t.empty(rows, device="cuda"), t.empty_like(x)
    dw, dw32 = t.empty_like(w), t.full((v, c), 0.25, device="cuda")
    op.train(x, w, target, loss, dx, dw, lse=lse, alpha=2.0 ** 12)
    op.train(x, w, target, loss, dx, dw32, alpha=2.0 ** 12, accumulate=1)
    live = target >= 0
    z = x.double() @ w.double().t()
    ref_lse = t.logsumexp(z, 1) * live
    at = target.clamp(min=0).long()
    ref_loss = (ref_lse - z.gather(1, at[:, None])[:, 0]) * live
    # 2^-24 of a logit of 8 products and of lse, sums of 2^21 terms in chains of at most 400
    assert float((lse - ref_lse).abs().max()) < 500 * 2.0 ** -24 + 20 * 2.0 ** -24 * float(z.abs().max())
    assert float((loss - ref_loss).abs().max()) < 500 * 2.0 ** -24 + 40 * 2.0 ** -24 * float(z.abs().max())
    p = z.sub_(ref_lse[:, None]).exp_().mul_(live[:, None])
    p[t.arange(rows, device="cuda"), at] -= live.double()
    p *= 2.0 ** 12
    ref_dx, ref_dw = p @ w.double(), p.t() @ x.double()
    # one rounding of each gradient of a logit, its storage before, and one of the result
    for got, ref, mag in ((dx, ref_dx, p.abs() @ w.double().abs()), (dw, ref_dw, p.abs().t() @ x.double().abs()),
                          (dw32 - 0.25, ref_dw, p.abs().t() @ x.double().abs() + 2.0 ** -12)):
        bound = (2.0 ** -11 + 2.0 ** -12 + 2.0 ** -15) * mag + 2.0 ** -11 * ref.abs() + 2.0 ** -23 + 2.0 ** 12 * 2.0 ** -28
        assert bool(((got.double() - ref).abs() <= bound).all())


def test_a_teachers_nan(nnlib):
    """A NaN among a teacher's logits, with any bits, is the row's and no other's."""
    t = U.torch()
    rng = np.random.default_rng(15)
    x, w, targets, teacher = W.loss_inputs(rng, 20, 24, 100, "bf16", k=4)
    X, Wt = (t.from_numpy(a).bfloat16().cuda() for a in (x, w))
    T = t.from_numpy(targets.astype(np.int32)).cuda()
    op = nc.CrossEntropy(20, 24, 100, dtype=nc.NNCONV_BF16, k=4)
    got = []
    for bits in (None, 0x7FC0DEAD, 0x7FC00000, 0x7F800001):
        Q = t.from_numpy(teacher).float()
        if bits is not None:
            Q.view(t.int32)[6, 2] = bits
        loss, dx = t.empty(20, device="cuda"), t.empty_like(X)
        op.train(X, Wt, T, loss, dx, teacher=Q.cuda())
        got.append((loss.cpu(), dx.cpu()))
    rest = t.arange(20) != 6
    for loss, dx in got[1:]:
        assert bool(loss[6].isnan()) and bool(dx[6].isnan().all())
        assert t.equal(loss[rest], got[0][0][rest]) and t.equal(dx[rest], got[0][1][rest])


@pytest.mark.parametrize("train", [False, True])
def test_many_short_rows(nnlib, train):
    """More rows than one launch's tiles of a small vocabulary, and forward calls of several pieces."""
    t = U.torch()
    rows, c, v = 70001, 8, 70
    g = t.Generator(device="cuda").manual_seed(1)
    x, w = t.randn((rows, c), generator=g, device="cuda").half(), t.randn((v, c), generator=g, device="cuda").half()
    target = t.randint(-1, v, (rows,), generator=g, device="cuda", dtype=t.int32)
    op = nc.CrossEntropy(rows, c, v)
    loss, dx, dw = t.empty(rows, device="cuda"), t.empty_like(x), t.empty(v, c, device="cuda")
    if train:
        op.train(x, w, target, loss, dx, dw)
    else:
        op.fwd(x, w, target, loss)
    live = target >= 0
    z = t.log_softmax(x.double() @ w.double().t(), 1)
    want = -z.gather(1, target.clamp(min=0).long()[:, None])[:, 0] * live
    assert float((loss - want).abs().max()) < 2.0 ** -18
    if train:
        dz = z.exp() * live[:, None]
        dz[t.arange(rows, device="cuda"), target.clamp(min=0).long()] -= live.double()
        # one rounding of dz, its storage before, one of the result
        assert bool(((dx.double() - dz @ w.double()).abs() <= 2.0 ** -9.5 * (dz.abs() @ w.double().abs()) + 2.0 ** -20).all())
        mag = dz.abs().t() @ x.double().abs()
        assert bool(((dw.double() - dz.t() @ x.double()).abs() <= 2.0 ** -10 * mag).all())


def test_forward_in_pieces(nnlib):
    """A vocabulary whose statistics of all rows pass the workspace's share: pieces of 256 rows and more."""
    t = U.torch()
    rows, c, v = 9000, 8, 400000  # 1024 rows a piece
    g = t.Generator(device="cuda").manual_seed(2)
    x, w = t.randn((rows, c), generator=g, device="cuda").bfloat16(), t.randn((v, c), generator=g, device="cuda").bfloat16()
    target = t.randint(0, v, (rows,), generator=g, device="cuda", dtype=t.int32)
    op = nc.CrossEntropy(rows, c, v, dtype=nc.NNCONV_BF16)
    loss, lse = t.empty(rows, device="cuda"), t.empty(rows, device="cuda")
    op.fwd(x, w, target, loss, lse=lse)
    for r in range(0, rows, 499):
        z = x[r].double() @ w.double().t()
        assert abs(float(lse[r] - t.logsumexp(z, 0))) < 2.0 ** -17
        assert abs(float(loss[r] - t.logsumexp(z, 0) + z[target[r]])) < 2.0 ** -16
