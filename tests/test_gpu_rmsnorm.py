"""nnconv_rmsnorm_* against the fp64 oracle.

Bounds: a 16-bit output is one rounding from the exact value, plus fp32
arithmetic: the sum of squares of c terms added in chains of at most
c / 64 + 6 is off by (c / 64 + 6) 2^-24 at most, half of which reaches rstd, and
y takes four more roundings.  For c up to 40001 that is below 2.5e-5 relative;
SLACK grows with c accordingly.  Gradient sums are bounded by the same share of
the sum of their terms' magnitudes."""
import numpy as np
import pytest

from oracle import sequence as S
from paper_2102_06725_amd import nnconv as nc

import sequence_util as U

pytestmark = pytest.mark.gpu
EPS = 1e-6


def slack(c, rows=0):
    return (c / 64 + rows / 16 + 24) * 2.0 ** -24


CASES = [  # rows, c, dtype, residual, where the sum goes, elements past 16-byte alignment
    (1, 1, "f16", True, "own", 0), (3, 2, "bf16", False, None, 0), (5, 7, "f16", True, "residual", 1),
    (70, 8, "bf16", True, "x", 0), (33, 9, "f16", False, None, 0), (129, 63, "bf16", True, "own", 0),
    (64, 64, "f16", True, "own", 0), (17, 65, "f16", True, "own", 3), (300, 72, "bf16", True, None, 0),
    (41, 200, "f16", True, "own", 0), (1000, 256, "bf16", True, "residual", 0), (9, 256, "f16", True, "own", 1),
    (5, 511, "f16", True, "own", 0), (6, 512, "bf16", True, "own", 0), (7, 520, "f16", False, None, 0),
    (11, 1000, "bf16", True, "own", 0), (30, 1152, "f16", True, "own", 0), (3, 2047, "bf16", True, "own", 0),
    (8, 2048, "bf16", True, "own", 0), (2, 2056, "f16", True, "x", 0), (5, 4096, "f16", True, "own", 0),
    (5, 4100, "bf16", True, "own", 5), (2, 8192, "f16", True, "own", 0), (3, 8200, "bf16", True, "own", 0),
    (2, 16384, "bf16", True, "own", 0), (2, 16392, "f16", True, "own", 0), (1, 40001, "f16", True, "own", 0),
    (5000, 96, "f16", True, "own", 0), (1, 2048, "f16", True, "own", 0),
    # every team of threads with a last vector that is shared, in place, and enough rows for several a team
    (700, 771, "bf16", True, "residual", 0), (600, 1025, "f16", True, "x", 0), (300, 3001, "f16", True, "own", 1),
    (140, 7777, "bf16", True, "residual", 0), (140, 9001, "f16", True, "x", 0),
    # rows of one to four vectors, more of them than a workgroup takes at once
    (5003, 8, "f16", True, "residual", 1), (5003, 9, "bf16", True, "x", 0), (2111, 15, "f16", True, "own", 0),
    (2111, 16, "bf16", True, "residual", 0), (2111, 17, "f16", True, "x", 3), (1301, 24, "bf16", True, "own", 0),
    (1301, 31, "f16", True, "residual", 0), (1301, 32, "bf16", False, None, 0), (1301, 33, "f16", True, "own", 0),
]


def inputs(rows, c, dtype, residual, seed=0):
    rng = np.random.default_rng(seed + rows * 100003 + c)
    loud = 1.0 + 20.0 * (rng.random(c) < 0.02)
    return (U.normal(rng, (rows, c), dtype), U.normal(rng, (rows, c), dtype, 2.0) * 1.0 if residual else None,
            (1.0 + 0.3 * rng.standard_normal(c)).astype(np.float32).astype(np.float64) * loud, rng)


def forward(rows, c, dtype, x, res, gain, where, shift, group=None, stream=None, eps=EPS):
    """Buffers of one forward call; group None: a 16-bit y."""
    X, R = U.Buf(x, dtype, shift=shift), None if res is None else U.Buf(res, dtype, shift=shift)
    G = U.Buf(gain, "f32")
    Sm = {"own": lambda: U.Buf(dtype=dtype, shape=(rows, c), shift=shift), "x": lambda: X, "residual": lambda: R,
          None: lambda: None}[where]()
    rstd = U.Buf(dtype="f32", shape=(rows,))
    d = nc.nnconv_rmsnorm_desc(rows, c, U.CODE[dtype], group or 0, eps)
    if group is None:
        Y, SC = U.Buf(dtype=dtype, shape=(rows, c), shift=shift), None
        nc.check(nc.nnconv_rmsnorm_fwd(d, X.data_ptr(), U.ptr(R), G.data_ptr(), U.ptr(Sm), Y.data_ptr(), rstd.data_ptr(), stream))
    else:
        Y = U.Buf(dtype="e4m3", shape=(rows, c), shift=shift)
        SC = U.Buf(dtype="f32", shape=(rows, -(-c // group) if group else 1))
        nc.check(nc.nnconv_rmsnorm_fwd_q8(d, X.data_ptr(), U.ptr(R), G.data_ptr(), U.ptr(Sm), Y.data_ptr(), SC.data_ptr(),
                                          rstd.data_ptr(), stream))
    return dict(X=X, R=R, G=G, S=Sm, Y=Y, SC=SC, rstd=rstd, desc=d)


@pytest.mark.parametrize("rows,c,dtype,residual,where,shift", CASES)
def test_forward_and_backward(nnlib, rows, c, dtype, residual, where, shift):
    x, res, gain, rng = inputs(rows, c, dtype, residual)
    b = forward(rows, c, dtype, x, res, gain, where, shift)
    U.torch().cuda.synchronize()
    r, rstd, y = S.rmsnorm_fwd(x, res, gain, EPS, U.round16(dtype))
    if where is not None:
        assert np.array_equal(b["S"].f64(), r)
    if where != "x":
        assert np.array_equal(b["X"].f64(), x)
    U.close32(b["rstd"].f64(), rstd, slack(c) * rstd)
    U.close16(b["Y"].f64(), y, dtype, slack(c) * np.abs(y))

    # backward on the stored sum, with and without what arrives along the residual stream
    dy, dsum = U.normal(rng, (rows, c), dtype), U.normal(rng, (rows, c), dtype)
    old = rng.standard_normal(c).astype(np.float32).astype(np.float64)
    R = U.Buf(r, dtype, shift=shift)
    rs = rstd.astype(np.float32).astype(np.float64)
    RS = U.Buf(rs, "f32")
    st, nb = nc.nnconv_rmsnorm_workspace_size(b["desc"])
    ws = U.Buf(dtype="u8", shape=(nb,))
    flag = U.torch().zeros(1, dtype=U.torch().int32, device="cuda")
    for along, place, acc in ((None, "own", 0), (dsum, "own", 1), (dsum, "dsum", 0), (None, "dy", 1)):
        DY, DS = U.Buf(dy, dtype, shift=shift), None if along is None else U.Buf(along, dtype, shift=shift)
        DX = {"own": lambda: U.Buf(dtype=dtype, shape=(rows, c), shift=shift), "dsum": lambda: DS, "dy": lambda: DY}[place]()
        DG = U.Buf(old, "f32")
        nc.check(nc.nnconv_rmsnorm_bwd(b["desc"], R.data_ptr(), DY.data_ptr(), U.ptr(DS), b["G"].data_ptr(), RS.data_ptr(),
                                       DX.data_ptr(), DG.data_ptr(), 0.125, acc, flag.data_ptr(), ws.data_ptr(), nb, None))
        U.torch().cuda.synchronize()
        dx, dgain = S.rmsnorm_bwd(r, rs, gain, dy, along)
        xh = r * rs[:, None]
        p = np.abs(dy * gain)
        terms = rs[:, None] * (p + np.abs(xh) * (p * np.abs(xh)).mean(axis=1, keepdims=True)) + (0 if along is None else np.abs(along))
        U.close16(DX.f64(), dx, dtype, slack(c) * terms)
        want = dgain * 0.125 + (old if acc else 0.0)
        U.close32(DG.f64(), want, slack(24, rows) * (np.abs(dy * xh).sum(axis=0) * 0.125 + np.abs(old)))
        ws.host()
        assert int(flag.item()) == 0
    # without dgain no workspace is asked for
    DX = U.Buf(dtype=dtype, shape=(rows, c), shift=shift)
    DY = U.Buf(dy, dtype, shift=shift)
    nc.check(nc.nnconv_rmsnorm_bwd(b["desc"], R.data_ptr(), DY.data_ptr(), None, b["G"].data_ptr(), RS.data_ptr(), DX.data_ptr(),
                                   None, 1.0, 0, None, None, 0, None))
    dx, _ = S.rmsnorm_bwd(r, rs, gain, dy)
    U.close16(DX.f64(), dx, dtype, slack(c) * terms)


Q8 = [(r, c, dt, res, sh, g) for r, c, dt, res, sh in
      [(1, 1, "f16", True, 0), (9, 33, "bf16", True, 0), (70, 64, "f16", False, 0), (13, 100, "f16", True, 1),
       (5, 256, "bf16", True, 0), (40, 771, "bf16", True, 0), (6, 1000, "f16", True, 0), (3, 2048, "bf16", True, 0),
       (3, 4096, "f16", True, 0), (2, 4104, "f16", True, 3), (2, 8192, "bf16", True, 0), (2, 20000, "bf16", True, 0),
       (601, 8, "f16", True, 1), (601, 9, "bf16", True, 0), (601, 16, "f16", False, 0), (601, 23, "bf16", True, 0),
       (601, 32, "f16", True, 0)]
      for g in (0, 32, 64, 128)]


@pytest.mark.parametrize("rows,c,dtype,residual,shift,group", Q8)
def test_eight_bits(nnlib, rows, c, dtype, residual, shift, group):
    x, res, gain, _ = inputs(rows, c, dtype, residual)
    b = forward(rows, c, dtype, x, res, gain, "own" if residual else None, shift, group=group)
    U.torch().cuda.synchronize()
    r, rstd, y = S.rmsnorm_fwd(x, res, gain, EPS, U.round16(dtype))
    if residual:
        assert np.array_equal(b["S"].f64(), r)
    U.close32(b["rstd"].f64(), rstd, slack(c) * rstd)
    s = S.quantise_scales(y, group)
    got = b["SC"].f64()
    U.close32(got, s, slack(c) * s)
    per = np.repeat(got, group or c, axis=1)[:, :c]
    q = b["Y"].f64()
    assert np.abs(q).max() <= 448.0
    # half a unit of 3 mantissa bits, or of the subnormals' 2^-9
    assert np.all(np.abs(q * per - y) <= np.maximum(np.abs(y) * 2.0 ** -4, per * 2.0 ** -10) * 1.0001 + 4 * slack(c) * np.abs(y))
    # the largest of each group has the largest code
    top = np.stack([np.abs(q[:, i:i + (group or c)]).max(axis=1) for i in range(0, c, group or c)], axis=1)
    assert np.all(top[s > 0] == 448.0)


@pytest.mark.parametrize("c", [8, 100, 2048, 20000])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rows_do_not_touch_each_other(nnlib, c, dtype):
    """Zero rows, infinities, NaNs and the largest values stay in their rows."""
    x, res, gain, _ = inputs(12, c, dtype, True)
    top = float(U.torch().finfo(U.tdtype(dtype)).max)
    x[1], res[1] = 0.0, 0.0
    x[3, c // 2] = np.inf
    x[5, 0] = np.nan
    res[7, c - 1] = -np.inf
    if dtype == "f16":
        x[8], res[8] = top, -1.0
        x[9], res[9] = top, top       # the sum passes the type's range
    with np.errstate(all="ignore"):
        r, rstd, y = S.rmsnorm_fwd(x, res, gain, EPS, U.round16(dtype))
    for group in (None, 0, 64):
        b = forward(12, c, dtype, x, res, gain, "own", 0, group=group)
        assert np.array_equal(b["S"].f64(), r, equal_nan=True)
        if group is None:
            U.close16(b["Y"].f64(), y, dtype, slack(c) * np.nan_to_num(np.abs(y), posinf=0.0))
            continue
        q, sc = b["Y"].f64(), b["SC"].f64()
        assert np.array_equal(np.isnan(q), np.isnan(y))
        per = np.repeat(sc, group or c, axis=1)[:, :c]
        fine = np.isfinite(y)
        assert np.all(np.abs(q * per - y)[fine] <= (np.maximum(np.abs(y) * 2.0 ** -4, per * 2.0 ** -10) * 1.001)[fine])
        assert not q[1].any() and not sc[1].any()


def test_gradient_of_infinite_rows_sets_the_flag(nnlib):
    t = U.torch()
    rows, c = 40, 64
    x, _, gain, rng = inputs(rows, c, "f16", False)
    dy = U.normal(rng, (rows, c), "f16")
    d = nc.nnconv_rmsnorm_desc(rows, c, U.CODE["f16"], 0, EPS)
    st, nb = nc.nnconv_rmsnorm_workspace_size(d)
    for bad in (np.inf, np.nan):
        dy2 = dy.copy()
        dy2[17, 5] = bad
        _, rstd, _ = S.rmsnorm_fwd(x, None, gain, EPS, None)
        b = [U.Buf(v, k) for v, k in ((x, "f16"), (dy2, "f16"), (gain, "f32"), (rstd, "f32"))]
        DX, DG, ws = U.Buf(dtype="f16", shape=(rows, c)), U.Buf(dtype="f32", shape=(c,)), U.Buf(dtype="u8", shape=(nb,))
        flag = t.zeros(1, dtype=t.int32, device="cuda")
        nc.check(nc.nnconv_rmsnorm_bwd(d, b[0].data_ptr(), b[1].data_ptr(), None, b[2].data_ptr(), b[3].data_ptr(), DX.data_ptr(),
                                       DG.data_ptr(), 1.0, 0, flag.data_ptr(), ws.data_ptr(), nb, None))
        got = DG.f64()
        assert int(flag.item()) == 1 and not np.isfinite(got[5]) and np.isfinite(np.delete(got, 5)).all()
        dx = DX.f64()
        assert not np.isfinite(dx[17]).all() and np.isfinite(np.delete(dx, 17, axis=0)).all()


def test_no_rows(nnlib):
    """Nothing to normalise: a gradient that is overwritten is zero, one that is added to stays."""
    d = nc.nnconv_rmsnorm_desc(0, 70, U.CODE["f16"], 0, EPS)
    st, nb = nc.nnconv_rmsnorm_workspace_size(d)
    old = np.arange(70.0)
    one = U.Buf(np.ones(70), "f16")
    g = U.Buf(np.ones(70), "f32")
    for acc in (0, 1):
        DG, ws = U.Buf(old, "f32"), U.Buf(dtype="u8", shape=(max(nb, 4),))
        nc.check(nc.nnconv_rmsnorm_bwd(d, one.data_ptr(), one.data_ptr(), None, g.data_ptr(), g.data_ptr(), one.data_ptr(),
                                       DG.data_ptr(), 1.0, acc, None, ws.data_ptr(), nb, None))
        assert np.array_equal(DG.f64(), old if acc else 0 * old)


def test_other_stream_graph_and_repeats(nnlib):
    """Queued on the caller's stream; captured and replayed; bitwise the same each time."""
    t = U.torch()
    rows, c = 500, 1152
    x, res, gain, rng = inputs(rows, c, "bf16", True)
    dy = U.normal(rng, (rows, c), "bf16")
    X, R, DY, G = U.Buf(x, "bf16"), U.Buf(res, "bf16"), U.Buf(dy, "bf16"), U.Buf(gain, "f32")
    op = nc.RMSNorm(rows, c, dtype=U.CODE["bf16"], eps=EPS)
    out = {k: U.Buf(dtype="bf16", shape=(rows, c)) for k in ("sum", "y", "dx")}
    rstd, dgain = U.Buf(dtype="f32", shape=(rows,)), U.Buf(dtype="f32", shape=(c,))
    ws_dev = t.empty(1, device="cuda")
    DY.device = R.device = X.device = out["sum"].device = ws_dev.device

    def both(stream=None):
        op.fwd(X, G, out["y"], residual=R, sum=out["sum"], rstd=rstd, stream=stream)
        op.bwd(out["sum"], DY, G, rstd, out["dx"], dgain, stream=stream)

    def bits():
        return [v.host().view(t.uint8).clone() for v in list(out.values()) + [rstd, dgain]]
    both()
    t.cuda.synchronize()
    first = bits()
    s = t.cuda.Stream()
    with t.cuda.stream(s):
        both(s.cuda_stream)
    s.synchronize()
    assert all(bool((a == b).all()) for a, b in zip(first, bits()))
    g = t.cuda.CUDAGraph()
    with t.cuda.graph(g):
        both()
    for k in range(3):
        for v in list(out.values()) + [rstd, dgain]:
            v.buf[v.lo:v.lo + v.nbytes] = 0
        t.cuda.synchronize()
        g.replay()
        t.cuda.synchronize()
        assert all(bool((a == b).all()) for a, b in zip(first, bits())), "replay %d" % k


def test_offsets_past_32_bits(nnlib):
    """Rows past 2^32 bytes and 2^31 elements: the bits of calls on the last rows alone."""
    t = U.torch()
    rows, c, last = 550001, 4104, 300  # 2.26e9 elements
    g = t.Generator(device="cuda").manual_seed(3)
    x = t.empty((rows, c), dtype=t.float16, device="cuda")
    for k in range(0, rows, 50000):
        x[k:k + 50000] = t.randn((min(50000, rows - k), c), generator=g, device="cuda")
    gain = t.rand(c, generator=g, device="cuda")

    def three(v):
        n = v.shape[0]
        op = nc.RMSNorm(n, c, dtype=nc.NNCONV_F16, group=64)
        y, rstd = t.empty_like(v), t.empty(n, device="cuda")
        op.fwd(v, gain, y, rstd=rstd)
        q, scales = t.empty((n, c), dtype=t.uint8, device="cuda"), t.empty((n, -(-c // 64)), device="cuda")
        op.fwd_q8(v, gain, q, scales)
        dx = t.empty_like(v)
        op.bwd(v, y, gain, rstd, dx, dsum=v)
        return [k[-last:].clone() for k in (y, rstd, q, scales, dx)]
    for a, b in zip(three(x), three(x[-last:].clone())):
        assert bool((a.view(t.uint8) == b.view(t.uint8)).all())
