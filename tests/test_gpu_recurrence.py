"""nnconv_recurrence_* against the fp64 oracle.

Bounds, with u = 2^-24.  A gate's exponential has a relative error of (|z| + 4) u
at most (the argument's rounding, and the instruction's).  Its error moves a and
1 - a by opposite amounts, so h, a mean of h and x, moves by at most that share
of the largest |h|, |x| that it averages.  Every step's rounding adds u |h|, and
is forgotten at the rate 1 - a: at most min(t, 1 / min(1 - a)) of them
count.  Splitting the tokens and joining the parts adds a few roundings of the
same kind, hence the factors 2 and 4 below.  The gradients obey the same recurrence
in the other direction, on magnitudes that are summed here term by term."""
import numpy as np
import pytest

from oracle import sequence as S
from paper_2102_06725_amd import nnconv as nc

import sequence_util as U

pytestmark = pytest.mark.gpu
ULP = 2.0 ** -24


class Case:
    """Inputs of a geometry and the oracle's answer for them."""

    def __init__(self, n, t, c, dtype, with_g=True, with_bias=True, lengths=None, carry=True, pad=0, pady=0, shift=0, seed=0,
                 bias_top=7.0):
        rng = np.random.default_rng(seed + n * 7 + t * 1009 + c)
        self.n, self.t, self.c, self.dtype, self.lengths, self.shift = n, t, c, dtype, lengths, shift
        self.ld, self.ldy = c + pad, c + pady
        mk = lambda: U.normal(rng, (n, t, c), dtype)  # noqa: E731
        self.x, self.f, self.g = mk(), mk(), mk() if with_g else None
        self.dy = mk()
        f32 = lambda v: v.astype(np.float32).astype(np.float64)  # noqa: E731
        self.bias = f32(rng.random(c) * bias_top) if with_bias else None
        self.h0 = f32(rng.standard_normal((n, c))) if carry else None
        self.dht = f32(rng.standard_normal((n, c))) if carry else None

    def desc(self):
        return nc.nnconv_recurrence_desc(self.n, self.t, self.c, U.CODE[self.dtype], self.ld, self.ldy)

    def wide(self, v, ld):
        """[n][t][c] in rows of ld elements; what lies between is NaN, which nothing may read."""
        if v is None:
            return None
        out = np.full((self.n, self.t, ld), np.nan)
        out[..., :self.c] = v
        return out

    def device(self, v, y=False):
        return None if v is None else U.Buf(self.wide(v, self.ldy if y else self.ld), self.dtype, shift=self.shift)

    def out(self, y=False):
        return U.Buf(dtype=self.dtype, shape=(self.n, self.t, self.ldy if y else self.ld), shift=self.shift)

    def narrow(self, b):
        """The written part of an output; the elements between rows have to be untouched."""
        v = b.host().view(U.torch().uint8).numpy().reshape(b.shape[:2] + (2 * b.shape[2],))
        assert np.all(v[..., 2 * self.c:] == 0xA5)
        return b.f64()[..., :self.c]

    def lens(self):
        return None if self.lengths is None else U.torch().tensor(self.lengths, dtype=U.torch().int32, device="cuda")

    # ---- the device's answer

    def forward(self, in_place=False, save=True, stream=None):
        d = self.desc()
        b = {k: self.device(getattr(self, k)) for k in ("x", "f", "g")}
        bias = None if self.bias is None else U.Buf(self.bias, "f32")
        h0 = None if self.h0 is None else U.Buf(self.h0, "f32")
        ht = h0 if in_place else U.Buf(dtype="f32", shape=(self.n, self.c))
        y = self.out(True)
        st, nb = nc.nnconv_recurrence_saved_size(d)
        nc.check(st)
        saved = U.Buf(dtype="f32", shape=(nb // 4,)) if save else None
        st, wb = nc.nnconv_recurrence_workspace_size(d, nc.NNCONV_FWD)
        nc.check(st)
        ws = U.Buf(dtype="u8", shape=(wb,))
        lens = self.lens()
        nc.check(nc.nnconv_recurrence_fwd(d, b["x"].data_ptr(), b["f"].data_ptr(), U.ptr(bias), U.ptr(b["g"]), U.ptr(lens),
                                          U.ptr(h0), y.data_ptr(), ht.data_ptr(), U.ptr(saved), ws.data_ptr(), wb, stream))
        U.torch().cuda.synchronize()
        ws.host()
        self.b, self.bias_b, self.saved = b, bias, saved
        return self.narrow(y), ht.f64()

    def backward(self, in_place=False, old=None):
        d = self.desc()
        dy, dht = self.device(self.dy, True), None if self.dht is None else U.Buf(self.dht, "f32")
        dx, df, dg = self.out(), self.out(), None if self.g is None else self.out()
        dh0 = dht if in_place else U.Buf(dtype="f32", shape=(self.n, self.c))
        dbias = U.Buf(dtype="f32", shape=(self.c,)) if old is None else U.Buf(old, "f32")
        st, wb = nc.nnconv_recurrence_workspace_size(d, nc.NNCONV_DGRAD)
        nc.check(st)
        ws = U.Buf(dtype="u8", shape=(wb,))
        lens = self.lens()
        flag = U.torch().zeros(1, dtype=U.torch().int32, device="cuda")
        nc.check(nc.nnconv_recurrence_bwd(d, self.b["x"].data_ptr(), self.b["f"].data_ptr(), U.ptr(self.bias_b),
                                          U.ptr(self.b["g"]), U.ptr(lens), self.saved.data_ptr(), dy.data_ptr(), U.ptr(dht),
                                          dx.data_ptr(), df.data_ptr(), U.ptr(dg), dh0.data_ptr(), dbias.data_ptr(), 0.25,
                                          int(old is not None), flag.data_ptr(), ws.data_ptr(), wb, None))
        U.torch().cuda.synchronize()
        ws.host()
        self.saved.host()
        return (self.narrow(dx), self.narrow(df), None if dg is None else self.narrow(dg), dh0.f64(), dbias.f64(), int(flag.item()))

    # ---- the oracle's, with bounds

    def check(self, in_place=False, old=None):
        y, ht = self.forward(in_place)
        ry, h = S.recurrence_fwd(self.x, self.f, self.bias, self.g, self.lengths, self.h0)
        a, b = S.gates(self.f, self.bias)
        z = np.abs(self.f + (0 if self.bias is None else self.bias)).max(initial=0.0)
        steps = min(self.t, float((1.0 / b).max(initial=1.0)))
        k = ULP * (z + 8 + 2 * steps)
        big = np.maximum(np.abs(h).max(axis=1), np.abs(self.x).max(axis=1, initial=0.0))[:, None]  # [n][1][c]
        sil = 1.0 if self.g is None else np.abs(self.g) / (1.0 + np.exp(-self.g))
        U.close16(y, ry, self.dtype, k * big * sil + 8 * ULP * np.abs(ry))
        U.close32(ht, h[:, -1], k * big[:, 0])

        got = self.backward(in_place, old)
        ref = S.recurrence_bwd(self.x, self.f, self.bias, self.dy, h, self.g, self.lengths, self.dht)
        # magnitudes: dmag_t bounds |dh_t| and every partial sum in it
        lens = S._lengths(self.lengths, self.n, self.t)
        sm = np.abs(self.dy) * sil
        dmag = np.zeros_like(self.x)
        carry = np.zeros((self.n, self.c)) if self.dht is None else np.abs(self.dht)
        for j in range(self.t - 1, -1, -1):
            live = np.array([j < l for l in lens])[:, None]
            dmag[:, j] = np.where(live, carry + sm[:, j], 0.0)
            carry = np.where(live, dmag[:, j] * a[:, j], carry)
        dbig = dmag.max(axis=1, initial=0.0)[:, None]
        k4 = ULP * (z + 16 + 4 * steps)
        U.close16(got[0], ref[0], self.dtype, k4 * dbig * b)
        bound = k4 * dbig * 4 * big * a * b
        U.close16(got[1], ref[1], self.dtype, bound)
        if self.g is not None:
            U.close16(got[2], ref[2], self.dtype, k4 * 2 * np.abs(self.dy) * big * (1 + np.abs(self.g)))
        U.close32(got[3], ref[3], k4 * np.maximum(dbig[:, 0], 0 if self.dht is None else np.abs(self.dht)))
        want = ref[4] * 0.25 + (0.0 if old is None else old)
        sums = bound.sum(axis=(0, 1)) + 64 * ULP * np.abs(ref[1]).sum(axis=(0, 1))
        U.close32(got[4], want, sums * 0.25 + 4 * ULP * np.abs(want) + 1e-30)
        assert got[5] == 0


CASES = [
    # one to a few tokens: serving
    dict(n=1, t=1, c=1, dtype="f16"), dict(n=64, t=1, c=1152, dtype="bf16"), dict(n=3, t=1, c=77, dtype="f16", pad=3, shift=1),
    dict(n=5, t=2, c=8, dtype="bf16", with_g=False), dict(n=2, t=3, c=130, dtype="f16", with_bias=False, carry=False),
    dict(n=4, t=17, c=64, dtype="f16", pad=128, pady=8),
    # around the lengths at which the tokens are split
    dict(n=2, t=31, c=96, dtype="f16"), dict(n=2, t=32, c=96, dtype="bf16"), dict(n=1, t=33, c=128, dtype="f16"),
    dict(n=2, t=63, c=40, dtype="bf16"), dict(n=2, t=64, c=40, dtype="f16"), dict(n=2, t=65, c=40, dtype="f16", pad=5),
    dict(n=3, t=127, c=33, dtype="f16", pad=66, shift=1), dict(n=3, t=128, c=128, dtype="bf16", pad=256),
    dict(n=3, t=129, c=136, dtype="f16"), dict(n=1, t=191, c=260, dtype="f16"), dict(n=1, t=257, c=16, dtype="bf16", carry=False),
    dict(n=2, t=513, c=129, dtype="f16", with_g=False), dict(n=1, t=1025, c=24, dtype="f16"),
    dict(n=1, t=5000, c=8, dtype="f16"), dict(n=2, t=2049, c=200, dtype="bf16", pad=400),
    dict(n=70, t=130, c=9, dtype="f16"), dict(n=1, t=300, c=2048, dtype="f16"),
    # lengths: empty, one, on the edges of a stretch, past the end, below zero
    dict(n=9, t=200, c=72, dtype="f16", lengths=[0, 1, 63, 64, 65, 128, 200, 777, -5]),
    dict(n=4, t=1, c=72, dtype="f16", lengths=[0, 1, 2, -1]),
    dict(n=3, t=700, c=20, dtype="bf16", lengths=[0, 320, 699], carry=False),
    dict(n=2, t=90, c=16, dtype="f16", lengths=[0, 0], pad=1),
    # every number of waves and of teams of a wave, and the lengths where they change
    dict(n=2, t=6, c=200, dtype="f16"), dict(n=2, t=7, c=200, dtype="bf16"), dict(n=2, t=16, c=131, dtype="f16"),
    dict(n=2, t=17, c=130, dtype="f16"), dict(n=2, t=32, c=130, dtype="bf16", lengths=[31, 17]), dict(n=2, t=48, c=66, dtype="f16"),
    dict(n=3, t=64, c=64, dtype="f16"), dict(n=3, t=65, c=63, dtype="bf16", lengths=[0, 64, 33]), dict(n=2, t=32, c=33, dtype="f16"),
    dict(n=2, t=33, c=64, dtype="f16"), dict(n=2, t=64, c=32, dtype="f16"), dict(n=2, t=130, c=31, dtype="bf16"),
    dict(n=2, t=1300, c=17, dtype="f16", pad=34), dict(n=2, t=128, c=16, dtype="f16"), dict(n=2, t=129, c=2, dtype="f16"),
    dict(n=2, t=2500, c=15, dtype="bf16", lengths=[1025, 2500]), dict(n=1, t=9000, c=3, dtype="f16", with_g=False),
    # nothing to do but to hand the state on
    dict(n=3, t=0, c=10, dtype="f16"),
]


@pytest.mark.parametrize("kw", CASES, ids=lambda k: "-".join("%s%s" % p for p in k.items()).replace(" ", ""))
def test_against_oracle(nnlib, kw):
    Case(**kw).check()


@pytest.mark.parametrize("kw", [CASES[1], CASES[5], CASES[12], CASES[20], CASES[23]], ids=str)
def test_states_in_place_and_accumulation(nnlib, kw):
    c = Case(**dict(kw, seed=5))
    c.check(in_place=True, old=np.random.default_rng(1).standard_normal(c.c).astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("t", [1, 100, 400])
def test_gates_at_their_limits(nnlib, t):
    """f far past the limit, infinite f and x: a stays above 0 and below 1, nothing turns into NaN by itself."""
    c = Case(2, t, 64, "bf16", seed=3)
    c.f[0, 0, :8] = 1000.0
    c.f[0, 0, 8:16] = -1000.0
    c.f[1, t // 2, 16:24] = np.inf
    c.f[1, t // 2, 24:32] = -np.inf
    y, ht = c.forward()
    ry, h = S.recurrence_fwd(c.x, c.f, c.bias, c.g, None, c.h0)
    big = np.abs(h).max()
    k = ULP * (90 + 2 * t)
    U.close16(y, ry, "bf16", k * big * (1 + np.abs(c.g)))
    U.close32(ht, h[:, -1], k * big)


@pytest.mark.parametrize("t", [1, 40, 130, 1000])
def test_bad_values_stay_in_their_channel_and_go_forward(nnlib, t):
    """An infinite x makes its channel infinite from there on; a NaN likewise; nothing before, nothing beside."""
    c = Case(2, t, 64, "bf16", with_g=False, seed=4)
    j = t // 3
    c.x[0, j, 5] = np.inf
    c.x[1, j, 6] = np.nan
    c.f[0, j, 7] = np.nan
    y, ht = c.forward()
    assert np.isinf(y[0, j:, 5]).all() and np.isfinite(y[0, :j, 5]).all()
    assert np.isnan(y[1, j:, 6]).all() and np.isfinite(y[1, :j, 6]).all()
    assert np.isnan(y[0, j:, 7]).all() and np.isfinite(y[0, :j, 7]).all()
    rest = np.ones((2, 64), bool)
    rest[0, 5] = rest[1, 6] = rest[0, 7] = False
    assert np.isfinite(y.transpose(0, 2, 1)[rest]).all() and np.isfinite(ht[rest]).all()
    assert np.isinf(ht[0, 5]) and np.isnan(ht[1, 6]) and np.isnan(ht[0, 7])


def test_tokens_past_the_length_may_hold_anything(nnlib):
    lengths = [0, 70, 129]
    a = Case(3, 300, 48, "f16", lengths=lengths, seed=8)
    b = Case(3, 300, 48, "f16", lengths=lengths, seed=8)
    for i, l in enumerate(lengths):
        for v in (b.x, b.f, b.g, b.dy):
            v[i, l:] = np.nan
    ya, ha = a.forward()
    yb, hb = b.forward()
    assert np.array_equal(ya, yb) and np.array_equal(ha, hb)
    ga, gb = a.backward(), b.backward()
    for p, q, l in zip(ga[:5], gb[:5], range(5)):
        assert np.array_equal(p, q)
    for i, l in enumerate(lengths):
        for v in ga[:3]:
            assert not v[i, l:].any()


@pytest.mark.parametrize("t,cut", [(300, 1), (300, 128), (300, 299), (2000, 777)])
def test_a_sequence_in_two_calls(nnlib, t, cut):
    """The state carries a sequence from one call to the next, tokens one at a time included."""
    c = Case(2, t, 72, "bf16", seed=11)
    y, ht = c.forward()
    first, rest = Case(2, cut, 72, "bf16"), Case(2, t - cut, 72, "bf16")
    for k in ("x", "f", "g"):
        setattr(first, k, getattr(c, k)[:, :cut])
        setattr(rest, k, getattr(c, k)[:, cut:])
    first.bias = rest.bias = c.bias
    first.h0 = c.h0
    y1, mid = first.forward(in_place=True)
    rest.h0 = mid
    y2, end = rest.forward(in_place=True)
    k = ULP * (24 + 4 * t) * max(np.abs(mid).max(), np.abs(c.x).max())
    U.close32(end, ht, k)
    # both are one rounding from the state's exact value
    d = np.abs(np.concatenate([y1, y2], axis=1) - y)
    assert np.all(d <= 2 * U.HALF_ULP["bf16"] * np.abs(y) * 1.01 + 2 * k * np.abs(c.g))


def test_streams_graph_and_repeats(nnlib):
    t = U.torch()
    n, tt, c = 2, 3000, 96
    g = t.Generator(device="cuda").manual_seed(5)
    proj = t.randn((n, tt, 3 * c), generator=g, device="cuda").half()
    dy = t.randn((n, tt, c), generator=g, device="cuda").half()
    bias = t.rand(c, generator=g, device="cuda") * 6
    x, f, gate = (proj[..., i * c:(i + 1) * c] for i in range(3))
    op = nc.GatedRecurrence(n, tt, c, ld=3 * c, dtype=nc.NNCONV_F16)
    saved = op.saved()
    y, dproj = t.empty_like(dy), t.empty_like(proj)
    ht, dh0, dbias = t.empty((n, c), device="cuda"), t.empty((n, c), device="cuda"), t.empty(c, device="cuda")
    dx, df, dg = (dproj[..., i * c:(i + 1) * c] for i in range(3))
    outs = (y, dproj, ht, dh0, dbias)

    def both(stream=None):
        op.fwd(x, f, bias, y, g=gate, ht=ht, saved=saved, stream=stream)
        op.bwd(x, f, bias, saved, dy, dx, df, g=gate, dg=dg, dh0=dh0, dbias=dbias, stream=stream)

    def bits():
        return [v.clone().view(t.uint8) for v in outs]
    both()
    t.cuda.synchronize()
    first = bits()
    s = t.cuda.Stream()
    for k in range(3):
        for v in outs:
            v.zero_()
        t.cuda.synchronize()
        with t.cuda.stream(s):
            both()
        s.synchronize()
        assert all(bool((a == b).all()) for a, b in zip(first, bits())), k
    with t.cuda.stream(s):
        both()
    s.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph, stream=s):
        both()
    for k in range(4):
        for v in outs:
            v.zero_()
        t.cuda.synchronize()
        graph.replay()
        t.cuda.synchronize()
        assert all(bool((a == b).all()) for a, b in zip(first, bits())), "replay %d" % k


def test_two_streams_at_once(nnlib):
    """A handle used on two streams without ordering keeps their workspaces apart."""
    t = U.torch()
    n, tt, c = 1, 20000, 64
    g = t.Generator(device="cuda").manual_seed(6)
    op = nc.GatedRecurrence(n, tt, c, dtype=nc.NNCONV_BF16)
    sets = []
    for k in range(2):
        x, f = (t.randn((n, tt, c), generator=g, device="cuda").bfloat16() for _ in range(2))
        sets.append((x, f, t.empty_like(x), t.cuda.Stream()))
    bias = t.full((c,), 5.0, device="cuda")
    alone = []
    for x, f, y, _ in sets:
        op.fwd(x, f, bias, y)
        t.cuda.synchronize()
        alone.append(y.clone())
        y.zero_()
    t.cuda.synchronize()
    for _ in range(5):
        for x, f, y, s in sets:
            op.fwd(x, f, bias, y, stream=s.cuda_stream)
    t.cuda.synchronize()
    for (_, _, y, _), want in zip(sets, alone):
        assert bool((y.view(t.int16) == want.view(t.int16)).all())


def test_more_sequences_than_a_launch_takes(nnlib):
    """2^22 workgroups and some: the same bits as calls on a few of the sequences."""
    t = U.torch()
    n, tt, c = (1 << 22) + 5, 17, 2
    g = t.Generator(device="cuda").manual_seed(2)
    mk = lambda *s: t.randn(s, generator=g, device="cuda")  # noqa: E731
    x, f, dy = (mk(n, tt, c).half() for _ in range(3))
    bias, h0, dht = mk(c), mk(n, c), mk(n, c)

    def both(lo, hi):
        op = nc.GatedRecurrence(hi - lo, tt, c, dtype=nc.NNCONV_F16)
        a = [v[lo:hi] for v in (x, f, dy, h0, dht)]
        y, ht, saved = t.empty_like(a[0]), t.empty_like(a[3]), op.saved()
        dx, df, dh0, dbias = t.empty_like(a[0]), t.empty_like(a[0]), t.empty_like(a[3]), t.empty(c, device="cuda")
        op.fwd(a[0], a[1], bias, y, h0=a[3], ht=ht, saved=saved)
        op.bwd(a[0], a[1], bias, saved, a[2], dx, df, dht=a[4], dh0=dh0, dbias=dbias)
        return [y, ht, saved.view(-1, c), dx, df, dh0], dbias
    whole, dbias = both(0, n)
    for lo, hi in ((0, 9), ((1 << 22) - 4, n), (n // 2, n // 2 + 100)):
        part, _ = both(lo, hi)
        for a, b in zip(whole, part):
            assert bool((a[lo:hi].contiguous().view(t.uint8) == b.contiguous().view(t.uint8)).all())
    # every workgroup's share of the bias gradient is counted once
    want = t.zeros(c, dtype=t.float64, device="cuda")
    for k in range(0, n, 1 << 20):
        want += whole[4][k:k + (1 << 20)].double().sum((0, 1))
    # df is rounded to 11 bits in the sum that is compared with: a random walk over 7e7 terms below 2
    assert float((dbias.double() - want).abs().max()) <= 8 * (n * tt) ** 0.5 * 2.0 ** -11


def test_offsets_past_32_bits(nnlib):
    """Sequences that start 3 and more GB into the tensors: the bits of a call on the last one alone."""
    t = U.torch()
    n, tt, c = 3, 300001, 800  # 2.2e9 elements of the packed input, 0.7e9 of y
    g = t.Generator(device="cuda").manual_seed(3)
    proj = t.empty((n, tt, 3 * c), dtype=t.float16, device="cuda")
    for i in range(n):
        proj[i] = t.randn((tt, 3 * c), generator=g, device="cuda")
    dy = t.randn((n, tt, c), generator=g, device="cuda").half()
    bias, h0 = t.rand(c, generator=g, device="cuda") * 6, t.randn((n, c), generator=g, device="cuda")

    def both(lo):
        m = n - lo
        p, d, h = proj[lo:], dy[lo:], h0[lo:].contiguous()
        op = nc.GatedRecurrence(m, tt, c, ld=3 * c, dtype=nc.NNCONV_F16)
        x, f, gate = (p[..., i * c:(i + 1) * c] for i in range(3))
        y, dp, ht, saved = t.empty_like(d), t.empty_like(p), t.empty_like(h), op.saved()
        dx, df, dg = (dp[..., i * c:(i + 1) * c] for i in range(3))
        op.fwd(x, f, bias, y, g=gate, h0=h, ht=ht, saved=saved)
        op.bwd(x, f, bias, saved, d, dx, df, g=gate, dg=dg)
        return y[-1], ht[-1], dp[-1]
    for a, b in zip(both(0), both(n - 1)):
        assert bool((a.view(t.uint8) == b.view(t.uint8)).all())


@pytest.mark.parametrize("t", [1, 16, 17, 64])
@pytest.mark.parametrize("c", [129, 257, 131])
def test_states_in_place_where_a_channel_is_alone(nnlib, t, c):
    """An odd count's last channel, in a workgroup of its own too: many calls in place are one long sequence."""
    calls = 40
    whole = Case(8, t * calls, c, "f16", with_g=False, seed=2)
    y, ht = whole.forward()
    h = whole.h0
    for k in range(calls):
        part = Case(8, t, c, "f16", with_g=False)
        part.x, part.f = whole.x[:, k * t:(k + 1) * t], whole.f[:, k * t:(k + 1) * t]
        part.bias, part.h0 = whole.bias, h
        yk, h = part.forward(in_place=True)
        assert np.abs(yk - y[:, k * t:(k + 1) * t]).max() <= 2.0 ** -9 * max(1.0, np.abs(y).max())
    U.close32(h, ht, ULP * (24 + 4 * t * calls) * max(np.abs(h).max(), np.abs(whole.x).max()))
