"""What the handles of the sequence operators refuse: tensors of another shape, type, layout or device than
the handle was made for would be read or written past their end.  Every call here is refused before anything
is queued; the tests marked gpu check that what fits is taken in each layout that fits."""
import pytest

from paper_2102_06725_amd import nnconv as nc

import sequence_util as U

N, T, C = 2, 70, 48


def tensors(device="cpu", dtype="f16"):
    t = U.torch()
    half = lambda *s: t.zeros(s, dtype=U.tdtype(dtype), device=device)  # noqa: E731
    f = lambda *s: t.zeros(s, device=device)  # noqa: E731
    return half, f


def norm_calls(device="cpu"):
    half, f = tensors(device)
    t = U.torch()
    op = nc.RMSNorm(N * T, C, group=32)
    r = (N * T, C)
    fwd = dict(x=half(*r), gain=f(C), y=half(*r), residual=half(*r), sum=half(*r), rstd=f(N * T))
    q8 = dict(x=half(*r), gain=f(C), q=t.zeros(r, dtype=t.uint8, device=device), scales=f(N * T, 2), residual=half(*r), sum=half(*r),
              rstd=f(N * T))
    bwd = dict(sum=half(*r), dy=half(*r), gain=f(C), rstd=f(N * T), dx=half(*r), dgain=f(C), dsum=half(*r),
               overflow_flag=t.zeros(1, dtype=t.int32, device=device))
    return {"fwd": (op.fwd, fwd), "fwd_q8": (op.fwd_q8, q8), "bwd": (op.bwd, bwd)}


def recurrence_calls(device="cpu"):
    half, f = tensors(device)
    t = U.torch()
    op = nc.GatedRecurrence(N, T, C, ld=3 * C)
    third = lambda: half(N, T, 3 * C)[..., C:2 * C]  # noqa: E731
    i32 = lambda n: t.zeros(n, dtype=t.int32, device=device)  # noqa: E731
    fwd = dict(x=third(), f=third(), bias=f(C), y=half(N, T, C), g=third(), lengths=i32(N), h0=f(N, C), ht=f(N, C), saved=op.saved(device))
    bwd = dict(x=third(), f=third(), bias=f(C), saved=op.saved(device), dy=half(N, T, C), dx=third(), df=third(), g=third(), dg=third(),
               lengths=i32(N), dht=f(N, C), dh0=f(N, C), dbias=f(C), overflow_flag=i32(1))
    return {"fwd": (op.fwd, fwd), "bwd": (op.bwd, bwd)}


def spoilt(v):
    """(why, tensor) of tensors that the call's buffer for v must not be."""
    t = U.torch()
    yield "another type", v.to(t.float64)
    if v.dtype == t.float16:
        yield "the other 16-bit type", v.to(t.bfloat16)
        yield "fp32", v.float()
    if v.shape[-1] > 1:
        yield "fewer", v[..., :-1].contiguous()
        yield "transposed", v.movedim(-1, 0).contiguous().movedim(0, -1) if v.dim() > 1 else v.repeat_interleave(2)[::2]
        yield "every other", t.zeros(v.shape[:-1] + (2 * v.shape[-1],), dtype=v.dtype, device=v.device)[..., ::2]
    if v.dim() > 1:
        yield "a sequence less", v[:-1]
        yield "wider rows", t.zeros(v.shape[:-1] + (5 * v.shape[-1],), dtype=v.dtype, device=v.device)[..., :v.shape[-1]]
    yield "nothing", v.flatten()[:0]


CALLS = [("norm", k) for k in ("fwd", "fwd_q8", "bwd")] + [("recurrence", k) for k in ("fwd", "bwd")]


def call(op, kind, device="cpu"):
    return (norm_calls if op == "norm" else recurrence_calls)(device)[kind]


@pytest.mark.parametrize("op,kind", CALLS)
def test_shapes_types_and_layouts(nnlib, op, kind):
    fn, args = call(op, kind)
    for name, v in args.items():
        for why, bad in spoilt(v):
            if name == "overflow_flag" and why not in ("another type", "nothing"):
                continue
            with pytest.raises(ValueError, match="%s: %s" % (type(fn.__self__).__name__, name)):
                fn(**dict(args, **{name: bad}))


@pytest.mark.parametrize("op,kind", CALLS)
def test_memory_that_is_not_the_gpus(nnlib, op, kind):
    fn, args = call(op, kind)
    with pytest.raises(ValueError, match="current device"):
        fn(**args)


@pytest.mark.parametrize("op,kind", CALLS)
def test_what_a_call_needs(nnlib, op, kind):
    """Without one of the tensors that the C entry needs: its own refusal, or the handle's."""
    fn, args = call(op, kind)
    needs = {"norm": ("x", "gain", "y", "q", "scales", "sum", "dy", "rstd", "dx"), "recurrence": ("x", "f", "y", "saved", "dy", "dx", "df")}[op]
    for name in needs:
        if name in args and not (kind != "bwd" and name in ("sum", "rstd", "saved")):
            with pytest.raises((ValueError, nc.NNConvError)):
                fn(**dict(args, **{name: None}))


def test_a_stale_saved_tensor(nnlib):
    """States saved for fewer tokens do not reach as far as the present ones."""
    fn, args = recurrence_calls()["bwd"]
    op = fn.__self__
    op.t = 64
    short = op.saved("cpu")
    op.t = T
    with pytest.raises(ValueError, match="saved"):
        fn(**dict(args, saved=short))
    op.n = 1
    with pytest.raises(ValueError, match="GatedRecurrence: x"):
        fn(**args)


def test_changed_rows(nnlib):
    fn, args = norm_calls()["fwd"]
    fn.__self__.rows = N * T + 1
    with pytest.raises(ValueError, match="RMSNorm: x"):
        fn(**args)


@pytest.mark.gpu
@pytest.mark.parametrize("op,kind", CALLS)
def test_one_tensor_elsewhere(nnlib, op, kind):
    fn, args = call(op, kind, "cuda")
    fn(**args)
    for name, v in args.items():
        with pytest.raises(ValueError, match="%s: %s" % (type(fn.__self__).__name__, name)) if name not in ("x", "sum") else pytest.raises(ValueError):
            fn(**dict(args, **{name: v.cpu()}))


@pytest.mark.gpu
def test_layouts_that_fit(nnlib):
    """The same tokens as [n][t][c], as an image of height 1, as rows, and with strides that sizes of one leave open."""
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(1)
    p = t.randn((N, T, 3 * C), generator=g, device="cuda").half()
    want, outs = None, []
    op = nc.GatedRecurrence(N, T, C, ld=3 * C)
    for shape in ((N, T, C), (N, 1, T, C), (N * T, C), (1, N, T, C)):
        x, f, v = (k.view(shape[:-1] + (3 * C,))[..., i * C:(i + 1) * C] for i, k in enumerate((p, p, p)))
        y = t.zeros(shape, dtype=t.float16, device="cuda")
        op.fwd(x, f, None, y, g=v)
        outs.append(y.view(N, T, C))
    for y in outs:
        want = y if want is None else want
        assert bool((y == want).all()) and bool(y.any())
    one = nc.GatedRecurrence(1, 1, C, ld=3 * C)
    y = t.zeros((1, 1, C), dtype=t.float16, device="cuda")
    first = p[:1, :1].contiguous()
    one.fwd(first[..., :C].contiguous(), first[..., C:2 * C], None, y, g=first[..., 2 * C:])  # one token: no stride is looked at
    assert bool((y == want[:1, :1]).all())
    # saved states may lie in a larger tensor
    big = t.empty(10 * N * C, device="cuda")
    op.fwd(p[..., :C], p[..., C:2 * C], None, outs[0], saved=big)
    norm = nc.RMSNorm(N * T, 3 * C)
    flat, image = t.zeros((N * T, 3 * C), dtype=t.float16, device="cuda"), t.zeros((N, 1, T, 3 * C), dtype=t.float16, device="cuda")
    gain = t.ones(3 * C, device="cuda")
    norm.fwd(p, gain, flat)
    norm.fwd(p.view(N, 1, T, 3 * C), gain, image)
    assert bool((flat == image.view(N * T, 3 * C)).all()) and bool(flat.any())
