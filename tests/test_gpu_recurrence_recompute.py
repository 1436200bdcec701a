"""The recurrence where a wait for another workgroup's word gives up: the word is computed again from its tokens.

In the ordinary library that happens only where a word stays away for thousands of looks.  libnnconv_recompute.so has
the same kernels without the looks: every pair and every state in front of a place is computed again, so that these
tests run that path throughout.  It has to give the ordinary library's bits, and the oracle's values."""
import os

import numpy as np
import pytest

from paper_2102_06725_amd import build
from paper_2102_06725_amd import nnconv as nc

import sequence_util as U
from test_gpu_recurrence import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def recompute(nnlib):
    if not os.path.exists(build.RECOMPUTE_LIB):
        build.build()
    return nc.load(build.RECOMPUTE_LIB)


# chunks of 128 tokens forward and 64 backward and their multiples by the teams of a wave (2, 4 and 8 of them up to 64,
# 32 and 16 channels); groups of 2, 4, 8 and 16 chunks, whole and broken off
KINDS = [
    dict(n=2, t=129, c=130, dtype="f16"), dict(n=2, t=257, c=66, dtype="bf16"), dict(n=3, t=700, c=131, dtype="f16"),
    dict(n=1, t=2100, c=200, dtype="bf16", pad=9, pady=3), dict(n=2, t=1537, c=260, dtype="f16", with_g=False),
    dict(n=1, t=6000, c=72, dtype="f16", with_bias=False, carry=False), dict(n=1, t=17000, c=70, dtype="f16"),
    dict(n=2, t=300, c=64, dtype="f16"), dict(n=2, t=3000, c=33, dtype="bf16"), dict(n=3, t=1100, c=32, dtype="f16", with_g=False),
    dict(n=1, t=5000, c=17, dtype="f16", pad=1, shift=1), dict(n=2, t=2500, c=16, dtype="bf16"), dict(n=1, t=9001, c=3, dtype="f16"),
    dict(n=5, t=1400, c=90, dtype="f16", lengths=[0, 1, 640, 1399, 5000]), dict(n=4, t=4500, c=15, dtype="f16", lengths=[4500, 0, 1025, 2049]),
    dict(n=3, t=2000, c=48, dtype="bf16", lengths=[2000, 63, 1200], carry=False),
]
ids = lambda k: "-".join("%s%s" % p for p in k.items()).replace(" ", "")  # noqa: E731


def outputs(case, in_place=False, old=None):
    y, ht = case.forward(in_place)
    saved = case.saved.f64()
    return [v for v in (y, ht, saved) + case.backward(in_place, old)[:5] if v is not None]


@pytest.mark.parametrize("kw", KINDS, ids=ids)
def test_the_ordinary_librarys_bits(recompute, monkeypatch, kw):
    case = Case(seed=31, **kw)
    for pass_ in (nc.NNCONV_FWD, nc.NNCONV_DGRAD):  # the exchange is there: the sequence is more than one chunk
        assert nc.nnconv_recurrence_workspace_size(case.desc(), pass_)[1] >= 8 * 3 * case.n * case.c
    want = outputs(case)
    with monkeypatch.context() as m:
        m.setattr(nc, "load", lambda path=None: recompute)
        got = outputs(case)
    for k, (a, b) in enumerate(zip(got, want)):
        assert np.array_equal(a.view(np.uint64), b.view(np.uint64)), k


@pytest.mark.parametrize("kw", [KINDS[0], KINDS[3], KINDS[8], KINDS[11], KINDS[13]], ids=ids)
def test_against_oracle(recompute, monkeypatch, kw):
    monkeypatch.setattr(nc, "load", lambda path=None: recompute)
    Case(seed=32, **kw).check(in_place=True, old=np.linspace(-1.0, 1.0, kw["c"]).astype(np.float32).astype(np.float64))


def test_bad_values_go_the_same_way(recompute, monkeypatch):
    """Infinities and NaNs pass from chunk to chunk as they do through the words."""
    case = Case(2, 1500, 96, "bf16", with_g=False, seed=33)
    case.x[0, 100, 5], case.x[0, 700, 6], case.x[1, 3, 7] = np.inf, -np.inf, np.nan
    case.f[0, 900, 8], case.f[1, 20, 9], case.f[1, 21, 10] = np.nan, np.inf, -np.inf
    case.dy[1, 1400, 11], case.dy[0, 1300, 12] = np.inf, np.nan
    want = outputs(case)
    monkeypatch.setattr(nc, "load", lambda path=None: recompute)
    for k, (a, b) in enumerate(zip(outputs(case), want)):
        assert np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(np.nan_to_num(a, posinf=1e300, neginf=-1e300),
                                                                            np.nan_to_num(b, posinf=1e300, neginf=-1e300)), k
