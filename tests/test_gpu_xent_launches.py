"""How many workgroups the calls launch: as many as have work."""
import ctypes

import pytest

from paper_2102_06725_amd import nnconv as nc

import sequence_util as U

pytestmark = pytest.mark.gpu


class Dim3(ctypes.Structure):
    _fields_ = [("x", ctypes.c_uint32), ("y", ctypes.c_uint32), ("z", ctypes.c_uint32)]


class KernelNode(ctypes.Structure):  # hipKernelNodeParams
    _fields_ = [("block", Dim3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p), ("grid", Dim3), ("params", ctypes.c_void_p),
                ("shared", ctypes.c_uint32)]


def grids(call):
    """Workgroups of each kernel that `call` queues, from a captured graph's nodes."""
    t = U.torch()
    hip = ctypes.CDLL("libamdhip64.so")
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph(keep_graph=True)
    with t.cuda.graph(graph):
        call()
    handle, n = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t()
    assert hip.hipGraphGetNodes(handle, None, ctypes.byref(n)) == 0
    nodes = (ctypes.c_void_p * n.value)()
    assert hip.hipGraphGetNodes(handle, nodes, ctypes.byref(n)) == 0
    out = []
    for node in nodes:
        p = KernelNode()
        assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(p)) == 0  # no other kind is queued
        out.append(p.grid.x * p.grid.y * p.grid.z)
    return out


@pytest.mark.parametrize("rows,c,v,k", [(1, 1023, 9000, 32), (4, 331, 13000, 1024), (64, 77, 30000, 64), (1, 64, 9000, 200), (300, 41, 5000, 7)])
def test_teachers_launch(nnlib, rows, c, v, k):
    """The first launch against a teacher: shares of the rows' targets, and copies of w where its rows are no whole vectors."""
    t = U.torch()
    g = t.Generator(device="cuda").manual_seed(rows + k)
    x, w = t.randn((rows, c), generator=g, device="cuda").half(), (t.randn((v, c), generator=g, device="cuda") * c ** -0.5).half()
    targets = t.randint(-1, v, (rows, k), generator=g, device="cuda", dtype=t.int32)
    targets[:, 0] = t.arange(rows, device="cuda")
    teacher = t.randn((rows, k), generator=g, device="cuda")
    op = nc.CrossEntropy(rows, c, v, k=k)
    loss = t.empty(rows, device="cuda")
    op.fwd(x, w, targets, loss, teacher=teacher)
    first = grids(lambda: op.fwd(x, w, targets, loss, teacher=teacher))[0]
    copies = -(-v * (-(-c // 8)) // 1024) if c % 8 else 0
    shares = -(-k // 4)  # a wave a target at most
    assert rows + copies <= first <= rows * min(shares, max(1, 1024 // rows)) + copies
    # the parts that the shares and the copies make
    z = x.double() @ w.double().t()
    live = targets >= 0
    log_q = t.log_softmax(t.where(live, teacher.double(), -t.inf), 1)
    want = t.where(live, log_q.exp() * (log_q - (z - t.logsumexp(z, 1, keepdim=True)).gather(1, targets.clamp(min=0).long())), 0.0).sum(1)
    # logits of c products: (c + 2) 2^-23 of their magnitudes' sum, twice; shares and sums of k and v terms
    mag = float((x.double().abs() @ w.double().abs().t()).max())
    assert float((loss - want).abs().max()) <= 2 * (c + 2) * 2.0 ** -23 * mag + (k + 200 + v / 8192) * 2.0 ** -24 * 40
