"""What the AdamW handle refuses beside sizes and types: tensors that are not where the plan's kernels run."""
import pytest

from paper_2102_06725_amd import nnconv as nc

import sequence_util as U


def test_adamw_devices(nnlib):
    t = U.torch()
    z = lambda d="cpu": t.zeros(10, device=d)  # noqa: E731
    with pytest.raises(ValueError, match="current device"):
        nc.AdamW([dict(master=z(), grad=z(), m=z(), v=z())])


@pytest.mark.gpu
def test_adamw_tensors_elsewhere(nnlib):
    t = U.torch()
    z = lambda d="cuda", n=10: t.zeros(n, device=d)  # noqa: E731
    good = dict(master=z(), grad=z(), m=z(), v=z())
    for key in good:
        with pytest.raises(ValueError):
            nc.AdamW([good, dict(good, **{key: z("cpu")})])
    op, i32 = nc.AdamW([good]), lambda d, n=1: t.zeros(n, dtype=t.int32, device=d)  # noqa: E731
    step, state = i32("cuda"), i32("cuda", 6)
    nc.check(nc.nnconv_loss_scaler_init(state.data_ptr(), 1.0, 2.0, 10, nc.current_stream()))
    op.step(step, 1e-3, state=state, overflow_flag=i32("cuda"))
    for bad in (dict(step=i32("cpu")), dict(step=step.float()), dict(step=step.long()), dict(state=i32("cpu", 6)), dict(state=state[:4]),
                dict(overflow_flag=i32("cpu")), dict(overflow_flag=step.long()), dict(overflow_flag=step[:0])):
        with pytest.raises(ValueError):
            op.step(**dict(dict(step=step, lr=1e-3, state=state, overflow_flag=i32("cuda")), **bad))
    assert int(step.item()) == 1
