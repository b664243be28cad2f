"""More of the AdamW step: what test_gpu_lm_adamw.py leaves out.  Its helpers and bounds."""

import pytest
import torch
from test_gpu_lm_adamw import E24, HYPER, gen, randn, states

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2504_17672_b200 import binding
    return binding


@pytest.fixture(scope="module")
def ops(B):
    o = B.LmOps(0)
    yield o
    assert o.cocodc_lm_poll_status() == B.OK
    o.close()


def test_a_plan_is_stepped_at_once_on_another_stream(B, ops):
    g = gen(31)
    count, n = 400, 300
    p, grad, m = (randn(g, count, n) for _ in range(3))
    v = randn(g, count, n).square()
    want = states(p, grad, m, v, 1e-2, 1, 0.0, 1.0, **HYPER)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    plan = B.AdamTensors(ops, p, grad, m, v)
    ops.cocodc_lm_adamw(plan, 1e-2, step=1, stream=side)
    side.synchronize()
    assert torch.equal(m, want[0]) and torch.equal(v, want[1])
    assert bool(((p.double() - (want[3].double() - want[4].double())).abs() <= 8 * E24 * want[4].double().abs() + E24 * p.double().abs() + 1e-45).all())
