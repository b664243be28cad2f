"""The output head's gradient at the ends of its arguments' ranges."""

import pytest
import torch
from test_gpu_lm_ops import gen, put, randn

pytestmark = pytest.mark.gpu
F16, F32 = torch.float16, torch.float32


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


@pytest.mark.parametrize("T,D,V", [(3, 64, 200), (300, 64, 200), (20000, 64, 9000), (300, 63, 200)])
def test_half_precision_where_scale_and_factors_are_large(ops, T, D, V):
    """dlogp and scale whose product leaves fp32's range: what they multiply to nothing is 0, not NaN, and what is finite is right.  The rows of x are 0, so that
    dtable is, and p is 1 / V; every other row gets nothing."""
    g = gen(T)
    x, w = torch.zeros(T, D, dtype=F16, device="cuda"), randn(g, V, D, dtype=F16)
    ids = torch.arange(T, device="cuda") % V
    ids[1::2] = -1
    lse = torch.full((T,), float(torch.log(torch.tensor(float(V)))), device="cuda")
    dlogp = torch.full((T,), 2.0 ** 100, device="cuda")
    off = D % 8
    for tw in (F16, F32):
        dx, dw = torch.empty(T, D, dtype=F16, device="cuda"), torch.empty(V, D, dtype=tw, device="cuda")
        ops.cocodc_lm_head_grad(put(x, D + off, off), put(w, D + off, off), ids, lse, dlogp, None, dx, dw, scale=1e30)
        assert bool((dw == 0).all()) and bool((dx[1::2] == 0).all()) and bool(torch.isinf(dx[::2]).any())
        # as far apart as they can be, the product in range: the same gradient as with both moderate
        a, b = (torch.empty(T, D, dtype=F16, device="cuda") for _ in range(2))
        ops.cocodc_lm_head_grad(x, w, ids, lse, dlogp, None, a, None, scale=2.0 ** -98)
        ops.cocodc_lm_head_grad(x, w, ids, lse, dlogp * 2.0 ** -100, None, b, None, scale=4.0)
        assert torch.equal(a, b) and bool((a[::2].abs().amax(1) > 0).all())
