"""More of the norm: its output in 8 bits code by code, the accuracy of its scale.  Helpers and bounds of test_gpu_lm_norm.py."""

import pytest
import test_gpu_lm_norm as N
import torch
from test_gpu_lm_norm import E4M3, EPS, F32
from test_gpu_lm_ops import gen, randn

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


@pytest.mark.parametrize("T,D", [(16384, 3200), (60000, 601), (30000, 1024), (4000, 9001), (12000, 4104)])
@pytest.mark.parametrize("group", [0, 128])
def test_codes_are_those_of_the_quotient(ops, T, D, group):
    """round(z rstd weight / y_scale), one rounding to fp32 for the quotient and one to 8 bits, on every path: the codes are those of the same call's fp32 output
    divided by the scales.  (Of so many elements some lie where a quotient that is off by an ulp gives another code.)"""
    g = gen(T + D + group)
    x, w = randn(g, T, D, dtype=torch.bfloat16), randn(g, D, std=0.3).add(1)
    y, y8, scale = torch.empty(T, D, device="cuda"), torch.empty(T, D, dtype=E4M3, device="cuda"), torch.empty(T, (D + 127) // 128 if group else 1, device="cuda")
    ops.cocodc_lm_norm(x, w, y, eps=EPS)
    ops.cocodc_lm_norm(x, w, y8, y_scale=scale, eps=EPS)
    width = group or D
    want = (y / scale.repeat_interleave(width, 1)[:, :D]).to(E4M3)
    assert torch.equal(y8.view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("T,D", [(3, 1024), (300, 1024), (300, 601), (3, 9001)])
@pytest.mark.parametrize("group", [0, 128])
def test_codes_beside_an_infinite_one(ops, T, D, group):
    """An infinite weight makes its column infinite and the scale with it: the column is NaN there, what shares the scale is 0, the rest as ever."""
    g = gen(T + D)
    x, w = randn(g, T, D), randn(g, D, std=0.1).add(1)
    y8, want = (torch.empty(T, D, dtype=E4M3, device="cuda") for _ in range(2))
    scale, clean = (torch.empty(T, (D + 127) // 128 if group else 1, device="cuda") for _ in range(2))
    ops.cocodc_lm_norm(x, w, want, y_scale=clean, eps=EPS)
    w[130] = float("inf")
    ops.cocodc_lm_norm(x, w, y8, y_scale=scale, eps=EPS)
    spoiled = torch.zeros(D, dtype=torch.bool, device="cuda")
    spoiled[128:256 if group else D] = True
    if not group:
        spoiled[:] = True
    assert bool(torch.isinf(scale[:, 1 if group else 0]).all())
    f = y8.float()
    assert bool(torch.isnan(f[:, 130]).all())
    f[:, 130] = 0
    assert bool((f[:, spoiled] == 0).all()) and torch.equal(f[:, ~spoiled], want.float()[:, ~spoiled])


@pytest.mark.parametrize("D,ty,ts", [(6344, F32, F32), (6400, F32, F32), (7616, torch.bfloat16, F32), (7680, torch.bfloat16, F32), (7680, torch.float16, F32)])
def test_widths_whose_rings_fill_shared_memory(ops, D, ty, ts):
    """Three rows of three arrays take all but a few hundred bytes of what a block may have, as soon as blocks have three rows or more."""
    N.test_norm_grad(ops, 700, D, ty, ts, F32, F32, True)
