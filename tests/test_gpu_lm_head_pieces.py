"""The output head's gradient where the vocabulary is taken in several pieces and dx's contraction in parts too, the last piece a single
column among them, against the definition in 64 bits.

Bounds as in test_gpu_lm_head.py, except for the accumulation: dx's products are accumulated over one piece at a time (at most
2^27 / T columns) and the pieces' sums are added in fp32, so K = 2^27 / T in place of the vocabulary, and 2 e for each piece."""

import pytest
import torch
from test_gpu_lm_head import inputs, logits
from test_gpu_lm_ops import E24, UNIT, randn, within

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


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


@pytest.mark.parametrize("T,D,V,kind,tw", [
    (4096, 256, 50257, BF16, F32), (4096, 256, 50257, F16, F16),        # two pieces, four parts
    (9376, 64, 760321, BF16, BF16)])                                    # 54 pieces whose last has one column, two parts
def test_pieces_and_parts(B, ops, T, D, V, kind, tw):
    g, x, w, ids = inputs(T, D, V, kind, seed=21)
    columns = 2 ** 27 // T
    pieces = (V + columns - 1) // columns
    assert B.library().cocodc_lm_head_grad_workspace(T, D, V) < 2 * T * V          # not all of dz at a time
    ids[::50] = V - 1                                                              # the last piece's columns get their share
    dlogp = randn(g, T, std=1e-4 if kind is F16 else 1.0)
    lse = torch.empty(T, device="cuda")
    rows = max(1, 2 ** 27 // V)
    for a in range(0, T, rows):
        lse[a:a + rows] = torch.logsumexp(x[a:a + rows].double() @ w.double().t(), 1).float()
    gx, gw = torch.empty_like(x), torch.empty(V, D, dtype=tw, device="cuda")
    ops.cocodc_lm_head_grad(x, w, ids, lse, dlogp, None, gx, gw)
    wd, most = w.double(), float((dlogp.abs() * (ids >= 0)).max())
    dw, ew = (torch.zeros(V, D, dtype=torch.float64, device="cuda") for _ in range(2))
    for a in range(0, T, rows):
        at = slice(a, a + rows)
        z, ez = logits(x[at], w, 1.0)
        l = lse[at].double()[:, None]
        d = torch.where(ids[at] >= 0, dlogp[at].double(), torch.zeros_like(dlogp[at], dtype=torch.float64))[:, None]
        dz = torch.exp(z - l) * -d
        edz = dz.abs() * (ez + E24 * (2 * z.abs() + l.abs()) + 2.0 ** -21 + 4 * E24)
        dz.scatter_add_(1, ids[at].clamp(min=0).unsqueeze(1), d)
        edz += 4 * E24 * d.abs()
        edz += UNIT[kind] * (dz.abs() + edz)
        if kind is F16:
            edz += 2.0 ** -34 * most
        both = dz.abs() + edz
        dx = dz @ wd
        within(gx[at], dx, edz @ wd.abs() + (2 * columns + 2 * pieces) * E24 * (both @ wd.abs()) + 4 * E24 * dx.abs(), "dx")
        xd = x[at].double()
        dw += dz.t() @ xd
        ew += edz.t() @ xd.abs() + 2 * T * E24 * (both.t() @ xd.abs())
    within(gw, dw, ew + 4 * E24 * dw.abs(), "dtable")
