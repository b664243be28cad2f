"""The output head with long contractions."""

import pytest
import torch
from test_gpu_lm_ops import E24, UNIT, gen, randn, within

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


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


def test_millions_of_products(ops):
    """Products -1, 0 and 1, whose sums are whole numbers below 2^24 in any order and any parts: the logits are exact, and what is left is the exponentials' error
    (bounds of test_gpu_lm_head.py with the logits' own error 0)."""
    T, V, D, scale = 3, 20, 2 ** 23 + 1024, 2.0 ** -10
    g = gen(41)
    x, w = (torch.randint(-1, 2, s, generator=g, device="cuda").to(BF16) for s in ((T, D), (V, D)))
    ids = torch.tensor([7, -1, 19], device="cuda")
    logp, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ops.cocodc_lm_head(x, w, ids, logp, lse=lse, scale=scale)
    z = (x.double() @ w.double().t()) * scale
    assert float(z.abs().max()) > 1.0
    want = torch.logsumexp(z, 1)
    el = E24 * (3 * z.abs().amax(1) + 300)
    within(lse, want, el, "lse")
    zy = z.gather(1, ids.clamp(min=0).unsqueeze(1)).squeeze(1)
    there = (ids >= 0).double()
    within(logp, (zy - want) * there, (el + 2 * E24 * (zy.abs() + want.abs())) * there, "logp")
    dlogp = randn(g, T)
    dx, dw = torch.empty_like(x), torch.empty(V, D, device="cuda")
    ops.cocodc_lm_head_grad(x, w, ids, lse, dlogp, None, dx, dw, scale=scale)
    d = (dlogp.double() * there)[:, None]
    p = torch.exp(z - lse.double()[:, None]) * -d
    edz = p.abs() * (E24 * (2 * z.abs() + lse.double().abs()[:, None] + 4) + 2.0 ** -21)
    dz = p.scatter_add(1, ids.clamp(min=0).unsqueeze(1), d)
    edz = edz + 4 * E24 * d.abs()
    edz = edz + UNIT[BF16] * (dz.abs() + edz)
    both = dz.abs() + edz
    for a in range(0, D, 2 ** 20):
        wd, xd = w[:, a:a + 2 ** 20].double(), x[:, a:a + 2 ** 20].double()
        want = dz @ wd * scale
        within(dx[:, a:a + 2 ** 20], want, (edz @ wd.abs() + 2 * V * E24 * (both @ wd.abs())) * scale + 4 * E24 * want.abs(), "dx")
        want = dz.t() @ xd * scale
        within(dw[:, a:a + 2 ** 20], want, (edz.t() @ xd.abs() + 2 * T * E24 * (both.t() @ xd.abs())) * scale + 4 * E24 * want.abs(), "dtable")


def errors(ops, D, seeds=4):
    """Relative errors of the log-sum-exp where each row has one large logit, whose products are positive on average."""
    out = []
    for seed in range(seeds):
        g = gen(1000 * seed + D)
        w = randn(g, 2000, D, std=2 * D ** -0.5, dtype=BF16)
        x = randn(g, 256, D) + 2 * w[:256].float()
        x = x.to(BF16)
        lse = torch.empty(256, device="cuda")
        ops.cocodc_lm_head(x, w, None, None, lse=lse)
        want = torch.logsumexp(x.double() @ w.double().t(), 1)
        out.append((lse.double() - want) / want)
    return torch.cat(out)


def test_parts_keep_the_error_of_a_short_contraction(ops):
    """The tensor cores cut what they accumulate.  Contractions of more than 704 products are accumulated in parts of about 512, so that their error, whose sign is the
    cutting's, stays below that of 704 products accumulated at a time.  (Without parts it grows with the length: 1.1 times at 768, 1.5 at 1024, 6 at 4096.)"""
    most = float(errors(ops, 704).abs().mean())
    for D in (768, 1024, 1088, 2048, 4096):
        e = errors(ops, D)
        assert float(e.abs().mean()) < most and abs(float(e.mean())) < most, D


def test_the_error_of_parts_by_arithmetic(ops):
    """Parts of 512: 32 steps of 16 products.  A step loses less than a spacing, half of it on average: at most e = 2^-24 of the partial sum, which grows from 0 to the
    part's sum, half of it on average: 32 e / 2.  The eight parts are added with rounding, which has no sign; the exponential and the logarithm cost another e.
    (Without parts it is eight times 32 e / 2 by this count, and 2.2e-6 in fact.)"""
    e = errors(ops, 4096)
    assert abs(float(e.mean())) < 17 * E24 and float(e.abs().mean()) < (17 + 2) * E24
