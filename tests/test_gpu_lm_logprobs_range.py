"""Token log probabilities over the range of their arguments: logits that share a large offset, large and small products of scale
and logit, against the definition in 64 bits measured from the row's largest logit.

Bounds, derived before any run (e = 2^-24, z = scale * x, r_j = z_j - max z, S = sum exp(r_j), p_j = exp(r_j) / S):
  S               each exponent is off by 2.5 e |r_j| (the constant log2 e * scale, one fma), relatively to p_j that is 2.5 e sum p |r| <=
                  2.5 e log V; the exponential 4 e; V / 512 + 20 rounded sums of positive terms; some 5 rescalings of a thread's sums and 2 joins
                  at 6 e each; the logarithm, of a value up to log V, 4 e log V:  E = e (V / 512 + 180) for log V <= 11
  log probability E + 3 e |r|: the distance of two logits is rounded once and multiplied once
  entropy         E for log S, 3 E for each unit of sum p |r| = entropy - log S: E (1 + 3 (entropy - log S))
  log-sum-exp     E + 2 e |max z|
None of these but the last grows with an offset of the logits.
"""

import math

import pytest
import torch

from test_gpu_lm_ops import BF16, E24, F16, F32, gen, put, randn, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2504_17672_b200 import binding as B
    o = B.LmOps(0)
    yield o
    assert o.cocodc_lm_poll_status() == B.OK
    o.close()


def reference(x, targets, scale):
    """(logp, entropy, lse, log probabilities of the whole row, log S, max z) in 64 bits; rows need a finite logit."""
    scale = float(torch.tensor(scale, dtype=F32))
    z = x.double()
    m = z.amax(1, keepdim=True)
    r = (z - m) * scale
    logS = torch.log(torch.exp(r).sum(1, keepdim=True))
    lp = r - logS
    p = torch.exp(lp)
    H = logS.squeeze(1) - torch.where(p > 0, p * r, torch.zeros_like(p)).sum(1)
    top = m.squeeze(1) * scale
    return lp.gather(1, targets.unsqueeze(1)).squeeze(1), H, top + logS.squeeze(1), lp, logS.squeeze(1), top


def check(ops, x, targets, scale, k):
    T, V = x.shape
    out = {n: torch.full((T,), 77.0, device="cuda") for n in ("logp", "entropy", "lse")}
    out["top_ids"] = torch.full((T, k), -5, dtype=torch.int32, device="cuda")
    out["top_logp"] = torch.full((T, k), 77.0, device="cuda")
    ops.cocodc_lm_logprobs(x, targets, scale=scale, **out)
    logp, H, lse, lp, logS, top = reference(x, targets, scale)
    E = E24 * (V / 512 + 180)
    far = lambda v: 3 * E24 * torch.nan_to_num(v, 0, 0, 0).abs()  # noqa: E731
    # what leaves fp32's range is infinite there
    as_f32 = lambda v: torch.where(v.abs() < 3.4028e38, v, torch.sign(v) * math.inf)  # noqa: E731
    within(out["logp"], as_f32(logp), E + far(logp), "logp")
    within(out["entropy"], H, E * (1 + 3 * (H - logS).abs()), "entropy")
    within(out["lse"], as_f32(lse), E + 2 * E24 * top.abs(), "lse")
    order = torch.sort(x.double(), dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(out["top_ids"].long(), order)
    want = lp.gather(1, order)
    within(out["top_logp"], as_f32(want), E + far(want), "top")
    alone = torch.full((T,), 77.0, device="cuda")            # without alternatives: another kernel
    ops.cocodc_lm_logprobs(x, targets, alone, scale=scale)
    within(alone, as_f32(logp), E + far(logp), "logp alone")


# few rows are split over several blocks, many are not
@pytest.mark.parametrize("T,V", [(1, 1000), (1, 32000), (3, 40001), (200, 32000), (150, 77)])
@pytest.mark.parametrize("offset", [0.0, 1e3, -1e3, 1e4, -1e4, 1e5, -1e5, 1e6, -1e6])
def test_an_offset_costs_no_digits(ops, T, V, offset):
    g = gen(T + V)
    x = randn(g, T, V, std=2.0) + offset
    targets = torch.randint(0, V, (T,), generator=g, device="cuda")
    check(ops, put(x, V + 1, 1), targets, 1.0, 4)
    check(ops, x, targets, 0.8, 4)


@pytest.mark.parametrize("T,V", [(1, 1), (2, 64), (1, 40001), (3, 40001), (200, 3000)])
@pytest.mark.parametrize("scale", [1e-38, 1e-6, 1e-3, 30.0, 1e4, 1e6, 1e8, 3e8, 1e9, 1e10, 1e20, 1e30])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_scales(ops, T, V, scale, dtype):
    """Up to the largest scale: a temperature near zero, with and without masked logits."""
    g = gen(V)
    x = randn(g, T, V, std=3.0, dtype=dtype)
    targets = torch.randint(0, V, (T,), generator=g, device="cuda")
    targets[0] = x[0].float().argmax()
    check(ops, x, targets, scale, min(V, 3))
    if V > 1:
        x[:, 1::3] = -math.inf
        targets[-1] = V // 2 // 3 * 3
        check(ops, x, targets, scale, min(V, 3))
        x[:, V // 4:] = -math.inf                            # some blocks of a row have nothing left
        check(ops, x, targets, scale, 3)


@pytest.mark.parametrize("T,V", [(1, 1), (2, 64), (1, 40001), (3, 40001), (200, 3000)])
@pytest.mark.parametrize("value", [-1e4, -1e6, -1e8, -1e9, -1e10, -1e12, -1e15, -1e30, -3e38, 1e9, 1e12, 1e30, 3e38])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_logits(ops, T, V, value, dtype):
    """Rows of one value throughout, rows with that value in some or most places, rows of random multiples of it."""
    g = gen(V + 1)
    k = min(V, 3)
    targets = torch.randint(0, V, (T,), generator=g, device="cuda")
    same = torch.full((T, V), value, device="cuda").to(dtype)
    for scale in (1.0, 0.7, 1e-3):
        check(ops, same, targets, scale, k)
    x = randn(g, T, V, std=2.0, dtype=dtype)
    for keep in (torch.rand(T, V, generator=g, device="cuda") < 0.7, torch.arange(V, device="cuda").expand(T, V) < V // 5 + 1):
        for scale in (1.0, 1.3):
            check(ops, torch.where(keep, x, same), targets, scale, k)
    check(ops, (torch.rand(T, V, generator=g, device="cuda") * value).to(dtype), targets, 1.0, k)
    spread = (torch.rand(T, V, generator=g, device="cuda") * 2 - 1) * value      # distances beyond fp32's range at 3e38
    check(ops, spread.to(dtype), targets, 1.0, k)
    check(ops, spread.to(dtype), targets, 4.0 / abs(value), k)


@pytest.mark.parametrize("T,V", [(2, 64), (3, 40001), (150, 3000)])
@pytest.mark.parametrize("scale", [3e3, 1e4, 1e6, 1e8, 1e9, 1e10, 1e20, 1e30])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_gradient_at_a_temperature_near_zero(ops, T, V, scale, dtype):
    """The largest logit is a half above the others: at these scales it has all of the probability, exp(-1500) and less are 0.

    z and lse are the same fp32 number there, p is exactly 0 or 1; dlogp times scale is rounded twice, the entropy that the forward
    call gives is 0 up to 8 e, and so is what it is multiplied with."""
    g = gen(V)
    x = randn(g, T, V, std=0.5).clamp_(-2.5, 2.5)
    at = torch.randint(0, V, (T,), generator=g, device="cuda")
    x.scatter_(1, at.unsqueeze(1), 3.0 + torch.rand(T, 1, generator=g, device="cuda"))
    x = x.to(dtype)
    targets = torch.randint(0, V, (T,), generator=g, device="cuda")
    targets[0] = at[0]
    logp, H, lse = (torch.empty(T, device="cuda") for _ in range(3))
    ops.cocodc_lm_logprobs(x, targets, logp, entropy=H, lse=lse, scale=scale)
    dlogp, dH = randn(g, T), randn(g, T)
    got = torch.empty_like(x)
    want = torch.zeros(T, V, dtype=torch.float64, device="cuda")
    size = float(torch.tensor(scale, dtype=F32)) * dlogp.double()
    want.scatter_(1, targets.unsqueeze(1), size.unsqueeze(1))
    want.scatter_add_(1, at.unsqueeze(1), -size.unsqueeze(1))
    most = torch.finfo(dtype).max
    fits = lambda v: torch.where(v.abs() <= most, v, torch.sign(v) * math.inf)  # noqa: E731
    bound = torch.zeros_like(want).scatter_(1, at.unsqueeze(1), 16 * E24 * scale * dH.double().abs().unsqueeze(1)) + 2 * E24 * size.abs().unsqueeze(1)
    for a, b in ((dlogp, dH), (dlogp, None)):
        ops.cocodc_lm_logprobs_grad(x, targets, lse, H if b is not None else None, a, b, got, scale=scale)
        within(got, fits(want), bound, "gradient")


def test_gradient_without_a_finite_log_sum_exp(ops):
    """Beyond fp32's range no probabilities can be formed: NaN above it, zeros below it (as for rows of -Inf)."""
    x = torch.tensor([[1e20, 2e20, 0.0], [-1e20, -2e20, -1e20], [0.5, 0.25, 0.0]], device="cuda")
    lse, got = torch.empty(3, device="cuda"), torch.empty(3, 3, device="cuda")
    t = torch.tensor([0, 0, 0], device="cuda")
    logp = torch.empty(3, device="cuda")
    ops.cocodc_lm_logprobs(x, t, logp, lse=lse, scale=1e25)
    assert lse[0] == math.inf and lse[1] == -math.inf and abs(float(lse[2]) - 5e24) < 1e18
    ops.cocodc_lm_logprobs_grad(x, t, lse, None, torch.ones(3, device="cuda"), None, got, scale=1e25)
    assert bool(torch.isnan(got[0]).all()) and bool((got[1] == 0).all()) and bool((got[2] == 0).all())
