"""More of the AdamW step: what test_gpu_lm_adamw.py leaves out.  Its helpers and bounds."""

import pytest
import torch
from test_gpu_lm_adamw import E24, E4M3, HYPER, bits_of, gen, randn, states

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


def test_a_step_below_one_is_step_one_for_the_random_bits_too(B):
    ops = B.LmOps(0)
    g = gen(32)
    n = 2000
    p, grad = randn(g, n), randn(g, n)

    def stepped(**k):
        q, m, v = p.clone(), torch.zeros(n, device="cuda").to(E4M3), torch.zeros(n, device="cuda").to(E4M3)
        ms, vs = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
        ops.cocodc_lm_adamw(B.AdamTensors(ops, [q], [grad], [m], [v], m_scales=[ms], v_scales=[vs]), 1e-3, seed=5, **k)
        return q, m.view(torch.uint8), v.view(torch.uint8), ms, vs

    one = stepped(step=1)
    assert ops.cocodc_lm_poll_status() == B.OK
    for at in (0, -7):
        other = stepped(step_at=torch.tensor([at], device="cuda"))
        assert ops.cocodc_lm_poll_status() == B.ERR_INVALID_ARG
        assert all(torch.equal(a, b) for a, b in zip(one, other))
    assert not torch.equal(stepped(step=2)[1], one[1])


@pytest.mark.parametrize("eps", [1.5, 1e6, 0.0, 2.0 ** -126])
def test_any_eps(B, ops, eps):
    g = gen(33)
    n = 3000
    p, grad, m = (randn(g, n) for _ in range(3))
    v = randn(g, n).square()
    m[1000:], v[1000:], grad[1000:] = 0, 0, 0                    # never used: stands still with any eps above zero
    want = states(p, grad, m, v, 1e-2, 3, 0.0, 1.0, **{**HYPER, "eps": eps})
    ops.cocodc_lm_adamw(B.AdamTensors(ops, [p], [grad], [m], [v]), 1e-2, step=3, eps=eps)
    assert torch.equal(m, want[0]) and torch.equal(v, want[1])
    used = slice(0, n if eps else 1000)
    got, s = p[used].double(), want[4][used].double()
    assert bool(((got - (want[3][used].double() - s)).abs() <= 8 * E24 * s.abs() + E24 * got.abs() + 1e-45).all())
    assert eps or bool(torch.isnan(p[1000:]).all())              # 0 / 0


def test_every_bit_of_the_seed_counts(B, ops):
    g = gen(34)
    n = 5000
    grad = randn(g, n)

    def codes(seed):
        p, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda").to(E4M3), torch.zeros(n, device="cuda").to(E4M3)
        scales = [torch.zeros((n + 255) // 256, device="cuda") for _ in range(2)]
        ops.cocodc_lm_adamw(B.AdamTensors(ops, [p], [grad], [m], [v], m_scales=[scales[0]], v_scales=[scales[1]]), 1e-3, step=1, seed=seed)
        return m.view(torch.uint8).clone()

    first = codes(5)
    assert torch.equal(first, codes(5))
    for seed in (5 + 2 ** 32, 5 + 2 ** 40, 5 - 2 ** 63, 5 - 2 ** 32):
        # about half of the codes are rounded the other way with other bits
        assert int((codes(seed) != first).sum()) > n // 8, seed


def test_small_codes_are_cut_exactly(B, ops):
    """Below 2^-6 the 8-bit numbers are 2^-9 apart: floor(512 y + r / 65536) of them, y = value / scale in fp32, r 16 random bits.  Of so many values some come so near a
    whole number that rounding any part of this would tell."""
    g = gen(35)
    n = 2 ** 24
    grad = torch.exp2(-6.0 - 5 * torch.rand(n, generator=g, device="cuda"))
    grad[::256] = 448.0                                            # the scale is 1
    m, v = torch.zeros(n, device="cuda").to(E4M3), torch.zeros(n, device="cuda").to(E4M3)
    scales = [torch.zeros(n // 256, device="cuda") for _ in range(2)]
    plan = B.AdamTensors(ops, [torch.zeros(n, device="cuda")], [grad], [m], [v], m_scales=[scales[0]], v_scales=[scales[1]])
    ops.cocodc_lm_adamw(plan, 0.0, step=1, beta1=0.0, beta2=0.0, seed=9)
    r = bits_of(9, 1, 0, n)
    root = torch.sqrt(grad * grad)
    for codes, x, scale, bits in ((m, grad, scales[0], r & 0xFFFF), (v, root, scales[1], r >> 16)):
        y = x * (1 / scale).repeat_interleave(256)
        want = torch.floor(y.double() * 512 + bits.double() / 65536).clamp(min=1.0 if x is root else 0.0) / 512
        small = y < 2.0 ** -6
        assert int(small.sum()) > n // 2
        assert torch.equal(codes.double()[small], want[small])
