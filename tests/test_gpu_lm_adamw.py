"""The AdamW step over many tensors.  States in 32 and in 8 bits against a restatement in elementary fp32 operations, which gives the
same bits (the step itself: 4 ulp of the quotient), and against 64 bits.

Bounds against 64 bits (e = 2^-24): m: 3 e (|b1 m| + |(1 - b1) g|) and e for each rounded factor: 5 e; v the same, all terms positive: 6 e;
step: 4 e from m, root and factors, 3 e from v and the quotient, relative to the terms of m: 12 e; p: 2 e |p| and that."""

import math

import pytest
import torch
from test_gpu_lm_ops import E24, gen, randn

pytestmark = pytest.mark.gpu
F16, BF16, F32, E4M3 = torch.float16, torch.bfloat16, torch.float32, torch.float8_e4m3fn
HYPER = dict(beta1=0.9, beta2=0.95, eps=1e-8)


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


def factors(lr, step, beta1, beta2, eps):
    return lr / (1 - beta1 ** step), 1 / math.sqrt(1 - beta2 ** step)


def states(p, g, m, v, lr, step, decay, gs, beta1, beta2, eps):
    """(m, v, root, p without the step, step) in fp32, one rounding for each operation."""
    g = g.float() * gs
    m = m * beta1 + g * (1 - beta1)
    v = v * beta2 + (g * (1 - beta2)) * g
    root = torch.sqrt(v)
    k1, k2 = factors(lr, step, beta1, beta2, eps)
    return m, v, root, p * (1 - lr * decay), (m * k1) / (root * k2 + eps)


def make(g, sizes, offset=0, grad=F32, copy=BF16, bits=32):
    """Tensors at the given offset from a 256-byte boundary (in elements), and guards behind them."""
    def place(n, kind):
        buf = torch.full((offset + n + 40,), 3.0, device="cuda").to(kind)
        return buf[offset:offset + n], buf

    out = []
    for n in sizes:
        t = dict(p=place(n, F32), g=place(n, grad), m=place(n, E4M3 if bits == 8 else F32), v=place(n, E4M3 if bits == 8 else F32))
        t["p"][0].copy_(randn(g, n, std=0.02))
        t["g"][0].copy_(randn(g, n, std=1e-3))
        blocks = (n + 255) // 256
        if bits == 8:
            t["ms"], t["vs"] = torch.zeros(blocks, device="cuda"), torch.zeros(blocks, device="cuda")
            t["m"][0].zero_()
            t["v"][0].zero_()
        else:
            t["m"][0].copy_(randn(g, n, std=1e-3))
            t["v"][0].copy_(randn(g, n, std=1e-3).square())
        if copy is not None:
            t["c"] = place(n, copy)
        out.append(t)
    return out


def plan_of(B, ops, ts, decay):
    take = lambda k: [t[k][0] if isinstance(t[k], tuple) else t[k] for t in ts] if k in ts[0] else None  # noqa: E731
    return B.AdamTensors(ops, take("p"), take("g"), take("m"), take("v"), decay, copies=take("c"), m_scales=take("ms"), v_scales=take("vs"))


def guards(ts, sizes, offset):
    for t, n in zip(ts, sizes):
        for k in ("p", "g", "m", "v", "c"):
            if k in t:
                buf = t[k][1].float()
                assert bool((buf[:offset] == 3).all()) and bool((buf[offset + n:] == 3).all())


SIZES = [1, 7, 255, 256, 257, 4096, 4097, 10000, 1, 70001, 0, 513]


@pytest.mark.parametrize("offset", [0, 1, 4])
@pytest.mark.parametrize("grad,copy", [(F32, BF16), (BF16, F16), (F16, None)])
def test_states_in_32_bits(B, ops, offset, grad, copy):
    g = gen(offset)
    ts = make(g, SIZES, offset, grad, copy)
    decay = [0.1 * (i % 3) for i in range(len(SIZES))]
    clip = torch.tensor([0.37], device="cuda")
    plan = plan_of(B, ops, ts, decay)
    for step in (1, 2, 50):
        before = [{k: t[k][0].clone() for k in ("p", "g", "m", "v")} for t in ts]
        ops.cocodc_lm_adamw(plan, 2e-3, step=step, grad_scale=clip, **HYPER)
        for t, b, d in zip(ts, before, decay):
            m, v, root, p, s = states(b["p"], b["g"], b["m"], b["v"], 2e-3, step, d, clip, **HYPER)
            assert torch.equal(t["m"][0], m) and torch.equal(t["v"][0], v) and torch.equal(t["g"][0], b["g"])
            got = t["p"][0]
            assert bool(((got.double() - (p.double() - s.double())).abs() <= 8 * E24 * s.double().abs() + E24 * (p.double() - s.double()).abs() + 1e-45).all())
            if copy is not None:
                assert torch.equal(t["c"][0], got.to(copy))
            # 64 bits
            gd = b["g"].double() * float(clip)
            md, vd = 0.9 * b["m"].double() + 0.1 * gd, 0.95 * b["v"].double() + 0.05 * gd ** 2
            terms = 0.9 * b["m"].double().abs() + 0.1 * gd.abs()
            assert bool(((m.double() - md).abs() <= 5 * E24 * terms + 1e-44).all()) and bool(((v.double() - vd).abs() <= 6 * E24 * vd + 1e-44).all())
            den = (vd / (1 - 0.95 ** step)).sqrt() + 1e-8
            pd = b["p"].double() * (1 - 2e-3 * d) - 2e-3 / (1 - 0.9 ** step) * md / den
            lim = 3 * E24 * b["p"].double().abs() + 16 * E24 * 2e-3 / (1 - 0.9 ** step) * terms / den
            assert bool(((got.double() - pd).abs() <= lim + 1e-30).all())
    guards(ts, SIZES, offset)


def mix(x):
    mask = 0xFFFFFFFF
    mul = lambda x, c: (x * (c & 0xFFFF) + (((x * (c >> 16)) & 0xFFFF) << 16)) & mask  # noqa: E731
    x = mul(x ^ (x >> 16), 0x85EBCA6B)
    x = mul(x ^ (x >> 13), 0xC2B2AE35)
    return x ^ (x >> 16)


def bits_of(seed, step, tensor, n):
    i = torch.arange(n, device="cuda")
    key = torch.full_like(i, seed & 0xFFFFFFFF)
    for part in (step, tensor, i // 256):
        key = mix((key + 0x9E3779B9) & 0xFFFFFFFF) ^ part
    key = mix((key + 0x9E3779B9) & 0xFFFFFFFF)
    return mix((key + (i % 256) * 0x9E3779B9) & 0xFFFFFFFF)


def code_8(x, bits):
    """x in [0, 448] rounded down, or up where the part cut off, in 16 bits, plus the random bits carries."""
    exponent = torch.floor(torch.log2(x.double().clamp(min=2.0 ** -9))).clamp(min=-6)
    spacing = torch.exp2(exponent - 3)
    below = x < 2.0 ** -6
    part = torch.where(below, (x * 512 + bits.float() / 65536).double(), x.double() / spacing + bits.double() / 65536)
    return torch.floor(part) * spacing


def blocks_max(x):
    n = x.numel()
    return torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256).amax(1)


@pytest.mark.parametrize("offset", [0, 1, 16])
@pytest.mark.parametrize("grad,copy", [(F32, None), (BF16, BF16), (F16, F16)])
def test_states_in_8_bits(B, ops, offset, grad, copy):
    g = gen(100 + offset)
    sizes = [n for n in SIZES]
    ts = make(g, sizes, offset, grad, copy, bits=8)
    plan = plan_of(B, ops, ts, 0.05)
    assert plan.state_bits == 8
    for step, seed in ((1, 0), (2, 12345), (3, 2 ** 31 + 7)):
        for t in ts:
            t["g"][0].copy_(randn(g, t["g"][0].numel(), std=1e-3) * torch.exp(randn(g, t["g"][0].numel(), std=2.0)))
        before = [{k: (t[k][0] if isinstance(t[k], tuple) else t[k]).clone() for k in ("p", "g", "m", "v", "ms", "vs")} for t in ts]
        ops.cocodc_lm_adamw(plan, 1e-3, step=step, seed=seed, **HYPER)
        for i, (t, b) in enumerate(zip(ts, before)):
            n = b["p"].numel()
            if n == 0:
                continue
            spread = lambda s: s.repeat_interleave(256)[:n]  # noqa: E731
            m0, v0 = b["m"].float() * spread(b["ms"]), (b["v"].float() * spread(b["vs"])).square()
            m, v, root, p, s = states(b["p"], b["g"], m0, v0, 1e-3, step, 0.05, 1.0, **HYPER)
            got = t["p"][0]
            assert bool(((got.double() - (p.double() - s.double())).abs() <= 8 * E24 * s.double().abs() + E24 * (p.double() - s.double()).abs() + 1e-45).all())
            if copy is not None:
                assert torch.equal(t["c"][0], got.to(copy))
            r = bits_of(seed, step, i, n)
            for x, scale, codes, bits in ((m, t["ms"], t["m"][0], r & 0xFFFF), (root, t["vs"], t["v"][0], r >> 16)):
                assert torch.equal(scale, (blocks_max(x.abs()) * (1 / 448)).clamp(min=1e-30))
                y = (x.abs() * spread(1 / scale)).clamp(max=448)
                want = code_8(y, bits)
                if x is root:
                    want = torch.where(root > 0, want.clamp(min=2.0 ** -9), want)
                want = torch.where(x < 0, -want, want)
                assert torch.equal(codes.double(), want)
    guards(ts, sizes, offset)


def test_rounding_is_right_on_average(B, ops):
    """With beta = 0 and no rate, the states are the gradient and its magnitude; over many seeds their mean is the value, though single codes are a sixteenth apart.
    Of 4000 draws the mean is off by at most 6 standard deviations of (spacing / 2) / sqrt(4000)."""
    n, draws = 256, 4000
    grad = torch.exp(torch.linspace(-9, 0, n, device="cuda"))
    p = torch.zeros(n, device="cuda")
    m, v, ms, vs = torch.zeros(n, device="cuda").to(E4M3), torch.zeros(n, device="cuda").to(E4M3), torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    plan = B.AdamTensors(ops, [p], [grad], [m], [v], m_scales=[ms], v_scales=[vs])
    sums = torch.zeros(2, n, device="cuda", dtype=torch.float64)
    for seed in range(draws):
        ops.cocodc_lm_adamw(plan, 0.0, step=1, beta1=0.0, beta2=0.0, seed=seed)
        sums += torch.stack([m.double() * ms, v.double() * vs])
    y = grad.double() / float(ms)
    spacing = torch.exp2(torch.floor(torch.log2(y)).clamp(min=-6) - 3) * float(ms)
    lim = 6 * spacing / 2 / math.sqrt(draws) + spacing / 65536 + 4 * E24 * grad
    assert bool(((sums / draws - grad).abs() <= lim).all())


def test_steps_from_the_device_and_from_a_graph(B, ops):
    g = gen(7)
    n = 5000
    p, grad, m, v = randn(g, n), randn(g, n, std=1e-2), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    q = [t.clone() for t in (p, m, v)]
    held, eager = B.AdamTensors(ops, [p], [grad], [m], [v], 0.1), B.AdamTensors(ops, [q[0]], [grad], [q[1]], [q[2]], 0.1)
    step, rate, one = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.ones(1, device="cuda"), torch.ones(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(one)
        ops.cocodc_lm_adamw(held, 3e-3, step_at=step, lr_scale=rate)
    for t in range(1, 6):
        grad.copy_(randn(g, n, std=1e-2))
        rate.fill_(1.0 / t)
        graph.replay()
        ops.cocodc_lm_adamw(eager, 3e-3 * float(rate), step=t)
        # the rate reaches the kernel in fp32 times fp64 here, in fp64 there
        assert torch.equal(m, q[1]) and torch.equal(v, q[2]) and float((p - q[0]).abs().max()) <= 4 * E24 * float(p.abs().max())
    assert int(step) == 5


def test_a_step_below_one_is_recorded(B):
    ops = B.LmOps(0)
    n = 300
    p, grad, m, v = (torch.ones(n, device="cuda") for _ in range(4))
    q, m2, v2 = p.clone(), m.clone(), v.clone()
    ops.cocodc_lm_adamw(B.AdamTensors(ops, [p], [grad], [m], [v]), 1e-3, step_at=torch.zeros(1, dtype=torch.int64, device="cuda"))
    assert ops.cocodc_lm_poll_status() == B.ERR_INVALID_ARG
    ops.cocodc_lm_adamw(B.AdamTensors(ops, [q], [grad], [m2], [v2]), 1e-3, step=1)
    assert ops.cocodc_lm_poll_status() == B.OK and torch.equal(p, q)


def test_many_tensors_and_many_blocks(B, ops):
    """A thousand tensors of one buffer, their sizes from one element up, in one launch; every one is its own."""
    g = gen(11)
    sizes = [(i * 7919) % 1500 + 1 for i in range(1000)]
    starts = [0]
    for n in sizes:
        starts.append(starts[-1] + n)
    flat = {k: randn(g, starts[-1]) for k in ("p", "g", "m")}
    flat["v"] = randn(g, starts[-1]).square()
    cut = lambda x: [x[a:a + n] for a, n in zip(starts, sizes)]  # noqa: E731
    before = {k: v.clone() for k, v in flat.items()}
    launches = ops.launch_count
    ops.cocodc_lm_adamw(B.AdamTensors(ops, *(cut(flat[k]) for k in "pgmv"), [0.0] * 1000), 1e-2, step=3)
    assert ops.launch_count == launches + 1
    m, v, root, p, s = states(*(before[k] for k in "pgmv"), 1e-2, 3, 0.0, 1.0, **HYPER)
    assert torch.equal(flat["m"], m) and torch.equal(flat["v"], v)
    assert bool(((flat["p"].double() - (p.double() - s.double())).abs() <= 8 * E24 * s.double().abs() + E24 * (p.double() - s.double()).abs()).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_values_that_are_not_finite(B, ops, bits):
    """They spoil their own element and no other; zeros stay zeros with a scale that divides."""
    n = 600
    g = gen(13)
    t = make(g, [n], bits=bits)[0]
    clean = {k: (x[0].clone() if isinstance(x, tuple) else x.clone()) for k, x in t.items()}
    t["g"][0][300:] = 0
    clean["g"][300:] = 0
    if bits == 32:
        t["m"][0][300:], t["v"][0][300:], clean["m"][300:], clean["v"][300:] = 0, 0, 0, 0
    t["g"][0][5], t["g"][0][9], t["g"][0][400] = float("nan"), float("inf"), float("-inf")
    for x in (t, clean):
        take = lambda k: [x[k][0] if isinstance(x[k], tuple) else x[k]]  # noqa: E731
        plan = B.AdamTensors(ops, take("p"), take("g"), take("m"), take("v"), copies=take("c"), m_scales=take("ms") if bits == 8 else None,
                             v_scales=take("vs") if bits == 8 else None)
        ops.cocodc_lm_adamw(plan, 1e-3, step=1, seed=3)
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    bad[[5, 9, 400]] = True
    assert bool(torch.isnan(t["p"][0][bad]).all()) and torch.equal(t["p"][0][~bad], clean["p"][~bad])
    if bits == 8:
        m, v = t["m"][0].float(), t["v"][0].float()
        assert bool(torch.isnan(m[bad]).all()) and bool(torch.isnan(v[bad]).all()) and bool(torch.isfinite(m[~bad]).all()) and bool(torch.isfinite(v[~bad]).all())
        assert float(t["ms"][2]) == float(torch.tensor(1e-30)) and bool((m[512:] == 0).all())


def test_nothing_to_step_and_refusals(B, ops):
    launches = ops.launch_count
    ops.cocodc_lm_adamw(B.AdamTensors(ops, [], [], [], []), 1e-3, step=1)
    e = torch.empty(0, device="cuda")
    ops.cocodc_lm_adamw(B.AdamTensors(ops, [e], [e], [e], [e]), 1e-3, step=1)
    p, g, m, v = (torch.ones(100, device="cuda") for _ in range(4))
    for bad in (dict(grads=[g[:99]]), dict(m=[m.half()]), dict(v=[v[:50]]), dict(params=[p.half()]), dict(grads=[g.double()]), dict(params=[p.cpu()]), dict(decay=[0.1, 0.1]),
                dict(copies=[torch.ones(100, device="cuda")]), dict(m_scales=[torch.ones(2, device="cuda")]), dict(params=[p.expand(2, 100).t()[:, 0], p])):
        with pytest.raises(ValueError):
            B.AdamTensors(ops, **{**dict(params=[p], grads=[g], m=[m], v=[v]), **bad})
    for bad in (dict(decay=-1.0), dict(m=[v]), dict(grads=[p]), dict(m_scales=[torch.ones(1, device="cuda")])):
        with pytest.raises(B.CocodcError):
            B.AdamTensors(ops, **{**dict(params=[p], grads=[g], m=[m], v=[v]), **bad})
    plan = B.AdamTensors(ops, [p], [g], [m], [v])
    for bad in (dict(step=0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(eps=float("nan"))):
        with pytest.raises(B.CocodcError):
            ops.cocodc_lm_adamw(plan, **{**dict(lr=1e-3, step=1), **bad})
    with pytest.raises(ValueError):
        ops.cocodc_lm_adamw(plan, 1e-3, step_at=torch.ones(1, device="cuda"))
    plan.close()
    with pytest.raises(B.CocodcError):
        ops.cocodc_lm_adamw(plan, 1e-3, step=1)
    assert ops.launch_count == launches
