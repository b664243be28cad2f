"""Edges of the norm, the output head and the optimizer: narrow matrices, fp32 gradients that are added to, offsets past 32 bits, calls at the
same time, columns of one buffer.  Bounds as in the operators' own test files."""

import pytest
import torch
from test_gpu_lm_head import gradient, inputs, logits, statistics
from test_gpu_lm_norm import EPS, chain
from test_gpu_lm_ops import E24, gen, randn, within

pytestmark = pytest.mark.gpu
F16, BF16, F32, E4M3 = torch.float16, torch.bfloat16, torch.float32, torch.float8_e4m3fn


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


@pytest.mark.parametrize("T,D,V", [(1, 8, 8), (5, 8, 1000), (200, 16, 24), (130, 40, 300), (128, 64, 64), (64, 1088, 500), (300, 2120, 260)])
@pytest.mark.parametrize("tw,accumulate", [(F32, True), (F32, False), (BF16, True), (BF16, False)])
def test_head_narrow_and_long(ops, T, D, V, tw, accumulate):
    g, x, w, ids = inputs(T, D, V, BF16, seed=11)
    z, ez = logits(x, w, 1.0)
    lse, el, logp, ep = statistics(z, ez, ids)
    got, gl = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ops.cocodc_lm_head(x, w, ids, got, lse=gl)
    within(gl, lse, el, "lse")
    within(got, logp, ep, "logp")
    dlogp = randn(g, T)
    dx, ex, dw, ew = gradient(x, w, ids, gl, dlogp, None, 1.0)
    first = randn(g, V, D, dtype=tw)
    gx, gw = torch.empty_like(x), first.clone()
    ops.cocodc_lm_head_grad(x, w, ids, gl, dlogp, None, gx, gw, accumulate=accumulate)
    within(gx, dx, ex, "dx")
    want = dw + first.double() if accumulate else dw
    within(gw, want, ew + E24 * (dw.abs() + first.double().abs()), "dtable")


def test_head_error_does_not_grow_with_the_contraction(ops):
    """Long contractions are accumulated in parts: the mean error of the log-sum-exp stays below a quarter of what cutting each of 16 products' sums
    could cost, K / 16 half spacings."""
    g, x, w, ids = inputs(256, 4096, 2000, BF16, seed=12)
    x = x + (w[:256] * 2).bfloat16()                                     # one large logit a row
    lse = torch.empty(256, device="cuda")
    ops.cocodc_lm_head(x, w, None, None, lse=lse)
    want = torch.logsumexp(x.double() @ w.double().t(), 1)
    assert float(((lse.double() - want).abs() / want).mean()) < 4096 / 16 * E24 / 4


def test_norm_past_32_bits(ops):
    T = 262200                                                          # 2.15e9 elements; rows too long for registers, and the longest that are not
    for D in (8200, 8192):
        x = torch.zeros(T, D, dtype=BF16, device="cuda")
        g = gen(1)
        x[-3:] = randn(g, 3, D, dtype=BF16)
        w = randn(g, D)
        y, rstd = torch.empty_like(x), torch.empty(T, device="cuda")
        ops.cocodc_lm_norm(x, w, y, rstd=rstd, eps=EPS)
        z = x[-3:].double()
        k = (z.square().mean(1) + EPS).rsqrt()
        ek = (chain(D) / 2 + 4) * E24
        within(rstd[-3:], k, k * ek)
        within(y[-3:], z * k[:, None] * w.double(), (z * k[:, None] * w.double()).abs() * (ek + 2 * E24))
        assert not bool(y[::997].count_nonzero())
        dw = torch.empty(D, device="cuda")
        dy = y
        dy[-3:] = 1
        dx = torch.empty_like(x)
        ops.cocodc_lm_norm_grad(dy, x, w, rstd, dx, dweight=dw)
        h = z * rstd[-3:].double()[:, None]
        within(dw, h.sum(0), 1000 * E24 * h.abs().sum(0))
        mean = (w.double() * h).mean(1, keepdim=True)
        off = (chain(D) + 2) * E24 * (w.double() * h).abs().mean(1, keepdim=True) + 4 * E24 * mean.abs()
        want = rstd[-3:].double()[:, None] * (w.double() - h * mean)
        within(dx[-3:], want, rstd[-3:].double()[:, None] * (2 * E24 * w.double().abs() + h.abs() * off) + 2 * E24 * want.abs())
        assert not bool(dx[::997].count_nonzero())
        del x, y, dy, dx


def test_adamw_past_32_bits(B, ops):
    n = 2 ** 31 + 1000
    p, grad = torch.ones(n, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4M3), torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4M3)
    scales = [torch.zeros((n + 255) // 256, device="cuda") for _ in range(2)]
    grad[-5:] = torch.tensor([1.0, -1.0, 2.0, 0.5, -3.0], device="cuda").bfloat16()
    ops.cocodc_lm_adamw(B.AdamTensors(ops, [p], [grad], [m], [v], m_scales=[scales[0]], v_scales=[scales[1]]), 0.25, step=1, seed=1)
    want = 1 - 0.25 * torch.sign(grad[-5:].float())
    assert float((p[-5:] - want).abs().max()) < 1e-6 and bool((p[2 ** 31 - 100:-5] == 1).all()) and bool((p[::100003] == 1).all())
    assert bool((m[-5:].float().sign() == grad[-5:].float().sign()).all()) and bool((v[-5:].float() > 0).all())


def test_columns_of_one_buffer(ops):
    """What a call reads and writes may be different columns of one buffer."""
    g = gen(4)
    T, D = 300, 256
    buf = randn(g, T, 4 * D, dtype=BF16)
    x, r, y, t = (buf[:, i * D:(i + 1) * D] for i in range(4))
    xs, rs = x.clone(), r.clone()
    w, want_y, want_t = randn(g, D), torch.empty(T, D, dtype=BF16, device="cuda"), torch.empty(T, D, dtype=BF16, device="cuda")
    ops.cocodc_lm_norm(xs, w, want_y, residual=rs, total=want_t)
    ops.cocodc_lm_norm(x, w, y, residual=r, total=t)
    assert torch.equal(y, want_y) and torch.equal(t, want_t) and torch.equal(x, xs) and torch.equal(r, rs)


def test_calls_at_the_same_time(B, ops):
    """Two streams, one handle, one plan each: the same bits as one after the other."""
    g = gen(6)
    n, T, D = 300001, 5000, 768
    grads = randn(g, n, std=1e-2)
    x, dy, w = randn(g, T, D, dtype=BF16), randn(g, T, D, dtype=BF16), randn(g, D)

    def state():
        f = lambda: torch.zeros(n, device="cuda")  # noqa: E731
        p, m, v = f(), f(), f()
        return dict(plan=B.AdamTensors(ops, [p], [grads], [m], [v], 0.1), p=p, y=torch.empty_like(x), rstd=torch.empty(T, device="cuda"),
                    dx=torch.empty_like(x), dw=torch.empty(D, device="cuda"),
                    ws=torch.empty(B.library().cocodc_lm_norm_grad_workspace(T, D), dtype=torch.uint8, device="cuda"))

    def work(s, stream=None):
        for t in range(1, 4):
            ops.cocodc_lm_adamw(s["plan"], 1e-3, step=t, stream=stream)
            ops.cocodc_lm_norm(x, w, s["y"], rstd=s["rstd"], stream=stream)
            ops.cocodc_lm_norm_grad(dy, x, w, s["rstd"], s["dx"], dweight=s["dw"], workspace=s["ws"], stream=stream)

    alone, streams = state(), [torch.cuda.Stream() for _ in range(2)]
    work(alone)
    both = [state() for _ in streams]
    torch.cuda.synchronize()
    for s, b in zip(streams, both):
        work(b, s)
    torch.cuda.synchronize()
    for b in both:
        assert all(torch.equal(alone[k], b[k]) for k in ("p", "y", "rstd", "dx", "dw"))
