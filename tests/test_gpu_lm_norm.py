"""The root-mean-square norm with the residual's addition, and its gradient, against plain implementations in 64 bits.

Bounds, derived before any run (u = half the spacing of the output type relative to the value, e = 2^-24):
  total     one fp32 sum (e), rounded once
  rstd      the sum of D squares: a thread adds at most n of them, then 16 steps of joins: (n + 18) e relatively, half of it after
            the root, 3 e for mean, root and quotient.  n = max(32, D / 256 + 1)
  y         z rstd w: rstd's error and 2 e, rounded once.  In 8 bits: half a spacing of y / scale, with 8 e for the quotient's
            rounding at a border; the scale is y's error and 2 e off
  dx        mean(g h): (n + 20) e mean |g h| + |mean| e; dx: rstd (2 e |g| + |h| (that + 3 e |mean|)) + e |dx|, rounded once
  dweight   a block's thread adds every (592 R)-th row at most, R >= 1 rows at a time, then at most 8 + 74 + 8 joins: (T / 592 + 100) e
            sum |dy h|, or T + 100 where T is small
"""

import pytest
import torch
from test_gpu_lm_ops import E24, gen, placed, put, randn, untouched, within

pytestmark = pytest.mark.gpu
F16, BF16, F32, E4M3 = torch.float16, torch.bfloat16, torch.float32, torch.float8_e4m3fn
EPS = 1e-5


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


def chain(D):
    return max(32, D // 256 + 1) + 18


def spacing_8(x):
    """Distance of the 8-bit numbers around |x|."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -9))).clamp(min=-6) - 3)


SIZES = [(1, 1), (1, 2048), (1, 3200), (1, 8200), (3, 127), (5, 1000), (33, 64), (300, 512), (301, 768), (300, 1024), (299, 1536), (298, 2048), (300, 3200),
         (297, 4104), (300, 5000), (297, 8192), (20, 9001), (700, 129), (2, 16384), (2500, 96)]


@pytest.mark.parametrize("T,D", SIZES)
@pytest.mark.parametrize("tx,ts,tw", [(BF16, BF16, BF16), (BF16, F32, F32), (F16, F16, F32), (F16, F32, F16), (F32, F32, F32), (F32, F32, BF16)])
@pytest.mark.parametrize("residual", [True, False])
def test_norm(ops, T, D, tx, ts, tw, residual):
    g = gen(T + D)
    x, r, w = randn(g, T, D, dtype=tx), randn(g, T, D, std=3.0, dtype=ts), randn(g, D, std=0.3).add(1).to(tw)
    for n, (ty, pitch, off) in enumerate(((tx, D, 0), (F32 if tx is not F32 else F16, D + 5, 1), (E4M3, (D + 31) // 16 * 16, 16), (E4M3, D + 3, 1))):
        y, buf = placed(T, D, ty if ty is not E4M3 else torch.uint8, pitch, off, fill=93 if ty is E4M3 else None)
        total, tbuf = placed(T, D, ts, pitch, off)
        rstd = torch.empty(T, device="cuda")
        groups = 0 if ty is not E4M3 else ((D + 127) // 128 if n == 2 else 1)
        scale = torch.empty(T, groups, device="cuda") if groups else None
        ops.cocodc_lm_norm(put(x, pitch, off), w, y.view(E4M3) if groups else y, residual=put(r, pitch, off) if residual else None,
                           total=total if residual else None, rstd=rstd, y_scale=scale, eps=EPS)
        z = x.double()
        if residual:
            want = x.double() + r.double()
            within(total, want, want.abs() * E24, "total")
            untouched(total, tbuf, float("nan"))
            z = total.double()
        k = (z.square().mean(1) + EPS).rsqrt()
        ek = (chain(D) / 2 + 4) * E24
        within(rstd, k, k * ek, "rstd")
        want = z * k[:, None] * w.double()
        if not groups:
            within(y, want, want.abs() * (ek + 2 * E24), "y")
            untouched(y, buf, float("nan"))
            continue
        untouched(y, buf, 93)
        width = 128 if n == 2 else D
        top = torch.stack([q.abs().amax(1) for q in want.split(width, 1)], 1) / 448
        within(scale, top.clamp(min=1e-30), top * (ek + 4 * E24), "scale")
        s = scale.double().repeat_interleave(width, 1)[:, :D]
        q = want / s
        lim = spacing_8(q) / 2 * (1 + 2.0 ** -20) + q.abs() * (ek + 8 * E24)
        assert bool(((y.view(E4M3).double() - q).abs() <= lim).all())


@pytest.mark.parametrize("T,D", SIZES + [(5000, 256), (40000, 64)])
@pytest.mark.parametrize("ty,ts,tw,td", [(BF16, BF16, F32, F32), (BF16, F32, BF16, BF16), (F16, F16, F16, F32), (F32, F32, F32, F32)])
@pytest.mark.parametrize("stream", [True, False])
def test_norm_grad(ops, T, D, ty, ts, tw, td, stream):
    g = gen(2 * T + D)
    s, dy, dt, w = randn(g, T, D, std=2.0, dtype=ts), randn(g, T, D, dtype=ty), randn(g, T, D, dtype=ts), randn(g, D, std=0.3).add(1).to(tw)
    rstd = (s.double().square().mean(1) + EPS).rsqrt().float()
    k, h = rstd.double()[:, None], s.double() * rstd.double()[:, None]
    gd = dy.double() * w.double()
    mean = (gd * h).mean(1, keepdim=True)
    want = k * (gd - h * mean) + (dt.double() if stream else 0)
    emean = (chain(D) + 2) * E24 * (gd * h).abs().mean(1, keepdim=True) + mean.abs() * E24
    bound = k * (2 * E24 * gd.abs() + h.abs() * (emean + 3 * E24 * mean.abs())) + 2 * E24 * want.abs()
    want_w, bound_w = (dy.double() * h).sum(0), (min(T, T // 592) + 100 + (T if T < 592 else 0)) * E24 * (dy.double() * h).abs().sum(0)
    for pitch, off in ((D, 0), (D + 3, 1), ((D + 15) // 8 * 8, 8)):
        dx, buf = placed(T, D, ts, pitch, off)
        dw = torch.full((D,), 0.5, device="cuda", dtype=td)
        ops.cocodc_lm_norm_grad(put(dy, pitch, off), put(s, pitch, off), w, rstd, dx, dweight=dw, dtotal=put(dt, pitch, off) if stream else None)
        within(dx, want, bound, "dx")
        untouched(dx, buf, float("nan"))
        within(dw, want_w, bound_w, "dweight")
    ops.cocodc_lm_norm_grad(dy, s, w, rstd, None, dweight=dw, accumulate=True)
    first = (dy.double() * h).sum(0).to(td).double()
    within(dw, want_w + first, bound_w * 3 + want_w.abs() * torch.finfo(td).eps, "accumulated")
    only = torch.empty_like(s)
    ops.cocodc_lm_norm_grad(dy, s, w, rstd, only, dtotal=dt if stream else None)
    within(only, want, bound, "dx alone")


def test_norm_gradient_against_differences(ops):
    """sum(dy y) along a direction, by central differences of the 64-bit definition."""
    g = gen(5)
    T, D, h = 7, 200, 1e-5
    s, dy, w = randn(g, T, D, std=2.0), randn(g, T, D), randn(g, D).add(1)
    rstd, dx, dw = (s.double().square().mean(1) + EPS).rsqrt().float(), torch.empty_like(s), torch.empty(D, device="cuda")
    ops.cocodc_lm_norm_grad(dy, s, w, rstd, dx, dweight=dw)

    def loss(s, w):
        return (dy.double() * s * (s.square().mean(1, keepdim=True) + EPS).rsqrt() * w).sum()

    a, b = randn(g, T, D).double(), randn(g, D).double()
    by_s = (loss(s.double() + h * a, w.double()) - loss(s.double() - h * a, w.double())) / (2 * h)
    by_w = (loss(s.double(), w.double() + h * b) - loss(s.double(), w.double() - h * b)) / (2 * h)
    # fp32 gradients: about 60 roundings of their terms; differences: h^2 and 1e-16 / h
    assert abs(float((dx.double() * a).sum() - by_s)) < 60 * E24 * float((dx.double() * a).abs().sum()) + 1e-7
    assert abs(float((dw.double() * b).sum() - by_w)) < 60 * E24 * float((dw.double() * b).abs().sum()) + 1e-7


def test_the_residual_stream_in_place_and_repeated(ops):
    g = gen(3)
    for T, D, ts in ((5, 2048, BF16), (700, 1024, F32), (9, 9000, BF16), (600, 777, BF16)):
        x, r, w, dy = randn(g, T, D, dtype=BF16), randn(g, T, D, dtype=ts), randn(g, D), randn(g, T, D, dtype=BF16)
        y, y2, total, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty_like(r), torch.empty(T, device="cuda")
        ops.cocodc_lm_norm(x, w, y, residual=r, total=total, rstd=rstd)
        q = r.clone()
        ops.cocodc_lm_norm(x, w, y2, residual=q, total=q)
        assert torch.equal(y, y2) and torch.equal(q, total)
        dt = randn(g, T, D, dtype=ts)
        dx, dw, dw2 = torch.empty_like(total), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
        ops.cocodc_lm_norm_grad(dy, total, w, rstd, dx, dweight=dw, dtotal=dt)
        ops.cocodc_lm_norm_grad(dy, total, w, rstd, dt, dweight=dw2, dtotal=dt)
        assert torch.equal(dx, dt) and torch.equal(dw, dw2)


@pytest.mark.parametrize("T,D", [(3, 256), (700, 256), (700, 2000), (4, 9000)])
def test_rows_that_are_not_finite_stay_by_themselves(ops, T, D):
    g = gen(8)
    x, w = randn(g, T, D), torch.ones(D, device="cuda")
    x[0, 3], x[1, 5] = float("nan"), float("inf")
    x[2] = 0
    for group in (0, 128):
        y8, scale = torch.empty(T, D, dtype=E4M3, device="cuda"), torch.empty(T, (D + 127) // 128 if group else 1, device="cuda")
        y, rstd = torch.empty_like(x), torch.empty(T, device="cuda")
        ops.cocodc_lm_norm(x, w, y, rstd=rstd, eps=0.0)
        assert bool(torch.isnan(y[0]).all()) and rstd[1] == 0 and bool(torch.isnan(y[1, 5])) and bool((y[1, 6:] == 0).all())
        assert bool(torch.isnan(y[2]).all())                                  # 0 times infinity: eps is what prevents it
        ops.cocodc_lm_norm(x, w, y8, y_scale=scale, eps=EPS)
        f = y8.float()
        assert bool(torch.isnan(f[0]).all()) and bool(torch.isnan(f[1, 5])) and bool((f[1, 6:] == 0).all()) and bool((f[2] == 0).all())
        assert bool((scale[:3] == torch.tensor(1e-30, device="cuda")).all()) and bool(torch.isfinite(f[3:]).all())


def test_empty_and_captured(B, ops):
    w = torch.ones(64, device="cuda")
    empty = torch.empty(0, 64, device="cuda")
    ops.cocodc_lm_norm(empty, w, empty.clone(), rstd=torch.empty(0, device="cuda"))
    dw = torch.full((64,), 3.0, device="cuda")
    ops.cocodc_lm_norm_grad(empty, empty, w, torch.empty(0, device="cuda"), None, dweight=dw, accumulate=True)
    assert bool((dw == 3).all())
    ops.cocodc_lm_norm_grad(empty, empty, w, torch.empty(0, device="cuda"), None, dweight=dw)
    assert bool((dw == 0).all())
    g = gen(1)
    x, dy = randn(g, 300, 640), randn(g, 300, 640)
    w = randn(g, 640)
    y, rstd, dx, dw = torch.empty_like(x), torch.empty(300, device="cuda"), torch.empty_like(x), torch.empty(640, device="cuda")
    ws = torch.empty(B.library().cocodc_lm_norm_grad_workspace(300, 640), dtype=torch.uint8, device="cuda")

    def both():
        ops.cocodc_lm_norm(x, w, y, rstd=rstd)
        ops.cocodc_lm_norm_grad(dy, x, w, rstd, dx, dweight=dw, workspace=ws)

    both()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
        with torch.cuda.graph(graph, stream=side):
            both()
    torch.cuda.current_stream().wait_stream(side)
    for k in range(2):
        x.copy_(randn(g, 300, 640))
        graph.replay()
        got = [t.clone() for t in (y, rstd, dx, dw)]
        both()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, rstd, dx, dw)))


def test_refusals_of_the_binding(B, ops):
    x, w = torch.randn(4, 256, device="cuda"), torch.ones(256, device="cuda")
    y, y8 = torch.empty_like(x), torch.empty(4, 256, dtype=E4M3, device="cuda")
    launches = ops.launch_count
    for bad in (dict(x=x[:3]), dict(weight=w[:255]), dict(y=x.t()), dict(x=x.double()), dict(y=y8, y_scale=torch.empty(4, 3, device="cuda")), dict(x=x.cpu()),
                dict(residual=x.half(), total=x.clone()), dict(rstd=torch.empty(3, device="cuda"))):
        with pytest.raises(ValueError):
            ops.cocodc_lm_norm(**{**dict(x=x, weight=w, y=y), **bad})
    for bad in (dict(y=y8), dict(residual=x.clone()), dict(total=x.clone()), dict(y=y, y_scale=torch.empty(4, device="cuda")), dict(eps=-1.0), dict(y=x)):
        with pytest.raises(B.CocodcError):
            ops.cocodc_lm_norm(**{**dict(x=x, weight=w, y=y), **bad})
    assert ops.launch_count == launches
