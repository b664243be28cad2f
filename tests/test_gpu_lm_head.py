"""The output head with its loss, and its gradient, against plain implementations in 64 bits.

Bounds, derived before any run (u = half the spacing of the type, e = 2^-24):
  logits    D products accumulated in fp32, which a tensor core may cut instead of round: 2 D e sum |x w|, times the scale, and 2 e |z|
  lse       an error of the logits' largest; z is rounded (base 2) and the exponential is 2^-22 off: e (3 max |z| + 300), sums of
            positive terms in less than 256 steps among them
  logp      both logit's and lse's errors, and 2 e (|z| + |lse|)
  dz        p is off by E = the logit's error + e (2 |z| + |lse|) + 2^-21 relatively: E p |slope|, 4 e (p |slope| + |hit|), then rounded: u |dz| (+ fp16: 2^-25
            of the power of two)
  dx, dtable   the sums of |dz error| |w| (|x|), the accumulation's 2 K e sum |dz w|, one rounding (accumulated: e of the sum)
"""

import math

import pytest
import torch
from test_gpu_lm_ops import E24, UNIT, gen, placed, put, randn, untouched, within

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


def inputs(T, D, V, kind, seed=0, std=2.0):
    g = gen(T + D + V + seed)
    x, w = randn(g, T, D, dtype=kind), randn(g, V, D, std=std * D ** -0.5, dtype=kind)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    ids[torch.rand(T, generator=g, device="cuda") < 0.1] = -1
    return g, x, w, ids


def logits(x, w, scale):
    z = (x.double() @ w.double().t()) * scale
    ez = 2 * x.shape[1] * E24 * (x.double().abs() @ w.double().abs().t()) * scale + 2 * E24 * z.abs()
    return z, ez


def statistics(z, ez, ids):
    lse = torch.logsumexp(z, 1)
    el = ez.amax(1) + E24 * (3 * z.abs().amax(1) + 300)
    at = ids.clamp(min=0).unsqueeze(1)
    zy, ey = z.gather(1, at).squeeze(1), ez.gather(1, at).squeeze(1)
    logp = torch.where(ids >= 0, zy - lse, torch.zeros_like(lse))
    return lse, el, logp, torch.where(ids >= 0, ey + el + 2 * E24 * (zy.abs() + lse.abs()), torch.zeros_like(lse))


SIZES = [(1, 1, 1), (1, 64, 1000), (1, 2048, 32000), (3, 72, 257), (7, 100, 333), (17, 64, 64), (33, 520, 1003), (128, 128, 512), (129, 136, 255), (200, 33, 700),
         (257, 768, 2049), (500, 64, 5003), (1333, 264, 1500)]


@pytest.mark.parametrize("T,D,V", SIZES)
@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("scale", [1.0, 1.7])
def test_head(ops, T, D, V, kind, scale):
    g, x, w, ids = inputs(T, D, V, kind)
    z, ez = logits(x, w, scale)
    lse, el, logp, ep = statistics(z, ez, ids)
    for i, (pitch, off) in enumerate(((D, 0), (D + 3, 1), ((D + 15) // 8 * 8, 8))):
        got, gl = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
        ops.cocodc_lm_head(put(x, pitch, off), put(w, pitch, off), ids.to(torch.int32 if i == 1 else torch.int64), got, lse=gl, scale=scale)
        within(gl, lse, el, "lse")
        within(got, logp, ep, "logp")
    ops.cocodc_lm_head(x, w, None, None, lse=gl, scale=scale)
    within(gl, lse, el, "lse alone")
    ops.cocodc_lm_head(x, w, ids, got, scale=scale)
    within(got, logp, ep, "logp alone")


GRADS = [(1, 64, 1000), (3, 72, 257), (7, 100, 333), (33, 520, 1003), (128, 128, 512), (129, 136, 255), (200, 33, 700), (257, 768, 2049), (500, 64, 5003),
         (1333, 264, 1500), (40, 2048, 4000)]


def gradient(x, w, ids, lse, dlogp, dlse, scale):
    z, ez = logits(x, w, scale)
    d = torch.where(ids >= 0, dlogp.double(), torch.zeros_like(lse.double())) if dlogp is not None else torch.zeros_like(lse.double())
    slope = (dlse.double() if dlse is not None else 0) - d
    p = torch.exp(z - lse.double()[:, None])
    hit = torch.zeros_like(z).scatter_(1, ids.clamp(min=0).unsqueeze(1), d.unsqueeze(1))
    dz = p * slope[:, None] + hit
    ps = p * slope.abs()[:, None]
    edz = ps * (ez + E24 * (2 * z.abs() + lse.double().abs()[:, None]) + 2.0 ** -21) + 4 * E24 * (ps + hit.abs())
    edz = edz + UNIT[x.dtype] * (dz.abs() + edz)
    if x.dtype is F16:
        edz = edz + 2.0 ** -25 * float((d.abs() + (dlse.double().abs() if dlse is not None else 0)).max()) * 2.0 ** -9
    both = dz.abs() + edz
    wd, xd = w.double(), x.double()
    dx, ex = dz @ wd * scale, (edz @ wd.abs() + 2 * dz.shape[1] * E24 * (both @ wd.abs())) * scale
    dw, ew = dz.t() @ xd * scale, (edz.t() @ xd.abs() + 2 * dz.shape[0] * E24 * (both.t() @ xd.abs())) * scale
    return dx, ex + 4 * E24 * dx.abs(), dw, ew + 4 * E24 * dw.abs()


@pytest.mark.parametrize("T,D,V", GRADS)
@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("which", ["both", "logp", "lse"])
def test_head_grad(ops, T, D, V, kind, which):
    g, x, w, ids = inputs(T, D, V, kind, seed=1)
    scale = 1.3
    lse = torch.logsumexp(logits(x, w, scale)[0], 1).float()
    dlogp = None if which == "lse" else randn(g, T, std=1e-4 if kind is F16 else 1.0)
    dlse = None if which == "logp" else randn(g, T, std=1e-5 if kind is F16 else 0.3)
    targets = None if which == "lse" else ids
    dx, ex, dw, ew = gradient(x, w, ids, lse, dlogp, dlse, scale)
    for n, (pitch, off, tw) in enumerate(((D, 0, kind), (D + 3, 1, F32), ((D + 15) // 8 * 8, 8, F32), ((D + 15) // 8 * 8, 8, kind))):
        gx, bx = placed(T, D, kind, pitch, off)
        gw, bw = placed(V, D, tw, pitch, off)
        ops.cocodc_lm_head_grad(put(x, pitch, off), put(w, pitch, off), targets, lse, dlogp, dlse, gx, gw, scale=scale)
        within(gx, dx, ex, ("dx", n))
        within(gw, dw, ew, ("dtable", n))
        untouched(gx, bx, float("nan"))
        untouched(gw, bw, float("nan"))
    first = gw.clone()
    ops.cocodc_lm_head_grad(x, w, targets, lse, dlogp, dlse, None, gw, scale=scale, accumulate=True)
    within(gw, first.double() + dw, ew + E24 * (dw.abs() + first.double().abs()), "accumulated")
    alone = torch.empty_like(x)
    ops.cocodc_lm_head_grad(x, w, targets, lse, dlogp, dlse, alone, None, scale=scale)
    within(alone, dx, ex, "dx alone")


@pytest.mark.parametrize("kind,D", [(BF16, 64), (F16, 64), (BF16, 50)])
def test_several_pieces_of_the_vocabulary(B, ops, kind, D):
    """Enough rows that dz is made in pieces: sums of dx over them, and every row of the table's gradient."""
    T, V = 40000 if D == 64 else 140000, 9001 if D == 64 else 1500
    g, x, w, ids = inputs(T, D, V, kind, seed=2)
    assert B.library().cocodc_lm_head_grad_workspace(T, D, V) < 2 * T * V
    lse, dlogp = torch.empty(T, device="cuda"), randn(g, T, std=1e-3)
    logp = torch.empty(T, device="cuda")
    ops.cocodc_lm_head(x, w, ids, logp, lse=lse)
    gx, gw = torch.empty_like(x), torch.empty_like(w)
    ops.cocodc_lm_head_grad(x, w, ids, lse, dlogp, None, gx, gw)
    dwant, ewant = torch.zeros(V, D, dtype=torch.float64, device="cuda"), torch.zeros(V, D, dtype=torch.float64, device="cuda")
    for a in range(0, T, 4000):
        part = slice(a, a + 4000)
        z, ez = logits(x[part], w, 1.0)
        l, el, lp, ep = statistics(z, ez, ids[part])
        within(lse[part], l, el, "lse")
        within(logp[part], lp, ep, "logp")
        dx, ex, dw, ew = gradient(x[part], w, ids[part], lse[part], dlogp[part], None, 1.0)
        within(gx[part], dx, ex, "dx")
        dwant += dw
        ewant += ew + 2 * T * E24 * dw.abs()
    within(gw, dwant, ewant, "dtable")


def test_head_gradient_against_differences(ops):
    """The mean log probability along a direction, by central differences of the 64-bit definition; lse to its own accuracy."""
    T, D, V, h = 60, 128, 900, 1e-5
    g, x, w, ids = inputs(T, D, V, BF16, seed=3)
    lse = torch.logsumexp(x.double() @ w.double().t(), 1).float()
    dlogp, dx, dw = torch.full((T,), -1.0 / T, device="cuda"), torch.empty_like(x), torch.empty(V, D, device="cuda")
    ops.cocodc_lm_head_grad(x, w, ids, lse, dlogp, None, dx, dw)

    def loss(x, w):
        lp = torch.log_softmax(x @ w.t(), 1)
        return -(lp.gather(1, ids.clamp(min=0).unsqueeze(1)).squeeze(1) * (ids >= 0)).sum() / T

    a, b = randn(g, T, D).double(), randn(g, V, D).double()
    by_x = (loss(x.double() + h * a, w.double()) - loss(x.double() - h * a, w.double())) / (2 * h)
    by_w = (loss(x.double(), w.double() + h * b) - loss(x.double(), w.double() - h * b)) / (2 * h)
    # dz is rounded to bfloat16 once (2^-9 on average over its terms), dx once more
    assert abs(float((dx.double() * a).sum() - by_x)) < 2.0 ** -8 * float((dx.double() * a).abs().sum())
    assert abs(float((dw.double() * b).sum() - by_w)) < 2.0 ** -8 * float((dw.double() * b).abs().sum())


@pytest.mark.parametrize("T,D,V,off", [(6, 64, 500, 0), (300, 64, 500, 0), (6, 64, 500, 1)])
def test_values_that_are_not_finite(ops, T, D, V, off):
    g, x, w, ids = inputs(T, D, V, BF16, seed=4)
    ids[:5] = 3
    x[0, 0] = float("nan")
    x[1] = 0
    x[1, 0], x[2] = 1, 0
    x[2, 0] = -1
    w[:, 0] = 0
    w[7, 0] = float("inf")                         # row 1: one logit is +Inf, row 2: one is -Inf (others: +-Inf or NaN there)
    x[3:, 0] = -1
    x, w = put(x, D + off, off), put(w, D + off, off)
    logp, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ops.cocodc_lm_head(x, w, ids, logp, lse=lse)
    assert bool(torch.isnan(lse[:2]).all()) and bool(torch.isnan(logp[:2]).all())
    z, ez = logits(x[2:], w, 1.0)
    ez[:, 7] = 0
    keep = torch.arange(V, device="cuda") != 7
    want, el, lp, ep = statistics(z[:, keep], ez[:, keep], torch.where(ids[2:] == 7, -1, ids[2:] - (ids[2:] > 7).long()))
    within(lse[2:], want, el, "lse")
    within(torch.where(ids[2:] == 7, torch.zeros_like(logp[2:]), logp[2:]), torch.where(ids[2:] == 7, torch.zeros_like(lp), lp), ep, "logp")
    # nothing but -Inf
    w2 = torch.full((V, D), 0.0, device="cuda", dtype=BF16)
    w2[:, 0] = float("-inf")
    x2 = torch.zeros(T, D, device="cuda", dtype=BF16)
    x2[:, 0] = 1
    x2, w2 = put(x2, D + off, off), put(w2, D + off, off)
    ops.cocodc_lm_head(x2, w2, torch.full((T,), 2, device="cuda"), logp, lse=lse)
    assert bool((lse == float("-inf")).all()) and bool((logp == float("-inf")).all())


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("kind", [BF16, F16])
def test_rows_that_get_nothing(ops, off, kind):
    """Rows without a target, with lse -Inf, or with factors of zero add nothing; a NaN lse gives NaN; all of them without a target: zeros."""
    T, D, V = 140, 64, 300
    g, x, w, ids = inputs(T, D, V, kind, seed=5)
    x, w = put(x, D + off, off), put(w, D + off, off)
    lse = torch.logsumexp(x.double() @ w.double().t(), 1).float()
    dlogp = torch.ones(T, device="cuda")
    ids[:6] = torch.tensor([-1, 4, 4, 4, -7, 5], device="cuda")
    lse[1], dlogp[2], lse[0], lse[4] = float("-inf"), 0.0, float("nan"), float("inf")
    dx, dw = torch.empty(T, D, dtype=kind, device="cuda"), torch.empty(V, D, device="cuda")
    ops.cocodc_lm_head_grad(x, w, ids, lse, dlogp, None, dx, dw)
    assert bool((dx[:3] == 0).all()) and bool((dx[4] == 0).all()) and bool(torch.isfinite(dx).all())
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[:3] = keep[4] = False
    wx, ex, ww, ew = gradient(x[keep], w, ids[keep], lse[keep], dlogp[keep], None, 1.0)
    within(dx[keep], wx, ex, "dx")
    within(dw, ww, ew, "dtable")
    lse[3] = float("nan")
    ops.cocodc_lm_head_grad(x, w, ids, lse, dlogp, None, dx, dw)
    assert bool(torch.isnan(dx[3]).all()) and bool((dx[2] == 0).all()) and bool(torch.isnan(dw).all())
    ops.cocodc_lm_head_grad(x, w, torch.full_like(ids, -1), lse, dlogp, None, dx, dw)
    assert bool((dx == 0).all()) and bool((dw == 0).all())


def test_targets_outside_the_vocabulary(B):
    ops = B.LmOps(0)
    g, x, w, ids = inputs(9, 64, 100, BF16, seed=6)
    bad = ids.clone()
    bad[4], ids[4] = 100, -1
    logp, want, lse = (torch.empty(9, device="cuda") for _ in range(3))
    ops.cocodc_lm_head(x, w, ids, want, lse=lse)
    assert ops.cocodc_lm_poll_status() == B.OK
    ops.cocodc_lm_head(x, w, bad, logp)
    assert torch.equal(logp, want) and ops.cocodc_lm_poll_status() == B.ERR_INVALID_ARG
    one = torch.ones(9, device="cuda")
    dx, dx2 = torch.empty_like(x), torch.empty_like(x)
    ops.cocodc_lm_head_grad(x, w, ids, lse, one, None, dx)
    assert ops.cocodc_lm_poll_status() == B.OK
    ops.cocodc_lm_head_grad(x, w, bad, lse, one, None, dx2)
    assert torch.equal(dx, dx2) and ops.cocodc_lm_poll_status() == B.ERR_INVALID_ARG


@pytest.mark.parametrize("kind", [BF16, F16])
def test_large_logits_and_scales(ops, kind):
    """Logits in the thousands, and offsets that a row shares, cost no more than the bound says."""
    T, D, V = 150, 64, 1000
    g, x, w, ids = inputs(T, D, V, kind, seed=7, std=200.0)
    for scale in (1.0, 1e-3, 30.0):
        z, ez = logits(x, w, scale)
        lse, el, logp, ep = statistics(z, ez, ids)
        got, gl = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        ops.cocodc_lm_head(x, w, ids, got, lse=gl, scale=scale)
        within(gl, lse, el, "lse")
        within(got, logp, ep, "logp")


def test_empty_calls(ops):
    x, w = torch.empty(0, 64, dtype=BF16, device="cuda"), torch.randn(100, 64, device="cuda").bfloat16()
    n = torch.empty(0, device="cuda")
    ops.cocodc_lm_head(x, w, torch.empty(0, dtype=torch.int64, device="cuda"), n, lse=n.clone())
    for kind in (F32, BF16):
        dw = torch.full((100, 72), 2.0, device="cuda", dtype=kind)
        ops.cocodc_lm_head_grad(x, w, torch.empty(0, dtype=torch.int64, device="cuda"), n, n.clone(), None, None, dw[:, :64], accumulate=True)
        assert bool((dw == 2).all())
        ops.cocodc_lm_head_grad(x, w, torch.empty(0, dtype=torch.int64, device="cuda"), n, n.clone(), None, None, dw[:, :64])
        assert bool((dw[:, :64] == 0).all()) and bool((dw[:, 64:] == 2).all())


def test_streams_graphs_and_repeated_calls(B, ops):
    """The same bits on another stream, from a graph on new inputs, and again; two workspaces at once."""
    T, D, V = 300, 256, 3001
    g, x, w, ids = inputs(T, D, V, BF16, seed=8)
    ids = ids.clamp(min=0)
    dlogp = randn(g, T)
    size = B.library().cocodc_lm_head_workspace(T, D, V), B.library().cocodc_lm_head_grad_workspace(T, D, V)

    def buffers():
        return dict(logp=torch.empty(T, device="cuda"), lse=torch.empty(T, device="cuda"), dx=torch.empty_like(x), dw=torch.empty(V, D, device="cuda"),
                    ws=[torch.full((n,), 0xff, dtype=torch.uint8, device="cuda") for n in size])

    def step(b, stream=None):
        ops.cocodc_lm_head(x, w, ids, b["logp"], lse=b["lse"], workspace=b["ws"][0], stream=stream)
        ops.cocodc_lm_head_grad(x, w, ids, b["lse"], dlogp, None, b["dx"], b["dw"], workspace=b["ws"][1], stream=stream)

    def same(a, b):
        return all(torch.equal(a[k], b[k]) for k in ("logp", "lse", "dx", "dw"))

    first = buffers()
    step(first)
    streams = [torch.cuda.Stream() for _ in range(2)]
    others = [buffers() for _ in streams]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, b in zip(streams, others):
            step(b, s)
    torch.cuda.synchronize()
    assert all(same(first, b) for b in others)
    graph, held = torch.cuda.CUDAGraph(), buffers()
    with torch.cuda.graph(graph):
        step(held)
    for _ in range(2):
        x.copy_(randn(g, T, D, dtype=BF16))
        graph.replay()
        step(first)
        assert same(first, held)


def test_offsets_past_32_bits(ops):
    """A table of more than 2^31 elements: its last rows are read, and their gradient is written, where they are."""
    V, D, T = 140001, 16384, 2
    w = torch.zeros(V, D, dtype=BF16, device="cuda")
    g = gen(9)
    last = randn(g, 3, D, std=0.05, dtype=BF16)
    w[-3:] = last
    x = randn(g, T, D, dtype=BF16)
    ids = torch.tensor([V - 1, V - 3], device="cuda")
    logp, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ops.cocodc_lm_head(x, w, ids, logp, lse=lse)
    z, ez = logits(x, last, 1.0)
    m = z.amax(1)
    want = m + torch.log(torch.exp(z - m[:, None]).sum(1) + (V - 3) * torch.exp(-m))
    within(lse, want, ez.amax(1) + E24 * (3 * z.abs().amax() + 300 + math.log(V)), "lse")
    within(logp, z[[0, 1], [2, 0]] - want, 3 * ez.amax(1) + 2 * E24 * (3 * z.abs().amax() + 300 + math.log(V)), "logp")
    dw, dx = torch.full((V, D), 5.0, dtype=BF16, device="cuda"), torch.empty_like(x)
    ops.cocodc_lm_head_grad(x, w, ids, lse, torch.ones(T, device="cuda"), None, dx, dw)
    p = torch.exp(torch.cat([z, torch.zeros(T, 1, dtype=torch.float64, device="cuda")], 1) - lse.double()[:, None])
    dz = -p
    dz[0, 2] += 1
    dz[1, 0] += 1
    got = dw[[V - 3, V - 2, V - 1, 0, 70000]].double()
    ref = torch.stack([dz[:, 0], dz[:, 1], dz[:, 2], dz[:, 3], dz[:, 3]]) @ x.double()
    # dz is rounded to bfloat16, then the result (and z's own error)
    lim = (2.0 ** -8 + 4 * float(ez.max())) * (torch.stack([dz[:, 0], dz[:, 1], dz[:, 2], dz[:, 3], dz[:, 3]]).abs() @ x.double().abs()) + 2.0 ** -8 * ref.abs() + 1e-30
    assert bool(((got - ref).abs() <= lim).all())
    assert not bool((dw[::1000] == 5).any())


def test_refusals_of_the_binding(B, ops):
    x, w, ids = torch.randn(4, 64, device="cuda").bfloat16(), torch.randn(100, 64, device="cuda").bfloat16(), torch.zeros(4, dtype=torch.int64, device="cuda")
    lse, out, dx = torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(x)
    launches = ops.launch_count
    for bad in (dict(table=w[:, :63]), dict(x=x.half()), dict(targets=ids[:3]), dict(logp=out[:3]), dict(logp=out.double()), dict(x=x.cpu()), dict(targets=ids.int().float())):
        with pytest.raises(ValueError):
            ops.cocodc_lm_head(**{**dict(x=x, table=w, targets=ids, logp=out), **bad})
    for bad in (dict(x=x.float(), table=w.float()), dict(scale=0.0), dict(targets=None), dict(logp=None), dict(logp=out, lse=out),
                dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(B.CocodcError):
            ops.cocodc_lm_head(**{**dict(x=x, table=w, targets=ids, logp=out), **bad})
    for bad in (dict(dx=dx[:3]), dict(dtable=w[:99].clone()), dict(dlogp=out[:3]), dict(dx=dx.float())):
        with pytest.raises(ValueError):
            ops.cocodc_lm_head_grad(**{**dict(x=x, table=w, targets=ids, lse=lse, dlogp=out, dlse=None, dx=dx), **bad})
    for bad in (dict(dx=x), dict(dtable=w), dict(dx=None), dict(dtable=w.half()), dict(dlogp=None), dict(lse=None),
                dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(B.CocodcError):
            ops.cocodc_lm_head_grad(**{**dict(x=x, table=w, targets=ids, lse=lse, dlogp=out, dlse=None, dx=dx), **bad})
    assert ops.launch_count == launches
