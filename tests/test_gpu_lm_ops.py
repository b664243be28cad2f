"""Operators of the local step (embedding lookup, gated block, token log probabilities, and their gradients) against plain
implementations in 64 bits.

Bounds, derived before any run (u = half the spacing of the output type, torch.finfo(type).eps / 2, relative to the value's
power of two: |error| <= u |value|, plus half the smallest subnormal; e = 2^-24):
  lookup          one fp32 product, rounded once: the same bits as (W.float() * scale).to(type)
  table gradient  n terms added in fp32 in some order: (n + 2) e sum |scale * dy|, then one rounding
  products        K terms accumulated in fp32; a tensor core may cut instead of round, so 2 e a step: 2 K e sum |a b|
  h               |act'| <= 1.13: 1.13 |u| err(g) + (|act(g)| + |act'| err(g)) err(u) + 2^-18 |h| for the approximate exponential
                  and division, then one rounding
  dx, dw          dg and du are rounded to the type first (u each, plus the 2^-18), then the products' bound, one rounding
  log-sum-exp     z = scale * x costs e |z| three times over, the exponential 2^-22, the sum less than 256 rounding steps
                  of positive terms: E = e (3 max|z| + 300); the log probability the same plus e |logp|
  entropy         p is E off relatively, so is each term: 2 E (1 + H + range of z's that matter <= 40)
  logit gradient  p off by E' = 2 E relatively: E' (|g| p + |h| p (|lp| + H + 1)), then one rounding
"""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

E24 = 2.0 ** -24
UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16, torch.float32)}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}
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


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, std=1.0, dtype=F32):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def placed(rows, cols, dtype, pitch=None, offset=0, fill=None):
    """A rows x cols view with row stride `pitch` that starts `offset` elements into its buffer."""
    pitch = cols if pitch is None else pitch
    buf = torch.empty(offset + max(1, rows) * pitch + 16, dtype=dtype, device="cuda")
    buf.fill_(float("nan") if fill is None else fill)
    return buf[offset:offset + rows * pitch].view(rows, pitch)[:, :cols], buf


def put(x, pitch=None, offset=0):
    v, _ = placed(*x.shape, x.dtype, pitch, offset)
    v.copy_(x)
    return v


def within(got, want, bound, what=""):
    """Every element of got within bound of want after its own type's rounding; non-finite values agree exactly."""
    u, tiny = UNIT[got.dtype], TINY[got.dtype]
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what
    ok = torch.isfinite(want)
    err = (got - want).abs()[ok]
    lim = (bound + u * (want.abs() + bound) + tiny)
    lim = lim.expand_as(want)[ok] if isinstance(lim, torch.Tensor) else lim
    assert bool((err <= lim).all()), (what, float((err / lim).max()))


def untouched(view, buf, fill):
    """The bytes of buf outside view still hold the fill value."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    off = view.storage_offset()
    rows, cols = view.shape
    for r in range(rows):
        mask[off + r * view.stride(0): off + r * view.stride(0) + cols] = False
    rest = buf[mask]
    assert bool((torch.isnan(rest) if math.isnan(fill) else rest == fill).all())


# ---------------------------------------------------------------------------------------------------- embedding lookup

@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (1, 50257, 768), (7, 300, 33), (33, 17, 8), (64, 1000, 1024), (1000, 50, 257),
                                   (129, 5000, 4104)])
@pytest.mark.parametrize("tin,tout", [(F32, BF16), (BF16, BF16), (F16, F32), (F32, F32), (BF16, F16)])
def test_embed(ops, T, V, D, tin, tout):
    g = gen(T + V + D)
    w = randn(g, V, D, dtype=tin)
    ids = torch.randint(-1, V, (T,), generator=g, device="cuda")
    for kind, pitch_w, pitch_y, off in ((torch.int64, D, D, 0), (torch.int32, D + 3, D + 5, 1), (torch.int64, D + 8, D + 16, 8)):
        y, buf = placed(T, D, tout, pitch_y, off)
        ops.cocodc_lm_embed(put(w, pitch_w, off), ids.to(kind), y, scale=1.7)
        want = (w[ids.clamp(min=0)].float() * torch.tensor(1.7, device="cuda")).to(tout)
        want[ids < 0] = 0
        assert torch.equal(y, want)
        untouched(y, buf, float("nan"))


def test_embed_ids_outside_the_table(B, ops):
    w = torch.ones(10, 16, device="cuda")
    y = torch.full((4, 16), 9.0, device="cuda")
    ops.cocodc_lm_embed(w, torch.tensor([3, 10, -7, 2 ** 40], device="cuda"), y)
    assert y[:, 0].tolist() == [1, 0, 0, 0]
    assert ops.cocodc_lm_poll_status() == B.ERR_INVALID_ARG and ops.cocodc_lm_poll_status() == B.OK


# --------------------------------------------------------------------------------------------------- its gradient

def embed_grad_ref(dy, ids, V, scale):
    keep = (ids >= 0) & (ids < V)
    d = dy.double()[keep]
    ref = torch.zeros(V, dy.shape[1], dtype=torch.float64, device="cuda").index_add_(0, ids[keep].long(), d) * scale
    mag = torch.zeros_like(ref).index_add_(0, ids[keep].long(), d.abs()) * abs(scale)
    n = torch.bincount(ids[keep].long(), minlength=V).double()
    return ref, (n + 2).unsqueeze(1) * E24 * mag


@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (1, 4000, 64), (31, 7, 8), (32, 50257, 96), (33, 2, 40), (500, 300, 768), (4099, 1000, 136),
                                   (3000, 120000, 16), (5000, 3, 520), (257, 129, 77), (700, 40, 2056), (20000, 800, 24)])
@pytest.mark.parametrize("tin,tout", [(BF16, F32), (F32, F32), (F16, F16), (BF16, BF16)])
def test_embed_grad(ops, T, V, D, tin, tout):
    g = gen(T * 3 + V + D)
    dy = randn(g, T, D, dtype=tin)
    ids = (torch.exp(torch.rand(T, generator=g, device="cuda") * math.log(V + 1)).long() - 1).clamp_(0, V - 1)
    ids[torch.rand(T, generator=g, device="cuda") < 0.05] = -1
    ref, bound = embed_grad_ref(dy, ids, V, 0.75)
    for kind, pd, pg, off in ((torch.int64, D, D, 0), (torch.int32, D + 3, D + 1, 1), (torch.int32, D + 8, D + 8, 8)):
        got, buf = placed(V, D, tout, pg, off)
        d = put(dy, pd, off)
        ops.cocodc_lm_embed_grad(d, ids.to(kind), got, scale=0.75)
        within(got, ref, bound, "plain")
        if V < 2000:
            untouched(got, buf, float("nan"))
        again = torch.empty_like(got).copy_(got)
        ops.cocodc_lm_embed_grad(d, ids.to(kind), got, scale=0.75)
        assert torch.equal(again, got)                      # the same bits every time
        if tout == F32:
            start = randn(g, V, D)
            acc = put(start, pg, off)
            ops.cocodc_lm_embed_grad(d, ids.to(kind), acc, scale=0.75, accumulate=True)
            named = torch.bincount(ids[ids >= 0], minlength=V) > 0
            within(acc, ref + start.double(), bound + E24 * start.abs().double(), "accumulated")
            assert torch.equal(acc[~named], start[~named])


@pytest.mark.parametrize("ids", [[5] * 3000, [-1] * 100, list(range(40)) * 60, [39] * 129 + [0] * 255 + [1]])
def test_embed_grad_shared_and_absent_tokens(ops, ids):
    ids = torch.tensor(ids, device="cuda")
    g = gen(3)
    dy = randn(g, ids.numel(), 264, dtype=BF16)
    got = torch.full((40, 264), float("nan"), device="cuda")
    ops.cocodc_lm_embed_grad(dy, ids, got, scale=2.0)
    ref, bound = embed_grad_ref(dy, ids, 40, 2.0)
    within(got, ref, bound)


def test_embed_grad_without_tokens_and_with_bad_ids(B, ops):
    got = torch.full((6, 5), 3.0, device="cuda")
    empty = torch.empty(0, 5, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    ops.cocodc_lm_embed_grad(empty, none, got, accumulate=True)
    assert bool((got == 3).all())
    ops.cocodc_lm_embed_grad(empty, none, got)
    assert bool((got == 0).all())
    ops.cocodc_lm_embed_grad(torch.ones(4, 5, device="cuda"), torch.tensor([1, 6, 1, 2 ** 33 + 1], device="cuda"), got)
    assert got[:, 0].tolist() == [0, 2, 0, 0, 0, 0]
    assert ops.cocodc_lm_poll_status() == B.ERR_INVALID_ARG


def test_embed_grad_against_differences(ops):
    """f(W) = sum(c * embed(W)) is linear in W: the difference quotient along any direction is the gradient."""
    g = gen(8)
    V, D, T = 60, 48, 300
    w, c, way = randn(g, V, D), randn(g, T, D), randn(g, V, D)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    grad, y0, y1 = torch.empty(V, D, device="cuda"), torch.empty(T, D, device="cuda"), torch.empty(T, D, device="cuda")
    ops.cocodc_lm_embed_grad(c, ids, grad, scale=3.0)
    ops.cocodc_lm_embed(w + way, ids, y1, scale=3.0)
    ops.cocodc_lm_embed(w - way, ids, y0, scale=3.0)
    quotient = float(((y1.double() - y0.double()) * c.double()).sum() / 2)
    size = float(3 * (way.double().abs()[ids] * c.double().abs()).sum())
    # w + way, w - way and the products are each rounded, the gradient's rows are sums of up to T terms
    assert abs(quotient - float((grad.double() * way.double()).sum())) <= size * E24 * (T + 20)


# ------------------------------------------------------------------------------------------------------- gated block

def activation(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    a, b = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(a * (g + b * g ** 3))
    return g * (1 + t) / 2, (1 + t) / 2 + g * (1 - t * t) * a * (1 + 3 * b * g * g) / 2


GLU_SHAPES = [(1, 1, 1), (1, 64, 128), (1, 2048, 5632), (2, 40, 24), (3, 72, 200), (7, 1000, 264), (8, 256, 512), (9, 264, 136),
              (16, 128, 1000), (17, 520, 72), (31, 8, 8), (33, 320, 416), (63, 136, 1032), (65, 200, 64), (127, 72, 264), (128, 128, 128),
              (129, 192, 384), (200, 33, 65), (257, 1024, 136), (300, 264, 520), (1000, 512, 776)]


GLU_WIDE = [(2100, 2600, 1000), (4000, 1288, 1411), (1290, 77, 5003)]      # more tiles than SMs


@pytest.mark.parametrize("T,D,F", GLU_SHAPES + GLU_WIDE)
@pytest.mark.parametrize("dtype,act", [(BF16, "silu"), (F16, "gelu"), (BF16, "gelu"), (F16, "silu")])
def test_glu(ops, T, D, F, dtype, act):
    g = gen(T + D + F)
    x = randn(g, T, D, dtype=dtype)
    wg, wu = (randn(g, F, D, std=1.5 * D ** -0.5, dtype=dtype) for _ in range(2))
    gate, up = x.double() @ wg.double().T, x.double() @ wu.double().T
    eg, eu = (2 * D * E24 * (x.double().abs() @ w.double().abs().T) for w in (wg, wu))
    value, slope = activation(gate, act)
    h = value * up
    eh = 1.13 * eg * (up.abs() + eu) + (value.abs() + 1.13 * eg) * eu + 2.0 ** -18 * h.abs()
    up8 = lambda n: (n + 7) // 8 * 8  # noqa: E731
    # 16-byte rows, contiguous (odd widths start at odd places), everything odd
    for px, pf, off in ((up8(D) + 8, up8(F) + 16, 8), (D, F, 0), (D + 1, F + 3, 1)):
        xx, a, b = put(x, px, off), put(wg, px, off), put(wu, px, off)
        out = [placed(T, F, dtype, pf, off) for _ in range(3)]
        ops.cocodc_lm_glu(xx, a, b, out[0][0], act=act)
        within(out[0][0], h, eh, "h")
        first = out[0][0].clone()
        out[0][1].fill_(float("nan"))
        ops.cocodc_lm_glu(xx, a, b, *(o[0] for o in out), act=act)
        assert torch.equal(first, out[0][0])                # keeping gate and up changes nothing
        within(out[1][0], gate, eg, "gate")
        within(out[2][0], up, eu, "up")
        for o in out:
            untouched(o[0], o[1], float("nan"))


@pytest.mark.parametrize("T,D,F", GLU_SHAPES + GLU_WIDE)
@pytest.mark.parametrize("dtype,act", [(BF16, "silu"), (F16, "gelu"), (BF16, "gelu")])
def test_glu_grad(ops, T, D, F, dtype, act):
    g = gen(T + D + F + 1)
    x, dh, gate, up = randn(g, T, D, dtype=dtype), *(randn(g, T, F, dtype=dtype) for _ in range(3))
    wg, wu = (randn(g, F, D, std=F ** -0.5, dtype=dtype) for _ in range(2))
    value, slope = activation(gate.double(), act)
    dg, du = dh.double() * up.double() * slope, dh.double() * value
    u, tiny = UNIT[dtype] + 2.0 ** -17, TINY[dtype]
    # the slope can be near zero by cancellation: its own error is 2^-18 of its parts, whose sum is at most 1.13 + 1
    eg = u * dg.abs() + 2.0 ** -17 * (dh.double() * up.double()).abs() + tiny
    eu = u * du.abs() + tiny
    xa, ga, ua = x.double().abs(), dg.abs() + eg, du.abs() + eu
    dx = dg @ wg.double() + du @ wu.double()
    ex = eg @ wg.double().abs() + eu @ wu.double().abs() + 4 * F * E24 * (ga @ wg.double().abs() + ua @ wu.double().abs())
    dwg, dwu = dg.T @ x.double(), du.T @ x.double()
    ewg, ewu = eg.T @ xa + 2 * T * E24 * (ga.T @ xa), eu.T @ xa + 2 * T * E24 * (ua.T @ xa)
    up8 = lambda n: (n + 7) // 8 * 8  # noqa: E731
    for px, pf, off in ((up8(D) + 8, up8(F) + 16, 8), (D, F, 0), (D + 1, F + 3, 1)):
        ins = [put(t, pf, off) for t in (dh, gate, up)] + [put(t, px, off) for t in (x, wg, wu)]
        out = [placed(n, D, dtype, px, off) for n in (T, F, F)]
        ops.cocodc_lm_glu_grad(*ins, *(o[0] for o in out), act=act)
        within(out[0][0], dx, ex, "dx")
        within(out[1][0], dwg, ewg, "dwg")
        within(out[2][0], dwu, ewu, "dwu")
        for o in out:
            untouched(o[0], o[1], float("nan"))
        alone = torch.empty(T, D, dtype=dtype, device="cuda")
        ops.cocodc_lm_glu_grad(*ins, dx=alone, act=act)
        if alone.stride(0) % 8 == out[0][0].stride(0) % 8 and px % 8 == 0:
            assert torch.equal(alone, out[0][0])
        within(alone, dx, ex, "dx alone")
        pair = [torch.empty(F, D, dtype=dtype, device="cuda") for _ in range(2)]
        ops.cocodc_lm_glu_grad(*ins, dwg=pair[0], dwu=pair[1], act=act)
        within(pair[0], dwg, ewg, "dwg alone")
        within(pair[1], dwu, ewu, "dwu alone")


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_glu_large_gates(ops, act):
    """Gates far outside the activation's bend: exactly 0 or the gate itself, slopes exactly 0 or 1, no NaN."""
    vals = torch.tensor([-3e38, -1e20, -1e4, -200.0, 0.0, 200.0, 1e4, 1e20, 3e38], device="cuda", dtype=BF16)
    n = vals.numel()
    gate, one = vals.repeat(n, 1).contiguous(), torch.ones(n, n, device="cuda", dtype=BF16)
    eye = torch.eye(n, device="cuda", dtype=BF16)
    dx, dwg, dwu = (torch.empty(n, n, device="cuda", dtype=BF16) for _ in range(3))
    ops.cocodc_lm_glu_grad(one, gate, one, eye, eye, eye * 0, dx, dwg, dwu, act=act)
    slope = torch.where(vals > 0, 1.0, 0.0)
    slope[vals == 0] = 0.5
    assert torch.equal(dx, slope.to(BF16).repeat(n, 1)) and torch.equal(dwg, slope.to(BF16).repeat(n, 1).T)
    assert torch.equal(dwu, vals.clamp(min=0).repeat(n, 1).T)
    h = torch.empty(n, n, device="cuda", dtype=BF16)
    ops.cocodc_lm_glu(one, torch.diag(vals.double()).to(BF16) @ torch.eye(n, device="cuda", dtype=BF16), eye, h, act=act)
    assert torch.equal(h, vals.clamp(min=0).repeat(n, 1))


def test_glu_non_finite_inputs_stay_in_their_rows(ops):
    g = gen(5)
    x = randn(g, 40, 200, dtype=BF16)
    wg, wu = (randn(g, 150, 200, dtype=BF16) for _ in range(2))
    wg, wu = put(wg, 208, 0), put(wu, 208, 0)
    clean, got = (torch.empty(40, 152, device="cuda", dtype=BF16)[:, :150] for _ in range(2))
    ops.cocodc_lm_glu(put(x, 208), wg, wu, clean)
    x[7, 3], x[20, 199] = float("nan"), float("inf")
    ops.cocodc_lm_glu(put(x, 208), wg, wu, got)
    rest = [i for i in range(40) if i not in (7, 20)]
    assert torch.equal(clean[rest], got[rest])
    assert bool(torch.isnan(got[7]).all()) and not bool(torch.isfinite(got[20]).all())


def test_glu_grad_against_differences(ops):
    """<gradient, direction> against the central difference of sum(c * h) of the formula in 64 bits."""
    g = gen(6)
    T, D, F = 70, 96, 88
    x = randn(g, T, D, dtype=F16)
    wg, wu = (randn(g, F, D, std=D ** -0.5, dtype=F16) for _ in range(2))
    c = randn(g, T, F, dtype=F16)
    h, gate, up = (torch.empty(T, F, dtype=F16, device="cuda") for _ in range(3))
    ops.cocodc_lm_glu(x, wg, wu, h, gate, up)
    grads = [torch.empty_like(t) for t in (x, wg, wu)]
    ops.cocodc_lm_glu_grad(c, gate, up, x, wg, wu, *grads)

    def f(x, wg, wu):
        return float((activation(x @ wg.T, "silu")[0] * (x @ wu.T) * c.double()).sum())

    at = [t.double() for t in (x, wg, wu)]
    for i in range(3):
        way = torch.randn(at[i].shape, generator=g, device="cuda", dtype=torch.float64)
        plus, minus = list(at), list(at)
        eps = 1e-4
        plus[i], minus[i] = at[i] + eps * way, at[i] - eps * way
        quotient = (f(*plus) - f(*minus)) / (2 * eps)
        inner = float((grads[i].double() * way).sum())
        # gate, up, dg, du and the gradient are each rounded to 11 bits, independently over thousands of terms
        size = float(torch.linalg.vector_norm(grads[i].double()) * torch.linalg.vector_norm(way))
        assert abs(quotient - inner) <= 6 * UNIT[F16] * size


def test_glu_no_tokens(ops):
    e = torch.empty(0, 16, dtype=BF16, device="cuda")
    w = torch.ones(24, 16, dtype=BF16, device="cuda")
    eh = torch.empty(0, 24, dtype=BF16, device="cuda")
    ops.cocodc_lm_glu(e, w, w.clone(), eh, eh.clone(), eh.clone())
    dw = [torch.full((24, 16), 7.0, dtype=BF16, device="cuda") for _ in range(2)]
    ops.cocodc_lm_glu_grad(eh, eh, eh, e, w, w.clone(), torch.empty_like(e), *dw)
    assert all(bool((d == 0).all()) for d in dw)


# --------------------------------------------------------------------------------------------------- log probabilities

def logprobs_ref(x, targets, scale, k):
    """(logp, entropy, lse, top ids, top logp) in 64 bits with the documented values for masked and invalid rows."""
    z = x.double() * scale
    bad = (torch.isnan(z) | (z == math.inf)).any(1)
    empty = (z == -math.inf).all(1)
    nan = torch.full((), math.nan, dtype=torch.float64, device="cuda")
    lse = torch.where(bad, nan, torch.logsumexp(z, 1))
    lp = z - lse.unsqueeze(1)
    lp[empty] = -math.inf
    p = torch.exp(lp)
    H = torch.where(bad, nan, -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1))
    logp = torch.zeros_like(lse)
    there = (targets >= 0) & (targets < x.shape[1])
    logp[there] = lp[there, targets[there].long()]
    # descending, equal ones by position; NaN counts as larger than +Inf
    rank = torch.where(torch.isnan(x), torch.full((), 1e300, dtype=torch.float64, device="cuda"), x.double())
    rank = torch.where(x == math.inf, torch.full_like(rank, 1e200), rank)
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :k]
    return logp, H, lse, order, lp.gather(1, order)


def check_logprobs(ops, x, targets, scale=1.0, k=0, kind=torch.int64):
    T, V = x.shape
    out = {n: torch.full((T,), 77.0, device="cuda") for n in ("logp", "entropy", "lse")}
    if k:
        out["top_ids"] = torch.full((T, k), -5, dtype=torch.int32, device="cuda")
        out["top_logp"] = torch.full((T, k), 77.0, device="cuda")
    ops.cocodc_lm_logprobs(x, targets.to(kind), scale=scale, **out)
    logp, H, lse, order, top = logprobs_ref(x, targets, scale, max(k, 1))
    z = x.double() * scale
    top_z = torch.where(torch.isfinite(z), z, torch.zeros_like(z)).abs().amax(1)
    e = E24 * (3 * top_z + 300)
    within(out["lse"], lse, e, "lse")
    within(out["logp"], logp, e + E24 * torch.nan_to_num(logp, 0, 0, 0).abs(), "logp")
    within(out["entropy"], H, 2 * e * (41 + torch.nan_to_num(H)), "entropy")
    if k:
        assert torch.equal(out["top_ids"].long(), order)
        within(out["top_logp"], top, e.unsqueeze(1) + E24 * torch.nan_to_num(top, 0, 0, 0).abs(), "top")
    return out


@pytest.mark.parametrize("T,V", [(1, 1), (1, 2), (3, 7), (2, 8), (5, 9), (1, 31), (4, 255), (7, 256), (1, 257), (3, 1000), (2, 2047), (300, 2049),
                                 (1, 4096), (2, 16391), (33, 5003), (1, 50257), (9, 50257), (150, 32000), (301, 10000), (2, 262147), (1, 128256)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_logprobs(ops, T, V, dtype):
    g = gen(T + V)
    x = randn(g, T, V, std=3.0, dtype=dtype)
    targets = torch.randint(-1, V, (T,), generator=g, device="cuda")
    for k, scale, kind, pitch, off in ((0, 1.0, torch.int64, V, 0), (1, 0.6, torch.int32, V + 1, 1), (min(8, V), 1.3, torch.int64, V + 3, 3),
                                       (min(32, V), 1.0, torch.int32, V + 16 - V % 16, 8), (min(5, V), 2.0, torch.int64, V, 5)):
        check_logprobs(ops, put(x, pitch, off), targets, scale, k, kind)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("V", [5, 64, 1000, 4099, 50257])
@pytest.mark.parametrize("T", [1, 12, 400])
def test_logprobs_masks(ops, dtype, V, T):
    if T * V > 5_000_000:
        T = 60
    low = torch.finfo(dtype).min
    g = gen(V)
    base = randn(g, T, V, dtype=dtype)
    targets = torch.randint(0, V, (T,), generator=g, device="cuda")
    k = min(5, V)
    keep = torch.rand(T, V, generator=g, device="cuda") < 0.3
    for mask in (-math.inf, low):
        x = torch.where(keep, base, torch.full_like(base, mask))
        check_logprobs(ops, x, targets, 1.0, k)
        one = torch.full_like(base, mask)                     # a single candidate, at the end, the start, the middle
        for i, at in enumerate((V - 1, 0, V // 2)):
            one[i % T] = mask
            one[i % T, at] = 1.5
        check_logprobs(ops, one, targets, 1.0, k)
        check_logprobs(ops, torch.full_like(base, mask), targets, 1.0, k)     # nothing left
        few = torch.full_like(base, mask)                     # fewer candidates than alternatives asked for
        few[:, V // 3], few[:, V - 2] = 0.5, 0.25
        check_logprobs(ops, few, targets, 1.0, k)
    mixed = torch.where(keep, torch.full_like(base, low), torch.full_like(base, -math.inf))
    check_logprobs(ops, mixed, targets, 1.0, k)
    for v in (math.nan, math.inf):
        x = base.clone()
        x[T // 2, V - 1] = v
        check_logprobs(ops, x, targets, 1.0, k)
        x[0] = -math.inf
        x[0, V // 2] = v
        check_logprobs(ops, x, targets, 1.0, k)
    x = base.clone()
    x[0, 0], x[0, V - 1] = math.nan, math.inf
    check_logprobs(ops, x, targets, 1.0, k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [8, 300, 5003, 50257])
def test_logprobs_ties(ops, dtype, V):
    T = 6
    targets = torch.zeros(T, dtype=torch.int64, device="cuda")
    k = min(32, V)
    for x in (torch.zeros(T, V, device="cuda"), torch.arange(V, device="cuda").float().flip(0).div(V).repeat(T, 1),
              torch.arange(V, device="cuda").float().div(V).repeat(T, 1), torch.randint(0, 3, (T, V), generator=gen(V), device="cuda").float(),
              -(torch.arange(V, device="cuda") % 2).float().repeat(T, 1) * 0.0):
        check_logprobs(ops, x.to(dtype), targets, 1.0, k)


def test_logprobs_outputs_are_optional(B, ops):
    x = randn(gen(1), 4, 100)
    t = torch.tensor([1, -1, 99, 5], device="cuda")
    full = check_logprobs(ops, x, t, k=3)
    lse, H = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    ops.cocodc_lm_logprobs(x, None, None, lse=lse)
    ops.cocodc_lm_logprobs(x, None, None, entropy=H)
    assert torch.equal(lse, full["lse"]) and torch.equal(H, full["entropy"])
    ids, top = torch.empty(4, 3, dtype=torch.int32, device="cuda"), torch.empty(4, 3, device="cuda")
    ops.cocodc_lm_logprobs(x, None, None, top_ids=ids, top_logp=top)
    assert torch.equal(ids, full["top_ids"]) and torch.equal(top, full["top_logp"])
    logp = torch.empty(4, device="cuda")
    ops.cocodc_lm_logprobs(x, torch.tensor([1, 100, 99, 2 ** 35], device="cuda"), logp)
    assert logp[1] == 0 and logp[3] == 0 and torch.equal(logp[[0, 2]], full["logp"][[0, 2]])
    assert ops.cocodc_lm_poll_status() == B.ERR_INVALID_ARG


def logprobs_grad_ref(x, targets, scale, lse, H, dlogp, dent):
    T, V = x.shape
    lp = x.double() * scale - lse.double().unsqueeze(1)
    p = torch.exp(lp)
    there = (targets >= 0) & (targets < V)
    gr = torch.where(there, dlogp.double(), torch.zeros((), dtype=torch.float64, device="cuda")).unsqueeze(1) if dlogp is not None else torch.zeros(T, 1, device="cuda").double()
    hh = dent.double().unsqueeze(1) if dent is not None else torch.zeros(T, 1, device="cuda").double()
    HH = H.double().unsqueeze(1) if dent is not None else torch.zeros(T, 1, device="cuda").double()
    inner = torch.where(p > 0, lp + HH, torch.zeros_like(lp))
    d = -p * (gr + hh * inner)
    size = p * (gr.abs() + hh.abs() * (inner.abs() + HH.abs() + 1))
    for t in range(T):
        if dlogp is not None and there[t]:
            d[t, targets[t]] += gr[t, 0]
    d[torch.isnan(lse)] = math.nan
    d[lse == -math.inf], size[lse == -math.inf] = 0, 0
    return d * scale, size * scale


@pytest.mark.parametrize("T,V", [(1, 1), (3, 7), (2, 8), (5, 257), (4, 2048), (33, 2049), (2, 16391), (9, 50257), (150, 3201)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_logprobs_grad(ops, T, V, dtype):
    g = gen(T + V)
    x = randn(g, T, V, std=3.0, dtype=dtype)
    x[:, V // 2:][torch.rand(T, V - V // 2, generator=g, device="cuda") < 0.1] = -math.inf
    if T > 2:
        x[1] = -math.inf
        x[2, V - 1] = math.nan
    targets = torch.randint(-1, V, (T,), generator=g, device="cuda")
    dlogp, dent = randn(g, T), randn(g, T)
    for scale, pitch, off, dpitch, doff, use in ((1.0, V, 0, V, 0, 3), (0.7, V + 3, 1, V + 3, 1, 3), (1.3, V + 1, 0, V + 2, 1, 1), (1.0, V + 8 - V % 8, 8, V + 8 - V % 8, 0, 2),
                                                (2.0, V, 3, V, 3, 3)):
        xx = put(x, pitch, off)
        lse, H = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        ops.cocodc_lm_logprobs(xx, None, None, entropy=H, lse=lse, scale=scale)
        got, buf = placed(T, V, dtype, dpitch, doff, fill=55.0)
        a, b = (dlogp if use & 1 else None), (dent if use & 2 else None)
        ops.cocodc_lm_logprobs_grad(xx, targets if use & 1 else None, lse, H if use & 2 else None, a, b, got, scale=scale)
        want, size = logprobs_grad_ref(x, targets, scale, lse, H, a, b)
        z = torch.where(torch.isfinite(x), x.double() * scale, torch.zeros((), dtype=torch.float64, device="cuda")).abs().amax(1, keepdim=True)
        bound = 2 * E24 * (3 * z + 300) * size + 2 * E24 * (dlogp.abs().double().unsqueeze(1) * scale)
        within(got, want, bound, "gradient")
        untouched(got, buf, 55.0)
        if dpitch == pitch and doff == off:
            ops.cocodc_lm_logprobs_grad(xx, targets if use & 1 else None, lse, H if use & 2 else None, a, b, xx, scale=scale)
            assert torch.equal(xx.nan_to_num(9.0), got.nan_to_num(9.0))       # in place: the same bits


def test_logprobs_grad_against_differences(ops):
    """Central differences of sum(a * logp + b * entropy) as the forward kernel computes it, on fp32 logits."""
    g = gen(4)
    T, V = 6, 301
    x, way = randn(g, T, V), randn(g, T, V)
    targets = torch.randint(0, V, (T,), generator=g, device="cuda")
    a, b = randn(g, T), randn(g, T)

    def f(y):
        logp, H, lse = (torch.empty(T, device="cuda") for _ in range(3))
        ops.cocodc_lm_logprobs(y, targets, logp, entropy=H, lse=lse, scale=0.8)
        return (logp.double() * a.double() + b.double() * H.double()).sum().item(), lse, H

    _, lse, H = f(x)
    d = torch.empty_like(x)
    ops.cocodc_lm_logprobs_grad(x, targets, lse, H, a, b, d, scale=0.8)
    eps = 2.0 ** -6
    quotient = (f(x + eps * way)[0] - f(x - eps * way)[0]) / (2 * eps)
    inner = float((d.double() * way.double()).sum())
    # values of up to about 10 a row, 1e-6 off each: 2 T 1e-5 / (2 eps); third derivatives of order one: T eps^2
    assert abs(quotient - inner) <= T * (1e-5 / eps + 10 * eps * eps)


# ----------------------------------------------------------------------------------------- streams, graphs, large offsets

def test_other_stream_and_graph_replay(ops):
    g = gen(2)
    V, D, F, T = 500, 64, 128, 40
    w, x0 = randn(g, V, D), torch.empty(T, D, dtype=BF16, device="cuda")
    wg, wu = (randn(g, F, D, dtype=BF16) for _ in range(2))
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    h, gate, up, dx = (torch.empty(T, n, dtype=BF16, device="cuda") for n in (F, F, F, D))
    dwg, dwu, dw = torch.empty_like(wg), torch.empty_like(wu), torch.empty_like(w)
    logp, lse, H = (torch.empty(T, device="cuda") for _ in range(3))
    ti, tl = torch.empty(T, 4, dtype=torch.int32, device="cuda"), torch.empty(T, 4, device="cuda")
    one = torch.ones(T, device="cuda")

    def step():
        ops.cocodc_lm_embed(w, ids, x0, scale=2.0)
        ops.cocodc_lm_glu(x0, wg, wu, h, gate, up)
        ops.cocodc_lm_logprobs(h, ids % F, logp, entropy=H, lse=lse, top_ids=ti, top_logp=tl)
        ops.cocodc_lm_logprobs_grad(h, ids % F, lse, H, one, one, h)
        ops.cocodc_lm_glu_grad(h, gate, up, x0, wg, wu, dx, dwg, dwu)
        ops.cocodc_lm_embed_grad(dx, ids, dw, scale=2.0)
        return [t.clone() for t in (logp, H, ti, tl, dwg, dwu, dw)]

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = step()
    for t in (x0, h, dw, dwg):
        t.zero_()
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, inside))


def test_offsets_beyond_32_bits(ops):
    """Row strides of more than 2^31 elements."""
    pitch = 2 ** 31 + 16
    buf = torch.empty(2 * pitch + 4096, dtype=BF16, device="cuda")
    far = buf.as_strided((2, 1024), (pitch, 1))
    g = gen(9)
    x = randn(g, 2, 1024, dtype=BF16)
    far.copy_(x)
    y = torch.empty(3, 1024, device="cuda")
    ids = torch.tensor([1, 0, 1], device="cuda")
    ops.cocodc_lm_embed(far, ids, y)
    assert torch.equal(y, x.float()[ids])
    check_logprobs(ops, far, torch.tensor([5, 1023], device="cuda"), 1.0, 4)
    w = randn(g, 256, 1024, std=0.03, dtype=BF16)
    near, h = torch.empty(2, 256, dtype=BF16, device="cuda"), torch.empty(2, 256, dtype=BF16, device="cuda")
    ops.cocodc_lm_glu(x, w, w.clone(), near)
    ops.cocodc_lm_glu(far, w, w.clone(), h)
    assert torch.equal(near, h)
    far.zero_()
    ops.cocodc_lm_embed_grad(y.to(BF16), ids, far)
    ref, bound = embed_grad_ref(y.to(BF16), ids, 2, 1.0)
    within(far, ref, bound)
    lse, H = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    ops.cocodc_lm_logprobs(x, None, None, entropy=H, lse=lse)
    d, one = torch.empty_like(x), torch.ones(2, device="cuda")
    ops.cocodc_lm_logprobs_grad(x, None, lse, H, None, one, d)
    ops.cocodc_lm_logprobs_grad(x, None, lse, H, None, one, far)
    assert torch.equal(d, far)


def test_no_rows_of_something(ops):
    """T = 0 as a slice of a longer buffer (its address is not NULL) and as an empty tensor (its address is)."""
    before = ops.launch_count
    for cut in (lambda t: t[:0], lambda t: torch.empty(0, *t.shape[1:], dtype=t.dtype, device="cuda")):
        x, h, w = cut(torch.ones(4, 16, dtype=BF16, device="cuda")), cut(torch.ones(4, 24, dtype=BF16, device="cuda")), torch.ones(24, 16, dtype=BF16, device="cuda")
        ids, f = cut(torch.zeros(4, dtype=torch.int64, device="cuda")), cut(torch.zeros(4, device="cuda"))
        ti, tl = cut(torch.zeros(4, 3, dtype=torch.int32, device="cuda")), cut(torch.zeros(4, 3, device="cuda"))
        empty = torch.empty(0, device="cuda")
        ops.cocodc_lm_embed(w, ids, x)
        ops.cocodc_lm_glu(x, w, w, h, gate=h, up=torch.empty(0, 24, dtype=BF16, device="cuda"))
        ops.cocodc_lm_logprobs(x, ids, empty, entropy=f, lse=empty, top_ids=ti, top_logp=tl)
        ops.cocodc_lm_logprobs_grad(x, ids, f, empty, f, empty, x)
        ops.cocodc_lm_glu_grad(h, h, h, x, w, w, dx=torch.empty(0, 16, dtype=BF16, device="cuda"))
    assert ops.launch_count == before


def test_long_masked_stretches_over_several_blocks(ops):
    """Few rows are split over blocks; whole parts masked, a part with the only NaN, alternatives from one part alone."""
    V = 40000
    g = gen(12)
    base = randn(g, 4, V, dtype=BF16)
    targets = torch.tensor([5, V - 1, V // 2, 0], device="cuda")
    for lo, hi in ((0, V - 3000), (3000, V), (1000, V - 1000)):
        x = base.clone()
        x[:, lo:hi] = -math.inf
        check_logprobs(ops, x, targets, 1.0, 20)
        x[2, hi - 1 if hi == V else lo] = math.nan
        check_logprobs(ops, x, targets, 1.0, 20)


# ------------------------------------------------------------------------------------------------------------- refusals

def test_refusals(B, ops):
    x, w = torch.ones(4, 16, dtype=BF16, device="cuda"), torch.ones(24, 16, dtype=BF16, device="cuda")
    h = torch.empty(4, 24, dtype=BF16, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    f = torch.empty(4, device="cuda")

    def refused(code, call, *a, **kw):
        with pytest.raises(B.CocodcError) as e:
            call(*a, **kw)
        assert e.value.code == code

    inv, alias, align = B.ERR_INVALID_ARG, B.ERR_ALIAS, B.ERR_ALIGNMENT
    before = ops.launch_count
    refused(alias, ops.cocodc_lm_embed, w, ids, w[:4])
    refused(alias, ops.cocodc_lm_embed_grad, x, ids, x)
    refused(inv, ops.cocodc_lm_embed_grad, x, ids, w, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    refused(align, ops.cocodc_lm_embed_grad, x, ids, w, workspace=torch.empty(100000, dtype=torch.uint8, device="cuda")[1:])
    refused(inv, ops.cocodc_lm_glu, x, w, w, h, gate=torch.empty_like(h))            # gate without up
    refused(alias, ops.cocodc_lm_glu, x, w, w, h, gate=h, up=torch.empty_like(h))
    refused(inv, ops.cocodc_lm_glu, x.float(), w.float(), w.float(), h.float())      # fp32 is not a type of the block
    refused(inv, ops.cocodc_lm_glu_grad, h, h, h, x, w, w)                           # no output asked for
    refused(inv, ops.cocodc_lm_glu_grad, h, h, h, x, w, w, dwg=torch.empty_like(w))  # dwg without dwu
    refused(alias, ops.cocodc_lm_glu_grad, h, h, h, x, w, w, dx=x)
    refused(inv, ops.cocodc_lm_logprobs, x, None, None)                              # no output asked for
    refused(inv, ops.cocodc_lm_logprobs, x, ids, None, lse=f)                        # targets without logp
    refused(inv, ops.cocodc_lm_logprobs, x, None, f)                                 # logp without targets
    refused(inv, ops.cocodc_lm_logprobs, x, ids, f, scale=0.0)
    refused(inv, ops.cocodc_lm_logprobs, x, ids, f, scale=float("nan"))
    refused(inv, ops.cocodc_lm_logprobs, x, ids, f, scale=float("inf"))
    refused(inv, ops.cocodc_lm_logprobs, x, ids, f, scale=1e31)
    refused(inv, ops.cocodc_lm_logprobs, x, None, None, lse=f, top_ids=torch.empty(4, 2, dtype=torch.int32, device="cuda"))   # no top_logp
    refused(alias, ops.cocodc_lm_logprobs, x, ids, f, lse=f)
    for k in (17, 33):                                                               # more than V, more than the limit
        refused(inv, ops.cocodc_lm_logprobs, x if k == 17 else w.view(4, 96), None, None,
                top_ids=torch.empty(4, k, dtype=torch.int32, device="cuda"), top_logp=torch.empty(4, k, device="cuda"))
    refused(inv, ops.cocodc_lm_logprobs_grad, x, None, f, f, None, None, torch.empty_like(x))
    refused(inv, ops.cocodc_lm_logprobs_grad, x, None, f, None, None, f, torch.empty_like(x))      # entropy missing
    wide = torch.empty(4, 32, dtype=BF16, device="cuda")
    refused(alias, ops.cocodc_lm_logprobs_grad, wide[:, :16], ids, f, None, f.clone(), None, wide[:, 8:24])
    assert ops.launch_count == before
    for call in (lambda: ops.cocodc_lm_embed(w, ids, torch.empty(4, 15, dtype=BF16, device="cuda")),
                 lambda: ops.cocodc_lm_embed(w, ids.float(), x), lambda: ops.cocodc_lm_embed(w.cpu(), ids, x),
                 lambda: ops.cocodc_lm_embed(w.to(torch.float64), ids, x), lambda: ops.cocodc_lm_embed(w.t(), ids, torch.empty(4, 24, device="cuda")),
                 lambda: ops.cocodc_lm_glu(x, w, w.half(), h), lambda: ops.cocodc_lm_logprobs(x, ids[:3], f)):
        with pytest.raises(ValueError):
            call()
    lib = B.library()
    p = x.data_ptr()
    assert lib.cocodc_lm_embed(ops._h, p + 1, 1, 16, 4, 16, ids.data_ptr(), 1, 4, 1.0, h.data_ptr(), 1, 16, None) == align
    assert lib.cocodc_lm_embed(ops._h, p, 7, 16, 4, 16, ids.data_ptr(), 1, 4, 1.0, h.data_ptr(), 1, 16, None) == inv
    assert lib.cocodc_lm_embed(ops._h, p, 1, 15, 4, 16, ids.data_ptr(), 1, 4, 1.0, h.data_ptr(), 1, 16, None) == inv
    assert lib.cocodc_lm_embed(ops._h, p, 1, 16, 4, 16, ids.data_ptr(), 1, -1, 1.0, h.data_ptr(), 1, 16, None) == inv
    assert lib.cocodc_lm_logprobs(ops._h, p + 1, 1, 16, 4, 16, None, 0, 1.0, None, None, f.data_ptr(), 0, None, None, None) == align
    assert ops.launch_count == before


def test_handle(B):
    o = B.LmOps(0)
    assert o.launch_count == 0 and o.cocodc_lm_poll_status() == B.OK
    y = torch.empty(1, 4, device="cuda")
    o.cocodc_lm_embed(torch.ones(2, 4, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), y)
    assert o.launch_count == 1
    o.close()
    o.close()
    with pytest.raises(B.CocodcError) as e:
        B.LmOps(torch.cuda.device_count())
    assert e.value.code == B.ERR_INVALID_ARG
