"""Host-only checks of the norm's, the output head's and the optimizer's entry points: no kernel is launched, no GPU is needed."""

import ctypes

import pytest

F32, BF16, F16, E4M3 = 0, 1, 2, 3
BIG = 2 ** 41


@pytest.fixture(scope="module")
def B():
    from paper_2504_17672_b200 import build
    build.build()
    from paper_2504_17672_b200 import binding
    return binding


@pytest.fixture(scope="module")
def lib(B):
    return B.library()


@pytest.fixture()
def handle():
    """Stands for a handle: calls that refuse their arguments do so before they look into it."""
    buffer = ctypes.create_string_buffer(256)
    yield ctypes.addressof(buffer)


A = [0x10000000 * (i + 1) for i in range(12)]     # addresses far apart, never followed


def norm(lib, h, **k):
    d = dict(x=A[0], x_type=BF16, xs=64, r=A[1], rs=64, sum_type=BF16, w=A[2], w_type=BF16, T=4, D=64, eps=1e-5, total=A[3], ts=64, y=A[4],
             y_type=BF16, ys=64, scale=None, group=0, rstd=A[6])
    d.update(k)
    return lib.cocodc_lm_norm(h, d["x"], d["x_type"], d["xs"], d["r"], d["rs"], d["sum_type"], d["w"], d["w_type"], d["T"], d["D"], d["eps"], d["total"],
                              d["ts"], d["y"], d["y_type"], d["ys"], d["scale"], d["group"], d["rstd"], None)


def norm_grad(lib, h, **k):
    d = dict(dy=A[0], y_type=BF16, ys=64, total=A[1], t_type=F32, ts=64, w=A[2], w_type=F32, rstd=A[3], T=4, D=64, dt=A[4], dts=64, dx=A[5], dxs=64,
             dw=A[6], dw_type=F32, acc=0, ws=A[7], size=1 << 20)
    d.update(k)
    return lib.cocodc_lm_norm_grad(h, *d.values(), None)


def head(lib, h, **k):
    d = dict(type=BF16, x=A[0], xs=64, table=A[1], ts=64, T=4, D=64, V=100, targets=A[2], it=1, scale=1.0, logp=A[3], lse=A[4], ws=A[5], size=1 << 20)
    d.update(k)
    return lib.cocodc_lm_head(h, *d.values(), None)


def head_grad(lib, h, **k):
    d = dict(type=BF16, x=A[0], xs=64, table=A[1], ts=64, T=4, D=64, V=100, targets=A[2], it=1, scale=1.0, lse=A[3], dlogp=A[4], dlse=A[5], dx=A[6],
             dxs=64, dtable=A[7], dt_type=BF16, dts=64, acc=0, ws=A[8], size=1 << 20)
    d.update(k)
    return lib.cocodc_lm_head_grad(h, *d.values(), None)


def test_null_handles_are_rejected(B, lib):
    for call in (norm, norm_grad, head, head_grad):
        assert call(lib, None) == B.ERR_INVALID_ARG
    plan = ctypes.c_void_p(1)
    assert lib.cocodc_lm_adam_create(ctypes.byref(plan), None, None, 0, 32) == B.ERR_INVALID_ARG and not plan
    assert lib.cocodc_lm_adam_create(None, None, None, 0, 32) == B.ERR_INVALID_ARG
    assert lib.cocodc_lm_adam_destroy(None) == B.OK
    assert lib.cocodc_lm_adamw(None, None, 1e-3, 0.9, 0.95, 1e-8, 1, None, None, None, 0, None) == B.ERR_INVALID_ARG


def test_records_hold_what_the_calls_take(B, lib):
    for name in ("norm", "norm_grad", "head", "head_grad", "adamw"):
        types = getattr(lib, "cocodc_lm_" + name).argtypes[1:]
        args = [0.5 if t in (ctypes.c_float, ctypes.c_double) else 7 for t in types]
        pack = getattr(B, "_" + name.upper())
        assert len(pack(0, *args)) == 8 * (1 + len(types)), name
        with pytest.raises(Exception):
            pack(0, *args, 7)


@pytest.mark.parametrize("bad", [
    dict(x_type=3), dict(w_type=3), dict(y_type=4), dict(T=-1), dict(T=BIG), dict(D=0), dict(D=2 ** 31), dict(xs=63), dict(ys=63), dict(rs=63), dict(ts=63),
    dict(xs=BIG), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(sum_type=F16), dict(sum_type=E4M3), dict(x=None), dict(w=None),
    dict(y=None), dict(r=None), dict(total=None), dict(scale=A[8]), dict(y_type=E4M3), dict(group=128), dict(y_type=E4M3, scale=A[8], group=64)])
def test_norm_refuses(B, lib, handle, bad):
    assert norm(lib, handle, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad,code", [
    (dict(x=A[0] + 1), "ALIGNMENT"), (dict(r=A[1] + 1), "ALIGNMENT"), (dict(rstd=A[6] + 2), "ALIGNMENT"), (dict(w=A[2] + 1), "ALIGNMENT"),
    (dict(y=A[0]), "ALIAS"), (dict(total=A[0]), "ALIAS"), (dict(total=A[1], ts=72), "ALIAS"), (dict(y=A[3] + 128), "ALIAS"), (dict(rstd=A[2]), "ALIAS"),
    (dict(y_type=E4M3, scale=A[6]), "ALIAS"), (dict(y=A[1]), "ALIAS")])
def test_norm_refuses_overlaps_and_odd_addresses(B, lib, handle, bad, code):
    assert norm(lib, handle, **bad) == getattr(B, "ERR_" + code)


@pytest.mark.parametrize("bad", [
    dict(y_type=3), dict(t_type=F16), dict(w_type=3), dict(dw_type=3), dict(T=-1), dict(D=0), dict(ys=63), dict(ts=1), dict(dts=63), dict(dxs=63), dict(dy=None),
    dict(total=None), dict(w=None), dict(rstd=None), dict(dx=None, dw=None), dict(ws=None), dict(size=16)])
def test_norm_grad_refuses(B, lib, handle, bad):
    assert norm_grad(lib, handle, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad,code", [
    (dict(ws=A[7] + 8), "ALIGNMENT"), (dict(dw=A[6] + 2), "ALIGNMENT"), (dict(total=A[1] + 2), "ALIGNMENT"), (dict(dx=A[1]), "ALIAS"), (dict(dx=A[4], dxs=72), "ALIAS"),
    (dict(dw=A[2]), "ALIAS"), (dict(dw=A[5]), "ALIAS"), (dict(ws=A[0]), "ALIAS")])
def test_norm_grad_refuses_overlaps_and_odd_addresses(B, lib, handle, bad, code):
    assert norm_grad(lib, handle, **bad) == getattr(B, "ERR_" + code)


@pytest.mark.parametrize("call", [head, head_grad])
@pytest.mark.parametrize("bad", [
    dict(type=F32), dict(type=E4M3), dict(T=-1), dict(T=2 ** 31), dict(D=0), dict(V=0), dict(V=2 ** 30 + 1), dict(xs=63), dict(ts=63), dict(xs=BIG), dict(it=2),
    dict(scale=0.0), dict(scale=-1.0), dict(scale=2e30), dict(scale=float("nan")), dict(x=None), dict(table=None), dict(targets=None), dict(ws=None), dict(size=16)])
def test_head_refuses(B, lib, handle, call, bad):
    assert call(lib, handle, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("call,bad,code", [
    (head, dict(logp=None), "INVALID_ARG"), (head, dict(logp=None, targets=None, lse=None), "INVALID_ARG"), (head, dict(x=A[0] + 1), "ALIGNMENT"),
    (head, dict(targets=A[2] + 4), "ALIGNMENT"), (head, dict(ws=A[5] + 4), "ALIGNMENT"), (head, dict(lse=A[3] + 4), "ALIAS"), (head, dict(logp=A[0]), "ALIAS"),
    (head, dict(ws=A[1] - 1024), "ALIAS"),
    (head_grad, dict(lse=None), "INVALID_ARG"), (head_grad, dict(dlogp=None), "INVALID_ARG"), (head_grad, dict(dlogp=None, targets=None, dlse=None), "INVALID_ARG"),
    (head_grad, dict(dx=None, dtable=None), "INVALID_ARG"), (head_grad, dict(dt_type=F16), "INVALID_ARG"), (head_grad, dict(dxs=63), "INVALID_ARG"),
    (head_grad, dict(dts=63), "INVALID_ARG"), (head_grad, dict(dx=A[0]), "ALIAS"), (head_grad, dict(dtable=A[1]), "ALIAS"), (head_grad, dict(dtable=A[6]), "ALIAS"),
    (head_grad, dict(ws=A[6] - 64 * 1024), "ALIAS"), (head_grad, dict(dlse=A[7], dt_type=F32), "ALIAS"), (head_grad, dict(dtable=A[7] + 2, dt_type=F32), "ALIGNMENT")])
def test_head_refuses_also(B, lib, handle, call, bad, code):
    assert call(lib, handle, **bad) == getattr(B, "ERR_" + code)


def test_nothing_to_do_is_no_error(B, lib, handle):
    assert norm(lib, handle, T=0, x=None, r=None, total=None, y=None, rstd=None) == B.OK
    assert norm_grad(lib, handle, T=0, dw=None) == B.OK
    assert head(lib, handle, T=0, x=None, targets=None, logp=None) == B.OK
    assert head_grad(lib, handle, T=0, dtable=None, dx=None, ws=None) == B.OK


def tensor(B, n=1000, at=0, state=4, **k):
    d = dict(p=A[at], grad=A[at + 1], m=A[at + 2], v=A[at + 3], m_scale=None, v_scale=None, copy=None, n=n, grad_type=F32, copy_type=BF16, decay=0.1, reserved=0)
    d.update(k)
    return B._Tensor(*d.values())


def create(B, lib, handle, tensors, bits=32):
    plan = ctypes.c_void_p()
    code = lib.cocodc_lm_adam_create(ctypes.byref(plan), handle, (B._Tensor * max(1, len(tensors)))(*tensors), len(tensors), bits)
    assert not plan
    return code


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(n=2 ** 39), dict(grad_type=3), dict(copy=A[6], copy_type=F32), dict(decay=-0.1), dict(decay=float("nan")), dict(decay=float("inf")),
    dict(reserved=1), dict(p=None), dict(grad=None), dict(m=None), dict(v=None), dict(m_scale=A[6])])
def test_plan_refuses(B, lib, handle, bad):
    assert create(B, lib, handle, [tensor(B, **bad)]) == B.ERR_INVALID_ARG


def test_plan_refuses_also(B, lib, handle):
    assert create(B, lib, handle, [tensor(B)], bits=16) == B.ERR_INVALID_ARG
    assert create(B, lib, handle, [tensor(B)], bits=8) == B.ERR_INVALID_ARG                       # no scales
    plan = ctypes.c_void_p()
    assert lib.cocodc_lm_adam_create(ctypes.byref(plan), handle, None, 1, 32) == B.ERR_INVALID_ARG
    assert lib.cocodc_lm_adam_create(ctypes.byref(plan), handle, None, -1, 32) == B.ERR_INVALID_ARG
    for odd in (dict(p=A[0] + 2), dict(grad=A[1] + 2), dict(m=A[2] + 2), dict(v=A[3] + 1), dict(copy=A[6] + 1)):
        assert create(B, lib, handle, [tensor(B, **odd)]) == B.ERR_ALIGNMENT
    two = lambda **k: [tensor(B), tensor(B, at=4, **k)]  # noqa: E731
    for same in (dict(p=A[0] + 3996), dict(m=A[0]), dict(v=A[2] + 400), dict(copy=A[3]), dict(grad=A[0]), dict(p=A[1] + 4), dict(copy=A[1])):
        assert create(B, lib, handle, two(**same)) == B.ERR_ALIAS, same
    s = dict(m_scale=A[8], v_scale=A[9])
    assert create(B, lib, handle, [tensor(B, **s), tensor(B, at=4, m_scale=A[8] + 12, v_scale=A[10])], bits=8) == B.ERR_ALIAS


@pytest.mark.parametrize("sizes", [(0, 1, 1), (0, 64, 100), (1, 1, 1), (1, 2048, 32000), (8192, 2048, 32000), (2 ** 31 - 1, 1, 2 ** 30), (77, 2 ** 31 - 1, 2 ** 17), (2 ** 31 - 1, 2 ** 17, 2 ** 30)])
def test_workspace_sizes(lib, sizes):
    T, D, V = sizes
    assert lib.cocodc_lm_head_workspace(T, D, V) >= 4 * T + 8 * T * ((V + 255) // 256)
    # dz of 1024 columns, or of all of them, in exact integers
    assert lib.cocodc_lm_head_grad_workspace(T, D, V) >= 2 * T * min(V, 1024) + (4 * T * D if 2 * T * V > 2 ** 28 and V > 1024 else 0)


def test_workspace_is_zero_for_sizes_that_the_calls_refuse(lib):
    for T, D, V in ((-1, 8, 8), (2 ** 31, 8, 8), (8, 0, 8), (8, 2 ** 31, 8), (8, 8, 0), (8, 8, 2 ** 30 + 1), (2 ** 31 - 1, 2 ** 18, 8), (8, 2 ** 19, 2 ** 30)):
        assert lib.cocodc_lm_head_workspace(T, D, V) == 0 and lib.cocodc_lm_head_grad_workspace(T, D, V) == 0
    for T, D in ((-1, 8), (BIG, 8), (8, 0), (8, 2 ** 31)):
        assert lib.cocodc_lm_norm_grad_workspace(T, D) == 0
    assert lib.cocodc_lm_norm_grad_workspace(2 ** 40, 2 ** 31 - 1) >= 4 * (2 ** 31 - 1)
    assert lib.cocodc_lm_head_grad_workspace(2 ** 20, 64, 2 ** 17) < 2 ** 20 * (64 * 4 + 2 * 1024) + 2 ** 20       # not the logits
