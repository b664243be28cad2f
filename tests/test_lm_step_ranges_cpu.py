"""Ranges that the header promises for the optimizer's arguments.  No kernel is launched: a plan without units has nothing to step."""

import ctypes

import pytest
from test_lm_step_cpu import B, create, handle, lib, tensor  # noqa: F401


@pytest.fixture()
def empty():
    """Stands for a plan of no units on the handle's device."""
    buffer = ctypes.create_string_buffer(256)
    yield ctypes.addressof(buffer)


def adamw(lib, handle, plan, **k):  # noqa: F811
    d = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=1, step_at=None, grad_scale=None, lr_scale=None, seed=0)
    d.update(k)
    return lib.cocodc_lm_adamw(handle, plan, *d.values(), None)


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -126, 1e-30, 1e-8, 1.0, 1.5, 1e4, 2.0 ** 125])
def test_eps(B, lib, handle, empty, eps):  # noqa: F811
    assert adamw(lib, handle, empty, eps=eps) == B.OK


@pytest.mark.parametrize("bad", [dict(eps=-1e-8), dict(eps=1e-50), dict(eps=1e-40), dict(eps=2.0 ** -127), dict(eps=2.0 ** 126), dict(eps=float("inf")), dict(eps=float("nan")),
                                 dict(beta1=1.0), dict(beta2=-0.1), dict(lr=float("inf")), dict(step=0)])
def test_refusals(B, lib, handle, empty, bad):  # noqa: F811
    assert adamw(lib, handle, empty, **bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("decay", [0.0, 0.1, 1e30, 2e30, 3.4e38])
def test_any_finite_decay(B, lib, handle, decay):  # noqa: F811
    plan = ctypes.c_void_p()
    code = lib.cocodc_lm_adam_create(ctypes.byref(plan), handle, (B._Tensor * 1)(tensor(B, decay=decay)), 1, 32)
    assert code == (B.OK if plan else B.ERR_CUDA)                # past the checks: without a GPU the device is what fails
    lib.cocodc_lm_adam_destroy(plan)
