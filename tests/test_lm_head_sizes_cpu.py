"""Sizes that the output head refuses before it looks for a device, as the header lists them.  No kernel is launched, no address followed."""

import pytest
from test_lm_step_cpu import B, handle, head, head_grad, lib  # noqa: F401


@pytest.mark.parametrize("T,D,V", [(2 ** 31 - 1, 64, 2 ** 30), (2 ** 24, 8, 2 ** 24)])
def test_forward(B, lib, handle, T, D, V):  # noqa: F811
    size = lib.cocodc_lm_head_workspace(T, D, V)
    assert size > 2 ** 41
    assert head(lib, handle, T=T, D=D, V=V, xs=D, ts=D, size=size) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("T,D,V", [(128, 2 ** 30, 64), (2 ** 30, 128, 64), (1, 2 ** 30, 2 ** 16)])
def test_gradient(B, lib, handle, T, D, V):  # noqa: F811
    assert head_grad(lib, handle, T=T, D=D, V=V, xs=D, ts=D, dxs=D, dts=D, size=lib.cocodc_lm_head_grad_workspace(T, D, V)) == B.ERR_INVALID_ARG
