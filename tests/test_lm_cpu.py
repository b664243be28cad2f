"""Host-only checks of the local step's entry points: no kernel is launched, no GPU is needed."""

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2504_17672_b200 import build
    build.build()
    from paper_2504_17672_b200 import binding
    return binding


def test_null_handle_is_rejected(B):
    lib = B.library()
    assert lib.cocodc_lm_create(None, 0) == B.ERR_INVALID_ARG
    assert lib.cocodc_lm_destroy(None) == B.OK
    assert lib.cocodc_lm_poll_status(None, None) == B.ERR_INVALID_ARG
    assert lib.cocodc_lm_launch_count(None) == 0
    assert lib.cocodc_lm_embed(None, None, 0, 1, 1, 1, None, 0, 1, 1.0, None, 0, 1, None) == B.ERR_INVALID_ARG
    assert lib.cocodc_lm_embed_grad(None, None, 0, 1, None, 0, 1, 1, 1, 1.0, 0, None, 0, 1, None, 0, None) == B.ERR_INVALID_ARG
    assert lib.cocodc_lm_glu(None, 0, 1, None, 1, None, None, 1, 1, 1, 1, None, 1, None, None, 1, None) == B.ERR_INVALID_ARG
    assert lib.cocodc_lm_glu_grad(None, 0, 1, None, 1, None, None, 1, None, 1, None, None, 1, 1, 1, 1, None, 1, None, None, 1,
                                  None, 0, None) == B.ERR_INVALID_ARG
    assert lib.cocodc_lm_logprobs(None, None, 0, 1, 1, 1, None, 0, 1.0, None, None, None, 0, None, None, None) == B.ERR_INVALID_ARG
    assert lib.cocodc_lm_logprobs_grad(None, None, 0, 1, 1, 1, None, 0, 1.0, None, None, None, None, None, 1, None) == B.ERR_INVALID_ARG


def test_records_hold_what_the_calls_take(B):
    """A record is the operator's number and the call's arguments without the handle; scale is its only floating word."""
    import ctypes
    lib = B.library()
    for name in ("embed", "embed_grad", "glu", "glu_grad", "logprobs", "logprobs_grad"):
        types = getattr(lib, "cocodc_lm_" + name).argtypes[1:]
        pack = getattr(B, "_" + name.upper())
        args = [0.5 if t is ctypes.c_float else 7 for t in types]
        assert len(pack(0, *args)) == 8 * (1 + len(types)), name
        with pytest.raises(Exception):
            pack(0, *args, 7)
    assert lib.cocodc_lm_submit(None, b"\0" * 256) == B.ERR_INVALID_ARG
    handle = ctypes.create_string_buffer(256)
    assert lib.cocodc_lm_submit(ctypes.addressof(handle), None) == B.ERR_INVALID_ARG
    assert lib.cocodc_lm_submit(ctypes.addressof(handle), b"\x63" + b"\0" * 255) == B.ERR_INVALID_ARG


def test_workspace_sizes(B):
    lib = B.library()
    for V, D, T in ((1, 1, 0), (50257, 768, 4099), (32000, 1024, 65536)):
        assert lib.cocodc_lm_embed_grad_workspace(V, D, T) >= 4 * (V + 1) + 8 * T
    for T, D, F in ((0, 1, 1), (8192, 2048, 5632), (7, 33, 65)):
        assert lib.cocodc_lm_glu_grad_workspace(T, D, F) >= 4 * T * F
    assert lib.cocodc_lm_embed_grad_workspace(-1, 4, 4) == 0
    assert lib.cocodc_lm_glu_grad_workspace(4, 4, 2 ** 60) == 0


def test_matrices_are_described_by_their_strides(B):
    import torch
    t = torch.zeros(6, 10)
    assert B._matrix(t, "t")[1] == 10
    assert B._matrix(t[::2, 2:7], "t") == (t.data_ptr() + 8, 20, 3, 5)
    assert B._matrix(t[:1, :4], "t")[1] >= 4
    with pytest.raises(ValueError):
        B._matrix(t.t(), "t")
    with pytest.raises(ValueError):
        B._matrix(t[0], "t")
