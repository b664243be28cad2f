"""What the calls report when a launch fails, and when an older error is left on the thread.  The failures are made on the host: a
stream whose capture has become invalid refuses every launch."""

import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu
RELAXED = 2                                                   # cudaStreamCaptureModeRelaxed


@pytest.fixture(scope="module")
def B():
    from paper_2504_17672_b200 import binding
    return binding


@pytest.fixture()
def ops(B):
    o = B.LmOps(0)
    yield o
    o.close()


@pytest.fixture()
def runtime():
    """torch's CUDA runtime.  (The library has one of its own, with its own record of errors.)"""
    lib = ctypes.CDLL("libcudart.so.12")
    yield lib
    lib.cudaGetLastError()


def calls(B, ops, stream):
    """One call of each operator on `stream`, every gradient by each of its ways; (name, call, launches)."""
    bf16, dev = torch.bfloat16, "cuda"
    x, w, h = torch.ones(200, 64, dtype=bf16, device=dev), torch.ones(2048, 64, dtype=bf16, device=dev), torch.ones(200, 2048, dtype=bf16, device=dev)
    odd_x, odd_w, odd_h = (torch.ones(t.shape[0], t.shape[1] + 1, dtype=bf16, device=dev)[:, 1:] for t in (x, w, h))
    dx, dw, du = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    ids, f, one = torch.zeros(200, dtype=torch.int64, device=dev), torch.zeros(200, device=dev), torch.ones(200, device=dev)
    table, lse = torch.zeros(50, 64, device=dev), torch.zeros(200, device=dev)
    work = torch.empty(B.library().cocodc_lm_glu_grad_workspace(200, 64, 2048), dtype=torch.uint8, device=dev)
    work_e = torch.empty(B.library().cocodc_lm_embed_grad_workspace(50, 64, 200), dtype=torch.uint8, device=dev)
    out = torch.empty_like(h)
    torch.cuda.synchronize()
    return [
        ("embed", lambda: ops.cocodc_lm_embed(table, ids, dx, stream=stream), 1),
        ("embed_grad", lambda: ops.cocodc_lm_embed_grad(x, ids, table, workspace=work_e, stream=stream), 2),
        ("glu", lambda: ops.cocodc_lm_glu(x, w, w, out, stream=stream), 1),
        ("glu few", lambda: ops.cocodc_lm_glu(x[:3], w, w, out[:3], stream=stream), 1),
        ("glu off 16 bytes", lambda: ops.cocodc_lm_glu(odd_x, odd_w, odd_w, out, stream=stream), 1),
        # 200 x 64 outputs are two tiles: the contraction over 2048 goes in parts, then the parts are added
        ("glu_grad", lambda: ops.cocodc_lm_glu_grad(h, h, h, x, w, w, dx, dw, du, workspace=work, stream=stream), 4),
        ("glu_grad off 16 bytes", lambda: ops.cocodc_lm_glu_grad(odd_h, odd_h, odd_h, odd_x, odd_w, odd_w, dx, dw, du, workspace=work, stream=stream), 3),
        ("logprobs", lambda: ops.cocodc_lm_logprobs(h, ids, f, lse=lse, stream=stream), 1),
        ("logprobs_grad", lambda: ops.cocodc_lm_logprobs_grad(h, ids, lse, None, one, None, out, stream=stream), 1),
    ]


def test_a_failed_launch_is_reported_and_nothing_is_launched_after_it(B, ops, runtime):
    stream = torch.cuda.Stream()
    every = calls(B, ops, stream)
    raw = ctypes.c_void_p(stream.cuda_stream)
    assert runtime.cudaStreamBeginCapture(raw, RELAXED) == 0
    try:
        assert runtime.cudaStreamSynchronize(raw) != 0        # not allowed while a stream is captured: the capture is invalid from here on
        for name, call, _ in every:
            before = ops.launch_count
            with pytest.raises(B.CocodcError) as e:
                call()
            assert e.value.code == B.ERR_CUDA and ops.launch_count == before, name
    finally:
        graph = ctypes.c_void_p()
        runtime.cudaStreamEndCapture(raw, ctypes.byref(graph))
        runtime.cudaGetLastError()
    for name, call, launches in every:                        # and the stream and the handle are as good as before
        before = ops.launch_count
        call()
        assert ops.launch_count == before + launches, name
    stream.synchronize()
    assert ops.cocodc_lm_poll_status() == B.OK


def test_an_older_error_is_not_a_calls_own(B, ops, runtime):
    stream = torch.cuda.Stream()
    every = calls(B, ops, None)
    raw = ctypes.c_void_p(stream.cuda_stream)
    for name, call, launches in every:
        assert runtime.cudaStreamBeginCapture(raw, RELAXED) == 0
        try:
            assert ops.cocodc_lm_poll_status(stream=stream) == B.ERR_CUDA       # waiting is refused, which is an error of the thread's
        finally:
            graph = ctypes.c_void_p()
            runtime.cudaStreamEndCapture(raw, ctypes.byref(graph))
            runtime.cudaGetLastError()
        before = ops.launch_count
        call()
        assert ops.launch_count == before + launches, name
    torch.cuda.synchronize()
    assert ops.cocodc_lm_poll_status() == B.OK
