"""Operands that are different columns of one buffer, or empty slices of another operand: legal, and with the same results as in
buffers of their own; operands that share an element: refused."""

import math

import pytest
import torch

from test_gpu_lm_ops import BF16, F16, F32, gen, randn

pytestmark = pytest.mark.gpu


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


def columns(rows, widths, dtype, gap=0):
    """Views of consecutive columns of one buffer whose every other element is NaN."""
    buf = torch.full((rows, sum(widths) + gap), math.nan, dtype=dtype, device="cuda")
    at, out = 0, []
    for w in widths:
        out.append(buf[:, at:at + w])
        at += w
    return (*out, buf)


# few tokens, narrow and wide tensor-core tiles, rows off 16 bytes
@pytest.mark.parametrize("T,D,F", [(1, 64, 128), (2, 64, 128), (8, 40, 33), (37, 128, 264), (200, 72, 36), (300, 264, 520), (2100, 264, 1032)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_gate_and_up_are_halves_of_one_buffer(ops, T, D, F, dtype):
    g = gen(T + F)
    x, dh = randn(g, T, D, dtype=dtype), randn(g, T, F, dtype=dtype)
    weights = randn(g, F, 2 * D, std=D ** -0.5, dtype=dtype)
    wg, wu = weights[:, :D], weights[:, D:]
    h, gate, up = (torch.empty(T, F, dtype=dtype, device="cuda") for _ in range(3))
    ops.cocodc_lm_glu(x, wg, wu, h, gate, up)
    for gap in (0, 8):
        gate2, up2, buf = columns(T, (F, F), dtype, gap)
        h2 = torch.empty_like(h)
        ops.cocodc_lm_glu(x, wg, wu, h2, gate2, up2)
        # another path may take rows off 16 bytes, with fp32 sums in another order: one rounding of the type apart
        close = dict(rtol=2 * torch.finfo(dtype).eps, atol=1e-5)
        assert torch.allclose(h2.float(), h.float(), **close) and torch.allclose(gate2.float(), gate.float(), **close)
        assert torch.allclose(up2.float(), up.float(), **close) and bool(torch.isnan(buf[:, 2 * F:]).all())
        if F % 8 == 0:
            assert torch.equal(h2, h) and torch.equal(gate2, gate) and torch.equal(up2, up)
        up3, gate3, h3, buf = columns(T, (F, F, F), dtype, gap)        # the other way round, h beside them
        ops.cocodc_lm_glu(x, wg, wu, h3, gate3, up3)
        assert torch.equal(h3.nan_to_num(), h2.nan_to_num()) or F % 8
        assert torch.allclose(up3.float(), up.float(), **close) and bool(torch.isnan(buf[:, 3 * F:]).all())
        gate2, up2, _ = columns(T, (F, F), dtype, gap)
        gate2.copy_(gate), up2.copy_(up)
        want, got = ([torch.empty(n, D, dtype=dtype, device="cuda") for n in (T, F, F)] for _ in range(2))
        ops.cocodc_lm_glu_grad(dh, gate, up, x, wg, wu, *want)
        dwg, dwu, buf = columns(F, (D, D), dtype, gap)
        ops.cocodc_lm_glu_grad(dh, gate2, up2, x, wg, wu, got[0], dwg, dwu)
        assert torch.equal(got[0], want[0]) and torch.equal(dwg, want[1]) and torch.equal(dwu, want[2])
        assert bool(torch.isnan(buf[:, 2 * D:]).all())


@pytest.mark.parametrize("T,V", [(1, 64), (2, 64), (5, 1000), (3, 777), (200, 4099)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_logits_and_their_gradient_in_one_buffer(ops, T, V, dtype):
    g = gen(V)
    logits, grad, buf = columns(T, (V, V), dtype, 3)
    logits.copy_(randn(g, T, V))
    targets = torch.randint(0, V, (T,), generator=g, device="cuda")
    lse, one, logp = (torch.empty(T, device="cuda") for _ in range(3))
    one.fill_(1.0)
    ops.cocodc_lm_logprobs(logits, targets, logp, lse=lse)
    want = torch.empty(T, V, dtype=dtype, device="cuda")
    ops.cocodc_lm_logprobs_grad(logits, targets, lse, None, one, None, want)
    before = logits.clone()
    ops.cocodc_lm_logprobs_grad(logits, targets, lse, None, one, None, grad)
    assert torch.equal(grad, want) and torch.equal(logits, before) and bool(torch.isnan(buf[:, 2 * V:]).all())


@pytest.mark.parametrize("D", [16, 33, 264])
def test_table_and_rows_in_one_buffer(ops, D):
    g = gen(D)
    table, y, buf = columns(50, (D, D), F32, 4)
    w = randn(g, 50, D)
    table.copy_(w)
    ids = torch.randint(0, 50, (50,), generator=g, device="cuda")
    ops.cocodc_lm_embed(table, ids, y, scale=2.0)
    assert torch.equal(y, 2.0 * w[ids]) and torch.equal(table, w)
    want = torch.empty(50, D, device="cuda")
    ops.cocodc_lm_embed_grad(y, ids, want)
    dy = y.clone()
    ops.cocodc_lm_embed_grad(y, ids, table)
    assert torch.equal(table, want) and torch.equal(y, dy) and bool(torch.isnan(buf[:, 2 * D:]).all())


def test_empty_operands_lie_in_nobodys_way(B, ops):
    """T = 0 with the addresses of the empty operands in the middle of the outputs (a tensor without elements has address 0 in torch)."""
    lib, stream = B.library(), torch.cuda.current_stream().cuda_stream
    dwg, dwu = (torch.full((24, 16), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    w = torch.ones(24, 16, dtype=BF16, device="cuda")
    work = torch.empty(lib.cocodc_lm_glu_grad_workspace(0, 16, 24), dtype=torch.uint8, device="cuda")
    x, h, dx = dwg.data_ptr() + 64, dwu.data_ptr() + 128, dwu.data_ptr() + 32
    assert lib.cocodc_lm_glu_grad(ops._h, B.ACT_SILU, 1, h, 24, h, h, 24, x, 16, w.data_ptr(), w.data_ptr(), 16, 0, 16, 24, dx, 16,
                                  dwg.data_ptr(), dwu.data_ptr(), 16, work.data_ptr(), work.numel(), stream) == B.OK
    assert bool((dwg == 0).all()) and bool((dwu == 0).all())
    table = torch.full((6, 8), 3.0, device="cuda")
    work = torch.empty(lib.cocodc_lm_embed_grad_workspace(6, 8, 0), dtype=torch.uint8, device="cuda")
    assert lib.cocodc_lm_embed_grad(ops._h, table.data_ptr() + 32, 0, 8, table.data_ptr() + 64, 1, 0, 6, 8, 1.0, 0, table.data_ptr(), 0, 8,
                                    work.data_ptr(), work.numel(), stream) == B.OK
    assert bool((table == 0).all())


def test_what_overlaps_is_refused(B, ops):
    x, w = torch.ones(4, 16, dtype=BF16, device="cuda"), torch.ones(24, 16, dtype=BF16, device="cuda")
    h = torch.empty(4, 24, dtype=BF16, device="cuda")
    buf = torch.empty(4, 96, dtype=BF16, device="cuda")
    before = ops.launch_count
    for gate, up in ((buf[:, :24], buf[:, 23:47]), (buf[:, 23:47], buf[:, :24])):      # one column in common
        with pytest.raises(B.CocodcError) as e:
            ops.cocodc_lm_glu(x, w, w, h, gate=gate, up=up)
        assert e.value.code == B.ERR_ALIAS
    logits = torch.zeros(8, 40, device="cuda")
    f = torch.zeros(3, device="cuda")
    ids = torch.zeros(3, dtype=torch.int64, device="cuda")
    flat = logits.view(-1)
    wraps = flat.as_strided((3, 16), (40, 1), 30)             # columns 30 .. 39 and 0 .. 5 of the row after
    wider = flat.as_strided((3, 16), (50, 1), 20)
    inside = flat.as_strided((1, 16), (16, 1), 70)            # columns 30 .. 39 of row 1 and 0 .. 5 of row 2
    for d in (wraps, wider):
        with pytest.raises(B.CocodcError) as e:
            ops.cocodc_lm_logprobs_grad(logits[:3, :16], ids, f, None, f.clone(), None, d)
        assert e.value.code == B.ERR_ALIAS
    with pytest.raises(B.CocodcError) as e:
        ops.cocodc_lm_embed(logits[:, :16], ids[:1], inside)
    assert e.value.code == B.ERR_ALIAS
    assert ops.launch_count == before
