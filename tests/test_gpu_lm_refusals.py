"""Calls of the local step's operators that must not be taken for others."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2504_17672_b200 import binding
    return binding


@pytest.fixture()
def ops(B):
    o = B.LmOps(0)
    yield o
    assert o.cocodc_lm_poll_status() == B.OK
    o.close()


def test_alternatives_need_both_of_their_outputs(B, ops):
    x = torch.randn(4, 100, device="cuda")
    lse, top = torch.empty(4, device="cuda"), torch.full((4, 3), 7.0, device="cuda")
    ids = torch.empty(4, 3, dtype=torch.int32, device="cuda")
    for one in (dict(top_logp=top), dict(top_ids=ids)):
        with pytest.raises(B.CocodcError) as e:
            ops.cocodc_lm_logprobs(x, None, None, lse=lse, **one)
        assert e.value.code == B.ERR_INVALID_ARG
    for two in (dict(top_ids=ids, top_logp=top[:, :2].contiguous()), dict(top_ids=ids[:3], top_logp=top), dict(top_ids=ids, top_logp=top.double()),
                dict(top_ids=ids.view(-1), top_logp=top), dict(top_logp=top.view(-1)), dict(top_ids=ids.t(), top_logp=top)):
        with pytest.raises(ValueError):
            ops.cocodc_lm_logprobs(x, None, None, lse=lse, **two)
    assert ops.launch_count == 0
    ops.cocodc_lm_logprobs(x, None, None, lse=lse, top_ids=ids[:, :0], top_logp=top[:, :0])       # none asked for
    ops.cocodc_lm_logprobs(x, None, None, lse=lse, top_ids=ids, top_logp=top)
    assert torch.equal(ids[:, 0].long(), x.argmax(1)) and ops.launch_count == 2
