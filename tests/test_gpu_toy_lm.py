"""The small language-model run: the local step's operators and the outer step together."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_toy_language_model_learns_and_synchronises():
    from paper_2504_17672_b200.toy_lm import run_toy_lm
    r = run_toy_lm(steps=120)
    start, end = r.losses[0][1], r.losses[-1][1]
    assert abs(start - math.log(509)) < 1.5            # an untrained model is near the uniform distribution
    assert end < 2.0 and r.evaluation[0] < 2.5         # the chain's entropy is 0.94
    assert r.evaluation[2] > 0.8 and r.syncs >= 8
    # the likeliest continuation follows the chain's most frequent map
    assert sum((a * 3 + 1) % 509 == b for a, b in zip(r.continuation, r.continuation[1:])) >= 8


def test_toy_gradients_against_autograd():
    """One local step's gradients against the same model in fp32 torch autograd on the same (bf16-rounded) weights."""
    from paper_2504_17672_b200 import binding as B
    from paper_2504_17672_b200.toy_lm import Worker
    V, D, F, T = 211, 64, 136, 96
    g = torch.Generator(device="cuda").manual_seed(1)
    row = (torch.randn(V * D + 3 * F * D, generator=g, device="cuda") * 0.1).bfloat16().float()
    grad = torch.zeros_like(row)
    ops = B.LmOps(0)
    k = Worker(ops, row, grad, V, D, F, T)
    ids, targets = (torch.randint(0, V, (T,), generator=g, device="cuda") for _ in range(2))
    loss = float(k.step(ids, targets))
    p = {n: v.detach().clone().requires_grad_() for n, v in k.w.items()}
    x = torch.nn.functional.embedding(ids, p["table"]) * math.sqrt(D)
    h = torch.nn.functional.silu(x @ p["gate"].t()) * (x @ p["up"].t())
    want = torch.nn.functional.cross_entropy((x + h @ p["down"].t()) @ p["table"].t(), targets)
    want.backward()
    # activations and their gradients are bfloat16 (2^-8) a dozen times over, independently over thousands of terms
    assert abs(loss - float(want.detach())) < 0.02 * abs(float(want.detach()))
    for n in p:
        err = torch.linalg.vector_norm(k.g[n] - p[n].grad) / torch.linalg.vector_norm(p[n].grad)
        assert float(err) < 12 * 2.0 ** -8, (n, float(err))
