"""The small language model whose whole step runs on the library's operators: gradients against autograd, the update against elementary
operations, and a run under the outer step.  How far a loss falls is not looked at."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def worker(V, D, F, T, seed=1, **kw):
    from paper_2504_17672_b200 import binding as B
    from paper_2504_17672_b200.toy_lm import CompleteWorker
    g = torch.Generator(device="cuda").manual_seed(seed)
    row = (torch.randn(V * D + 3 * F * D + 2 * D, generator=g, device="cuda") * 0.1).bfloat16().float()
    row[-2 * D:] = row[-2 * D:].add(1).bfloat16().float()
    grad = torch.zeros_like(row)
    ids, targets = (torch.randint(0, V, (T,), generator=g, device="cuda") for _ in range(2))
    return CompleteWorker(B.LmOps(0), row, grad, V, D, F, T, **kw), ids, targets


@pytest.mark.parametrize("V,D,F,T", [(211, 64, 136, 96), (509, 128, 344, 300), (100, 72, 40, 1)])
def test_gradients_against_autograd(V, D, F, T):
    k, ids, targets = worker(V, D, F, T)
    loss = float(k.step(ids, targets))
    p = {n: v.detach().clone().requires_grad_() for n, v in k.w.items()}

    def norm(x, w):
        return x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w

    x = torch.nn.functional.embedding(ids, p["table"]) * math.sqrt(D)
    n = norm(x, p["norm1"])
    h = torch.nn.functional.silu(n @ p["gate"].t()) * (n @ p["up"].t())
    want = torch.nn.functional.cross_entropy(norm(x + h @ p["down"].t(), p["norm2"]) @ p["table"].t(), targets)
    want.backward()
    # activations and their gradients are bfloat16 (2^-8) some sixteen times over
    assert abs(loss - float(want.detach())) < 0.02 * abs(float(want.detach()))
    for name in p:
        err = torch.linalg.vector_norm(k.g[name].float() - p[name].grad) / torch.linalg.vector_norm(p[name].grad)
        assert float(err) < 16 * 2.0 ** -8, (name, float(err))


@pytest.mark.parametrize("bits", [32, 8])
def test_update_moves_parameters_and_their_copies(bits):
    k, ids, targets = worker(211, 64, 136, 96, state_bits=bits)
    k.step(ids, targets)
    before = {n: v.clone() for n, v in k.w.items()}
    k.update(1, 1e-3, seed=5)
    for n, w in k.w.items():
        # the first step of AdamW: m / (1 - b1) = g, sqrt(v / (1 - b2)) = |g|, to 40 roundings
        g = k.g[n].float()
        want = before[n].double() * (1 - 1e-3 * (0.01 if w.dim() == 2 else 0.0)) - 1e-3 * g.double() / (g.double().abs() + 1e-8)
        assert bool(((w.double() - want).abs() <= 40 * 2.0 ** -24 * (1e-3 + want.abs())).all()), n
        if n in k.b:
            assert torch.equal(k.b[n], w.bfloat16()), n


@pytest.mark.parametrize("bits", [32, 8])
def test_run_under_the_outer_step_is_reproducible(bits):
    from paper_2504_17672_b200.toy_lm import run_toy_lm
    a, b = (run_toy_lm(steps=40, tokens=128, log_every=10, complete=True, state_bits=bits) for _ in range(2))
    assert a.losses == b.losses and a.continuation == b.continuation and a.syncs == b.syncs > 0
    assert all(math.isfinite(x) for _, x in a.losses)
