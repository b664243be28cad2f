"""Toy language-model run: M workers train a small model on synthetic text with the operators of the local step
(binding.LmOps) and are kept together by the outer synchronisation step (schedule.RoundDriver).

Every worker's fp32 parameters are one row of the stacked buffer that the outer step works on:
[token table V x D | gate F x D | up F x D | down D x F].  A local step is mixed precision, as in the paper's experiment
(Section 4.1): embedding lookup to bfloat16, a gated feed-forward block with a residual, the transposed table as output
head, the loss from the log probabilities of the next tokens, then the gradients in the same order backwards (the
table's two gradients meet in one fp32 buffer) and an Adam update.  The text is a Markov chain: after a token come
four possible ones with probabilities 0.7, 0.1, 0.1, 0.1, so that the best reachable loss is 0.94 nats a token;
each worker reads another part of it.

    python -m paper_2504_17672_b200.toy_lm       # prints the loss while it trains, an evaluation and a continuation
"""

from __future__ import annotations

import math
from dataclasses import dataclass
from typing import List, Tuple

import torch

from . import binding as B
from .schedule import RoundDriver


class Worker:
    """Views of one worker's parameters and gradients, and the buffers of its local step."""

    def __init__(self, ops: B.LmOps, row: torch.Tensor, grad: torch.Tensor, V: int, D: int, F: int, tokens: int):
        self.ops, self.V, self.D, self.F = ops, V, D, F
        at, self.w, self.g = 0, {}, {}
        for name, rows, cols in (("table", V, D), ("gate", F, D), ("up", F, D), ("down", D, F)):
            self.w[name] = row[at:at + rows * cols].view(rows, cols)
            self.g[name] = grad[at:at + rows * cols].view(rows, cols)
            at += rows * cols
        dev, bf16 = row.device, torch.bfloat16
        new = lambda *shape, dtype=bf16: torch.empty(*shape, dtype=dtype, device=dev)  # noqa: E731
        self.x, self.h, self.gate, self.up = new(tokens, D), new(tokens, F), new(tokens, F), new(tokens, F)
        self.dx, self.dwg, self.dwu = new(tokens, D), new(F, D), new(F, D)
        self.logp, self.lse = new(tokens, dtype=torch.float32), new(tokens, dtype=torch.float32)

    def forward(self, ids: torch.Tensor, train: bool = False) -> torch.Tensor:
        """Logits of the tokens after `ids`."""
        T = ids.numel()
        self.b = {k: v.to(torch.bfloat16) for k, v in self.w.items()}
        x, h = self.x[:T], self.h[:T]
        self.ops.cocodc_lm_embed(self.w["table"], ids, x, scale=math.sqrt(self.D))
        self.ops.cocodc_lm_glu(x, self.b["gate"], self.b["up"], h, gate=self.gate[:T] if train else None,
                               up=self.up[:T] if train else None)
        self.y = x + h @ self.b["down"].t()
        return self.y @ self.b["table"].t()

    def step(self, ids: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """Fills the gradients of the mean negative log probability of `targets`; returns it (on the device)."""
        T = ids.numel()
        logits = self.forward(ids, train=True)
        logp, lse = self.logp[:T], self.lse[:T]
        self.ops.cocodc_lm_logprobs(logits, targets, logp, lse=lse)
        each = torch.full((T,), -1.0 / T, device=logits.device)
        self.ops.cocodc_lm_logprobs_grad(logits, targets, lse, None, each, None, logits)       # in place
        dy = logits @ self.b["table"]
        self.g["table"].copy_(logits.t() @ self.y)
        self.g["down"].copy_(dy.t() @ self.h[:T])
        dx = self.dx[:T]
        self.ops.cocodc_lm_glu_grad(dy @ self.b["down"], self.gate[:T], self.up[:T], self.x[:T], self.b["gate"], self.b["up"],
                                    dx, self.dwg, self.dwu)
        self.g["gate"].copy_(self.dwg)
        self.g["up"].copy_(self.dwu)
        self.ops.cocodc_lm_embed_grad(dx + dy, ids, self.g["table"], scale=math.sqrt(self.D), accumulate=True)
        return -logp.mean()

    def evaluate(self, ids: torch.Tensor, targets: torch.Tensor, k: int = 4) -> Tuple[float, float, float]:
        """(loss, mean entropy, share of targets among the k likeliest tokens)."""
        T, dev = ids.numel(), ids.device
        logits = self.forward(ids)
        logp, entropy = torch.empty(T, device=dev), torch.empty(T, device=dev)
        top, top_logp = torch.empty(T, k, dtype=torch.int32, device=dev), torch.empty(T, k, device=dev)
        self.ops.cocodc_lm_logprobs(logits, targets, logp, entropy=entropy, top_ids=top, top_logp=top_logp)
        return float(-logp.mean()), float(entropy.mean()), float((top == targets.unsqueeze(1)).any(1).float().mean())

    def continuation(self, token: int, n: int) -> List[int]:
        """The likeliest next token, n times: the operators' single-token forms."""
        dev, out = self.x.device, [token]
        top, top_logp = torch.empty(1, 1, dtype=torch.int32, device=dev), torch.empty(1, 1, device=dev)
        at = torch.tensor([token], dtype=torch.int32, device=dev)
        for _ in range(n):
            self.ops.cocodc_lm_logprobs(self.forward(at), None, None, top_ids=top, top_logp=top_logp)
            at = top[0].clone()
            out.append(int(at))
        return out


def markov_text(g: torch.Generator, V: int, length: int, start: int, device) -> torch.Tensor:
    """Token t + 1 follows token t by one of four fixed affine maps, drawn with probabilities 0.7, 0.1, 0.1, 0.1."""
    r = torch.rand(length, generator=g, device=device).tolist()
    out, t = [], start
    for u in r:
        out.append(t)
        k = 0 if u < 0.7 else 1 + int((u - 0.7) * 10)
        t = (t * (3 + 2 * k) + 7 * k + 1) % V
    return torch.tensor(out, device=device)


@dataclass
class ToyLmResult:
    losses: List[Tuple[int, float]]      # (local step, mean loss over the workers)
    evaluation: Tuple[float, float, float]
    continuation: List[int]
    syncs: int


def run_toy_lm(*, M: int = 2, V: int = 509, D: int = 128, F: int = 344, tokens: int = 512, steps: int = 160, H: int = 16,
               tau: int = 2, lam: float = 0.5, lr: float = 3e-3, seed: int = 0, device: str = "cuda",
               log_every: int = 20) -> ToyLmResult:
    dev = torch.device(device, torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)
    sizes = [V * D, 3 * F * D]                               # fragments: the token table, the block
    N = (sum(sizes) + 3) // 4 * 4
    first = torch.cat([torch.randn(V * D, generator=g, device=dev) * 0.05, torch.randn(3 * F * D, generator=g, device=dev) * D ** -0.5,
                       torch.zeros(N - sum(sizes), device=dev)])
    w = first.repeat(M, 1)
    theta_g, outer_momentum = first.clone(), torch.zeros(N, device=dev)
    grad, m1, m2 = (torch.zeros_like(w) for _ in range(3))
    ops = B.LmOps(dev.index)
    workers = [Worker(ops, w[i], grad[i], V, D, F, tokens) for i in range(M)]
    text = [markov_text(g, V, 20 * tokens + 1, 1 + 17 * i, dev) for i in range(M + 1)]        # the last for the evaluation
    ctx = B.Context(N, [0, 1, 2], [0, sizes[0]], sizes, M, device=dev.index)
    hyper = B.Hyper(M=M, H=H, tau=tau, lam=lam, alpha=1.0)
    driver = RoundDriver(ctx, hyper, w, theta_g, outer_momentum, sizes, gamma=0.4, Tc=1.0, Ts=1.0,
                         budget_kind=B.BUDGET_COUNT, budget=1)
    losses = []
    for t in range(1, steps + 1):
        at = (t * tokens) % (19 * tokens)
        mean = torch.stack([k.step(x[at:at + tokens], x[at + 1:at + tokens + 1]) for k, x in zip(workers, text)]).mean()
        m1.lerp_(grad, 0.1)                                 # Adam on every worker's row
        m2.lerp_(grad * grad, 0.02)
        w.sub_(lr * (m1 / (1 - 0.9 ** t)) / ((m2 / (1 - 0.98 ** t)).sqrt() + 1e-8))
        driver.after_local_step(t)
        if t % log_every == 0 or t in (1, steps):
            losses.append((t, float(mean)))
    for status in (ctx.cocodc_poll_status(), ops.cocodc_lm_poll_status()):
        if status != B.OK:
            raise RuntimeError(f"device status {status}: {B.status_string(status)}")
    x = text[M]
    return ToyLmResult(losses, workers[0].evaluate(x[:tokens], x[1:tokens + 1]), workers[0].continuation(5, 12), driver.completed)


def main() -> None:
    r = run_toy_lm()
    print("local step  loss (nats a token)")
    for t, loss in r.losses:
        print(f"{t:10d}  {loss:.4f}")
    loss, entropy, hit = r.evaluation
    print(f"unseen text: loss {loss:.4f}, entropy {entropy:.4f}, target among the 4 likeliest {100 * hit:.1f} %  ({r.syncs} syncs)")
    print("continuation of token 5:", r.continuation)


if __name__ == "__main__":
    main()
