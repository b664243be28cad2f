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

With `--complete` the whole step runs on the library's operators: norms before the block (of the embedding) and before the head (of the sum with the
block's output), the loss from the head without keeping logits, and AdamW over all tensors at once, which takes the matrices' bfloat16
gradients as they are and leaves the bfloat16 copies that the next step reads; `--states 8` keeps its states in 8 bits.
"""

from __future__ import annotations

import argparse
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


class CompleteWorker(Worker):
    """The same model with norms, its step on the library's operators alone (and three plain products with `down`).

    Parameters [table | gate | up | down | norm of the embedding | norm before the head]; the gradients of the table and the norms are fp32 views
    of the gradient buffer, those of the matrices bfloat16 tensors that AdamW reads directly."""

    def __init__(self, ops: B.LmOps, row: torch.Tensor, grad: torch.Tensor, V: int, D: int, F: int, tokens: int, *, state_bits: int = 32,
                 decay: float = 0.01):
        super().__init__(ops, row, grad, V, D, F, tokens)
        at = V * D + 3 * F * D
        for name in ("norm1", "norm2"):
            self.w[name], self.g[name] = row[at:at + D], grad[at:at + D]
            at += D
        dev, bf16, f32 = row.device, torch.bfloat16, torch.float32
        self.g.update(gate=self.dwg, up=self.dwu, down=torch.empty(D, F, dtype=bf16, device=dev))
        self.b = {k: self.w[k].to(bf16) for k in ("table", "gate", "up", "down")}
        names = ("table", "gate", "up", "down", "norm1", "norm2")
        new = lambda n, dtype: torch.zeros(n, device=dev).to(dtype)  # noqa: E731
        state = torch.float8_e4m3fn if state_bits == 8 else f32
        self.m, self.v = ([new(self.w[k].numel(), state) for k in names] for _ in range(2))
        scales = [[new((self.w[k].numel() + B.LM_ADAM_BLOCK - 1) // B.LM_ADAM_BLOCK, f32) for k in names] for _ in range(2)] if state_bits == 8 else [None, None]
        self.plan = B.AdamTensors(ops, [self.w[k] for k in names], [self.g[k] for k in names], self.m, self.v,
                                  [decay if self.w[k].dim() == 2 else 0.0 for k in names], copies=[self.b.get(k) for k in names],
                                  m_scales=scales[0], v_scales=scales[1])
        full = lambda dtype=bf16: torch.empty(tokens, D, dtype=dtype, device=dev)  # noqa: E731
        self.n1, self.n2, self.s, self.dn = full(), full(), full(), full()
        self.rstd1, self.rstd2 = torch.empty(tokens, device=dev), torch.empty(tokens, device=dev)

    def refresh(self) -> None:
        """The copies of parameters that something else than the optimizer has changed (a completed synchronisation)."""
        for k, v in self.b.items():
            v.copy_(self.w[k])

    def _hidden(self, ids: torch.Tensor, train: bool) -> torch.Tensor:
        T = ids.numel()
        x, h, n1, n2, s = (t[:T] for t in (self.x, self.h, self.n1, self.n2, self.s))
        self.ops.cocodc_lm_embed(self.w["table"], ids, x, scale=math.sqrt(self.D))
        self.ops.cocodc_lm_norm(x, self.w["norm1"], n1, rstd=self.rstd1[:T])
        self.ops.cocodc_lm_glu(n1, self.b["gate"], self.b["up"], h, gate=self.gate[:T] if train else None, up=self.up[:T] if train else None)
        self.ops.cocodc_lm_norm(h @ self.b["down"].t(), self.w["norm2"], n2, residual=x, total=s, rstd=self.rstd2[:T])
        return n2

    def forward(self, ids: torch.Tensor, train: bool = False) -> torch.Tensor:
        return self._hidden(ids, train) @ self.b["table"].t()

    def step(self, ids: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        T = ids.numel()
        logp, lse = self.logp[:T], self.lse[:T]
        y = self._hidden(ids, train=True)
        self.ops.cocodc_lm_head(y, self.b["table"], targets, logp, lse=lse)
        each = torch.full((T,), -1.0 / T, device=y.device)
        dn, dx, h = self.dn[:T], self.dx[:T], self.h[:T]
        self.ops.cocodc_lm_head_grad(y, self.b["table"], targets, lse, each, None, dn, self.g["table"])
        ds = torch.empty_like(dn)
        self.ops.cocodc_lm_norm_grad(dn, self.s[:T], self.w["norm2"], self.rstd2[:T], ds, dweight=self.g["norm2"])
        torch.mm(ds.t(), h, out=self.g["down"])
        self.ops.cocodc_lm_glu_grad(ds @ self.b["down"], self.gate[:T], self.up[:T], self.n1[:T], self.b["gate"], self.b["up"], dn, self.dwg, self.dwu)
        self.ops.cocodc_lm_norm_grad(dn, self.x[:T], self.w["norm1"], self.rstd1[:T], dx, dweight=self.g["norm1"], dtotal=ds)
        self.ops.cocodc_lm_embed_grad(dx, ids, self.g["table"], scale=math.sqrt(self.D), accumulate=True)
        return -logp.mean()

    def update(self, t: int, lr: float, seed: int) -> None:
        self.ops.cocodc_lm_adamw(self.plan, lr, step=t, beta1=0.9, beta2=0.98, seed=seed)


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
               log_every: int = 20, complete: bool = False, state_bits: int = 32) -> ToyLmResult:
    dev = torch.device(device, torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(seed)
    sizes = [V * D, 3 * F * D + (2 * D if complete else 0)]  # fragments: the token table, the block
    N = (sum(sizes) + 3) // 4 * 4
    first = torch.cat([torch.randn(V * D, generator=g, device=dev) * 0.05, torch.randn(3 * F * D, generator=g, device=dev) * D ** -0.5,
                       torch.ones(2 * D if complete else 0, device=dev), torch.zeros(N - sum(sizes), device=dev)])
    w = first.repeat(M, 1)
    theta_g, outer_momentum = first.clone(), torch.zeros(N, device=dev)
    grad = torch.zeros_like(w)
    ops = B.LmOps(dev.index)
    if complete:
        workers = [CompleteWorker(ops, w[i], grad[i], V, D, F, tokens, state_bits=state_bits) for i in range(M)]
    else:
        m1, m2 = torch.zeros_like(w), torch.zeros_like(w)
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
        if complete:
            for i, k in enumerate(workers):
                k.update(t, lr, seed=seed * M + i)
        else:
            m1.lerp_(grad, 0.1)                             # Adam on every worker's row
            m2.lerp_(grad * grad, 0.02)
            w.sub_(lr * (m1 / (1 - 0.9 ** t)) / ((m2 / (1 - 0.98 ** t)).sqrt() + 1e-8))
        done = driver.completed
        driver.after_local_step(t)
        if complete and driver.completed != done:
            for k in workers:
                k.refresh()
        if t % log_every == 0 or t in (1, steps):
            losses.append((t, float(mean)))
    for status in (ctx.cocodc_poll_status(), ops.cocodc_lm_poll_status()):
        if status != B.OK:
            raise RuntimeError(f"device status {status}: {B.status_string(status)}")
    x = text[M]
    return ToyLmResult(losses, workers[0].evaluate(x[:tokens], x[1:tokens + 1]), workers[0].continuation(5, 12), driver.completed)


def main() -> None:
    ap = argparse.ArgumentParser(description="two workers train a small language model under the outer step")
    ap.add_argument("--complete", action="store_true", help="norms, the head's loss and AdamW by the library's operators too")
    ap.add_argument("--states", type=int, choices=(32, 8), default=32, help="bits of AdamW's states (with --complete)")
    args = ap.parse_args()
    r = run_toy_lm(complete=args.complete, state_bits=args.states)
    print("local step  loss (nats a token)")
    for t, loss in r.losses:
        print(f"{t:10d}  {loss:.4f}")
    loss, entropy, hit = r.evaluation
    print(f"unseen text: loss {loss:.4f}, entropy {entropy:.4f}, target among the 4 likeliest {100 * hit:.1f} %  ({r.syncs} syncs)")
    print("continuation of token 5:", r.continuation)


if __name__ == "__main__":
    main()
