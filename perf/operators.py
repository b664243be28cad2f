"""Cases that measure the operators of a worker's local step: what goes into a language model (the embedding lookup), what
its feed-forward half computes (the gated pair of projections) and what comes out (log probabilities of given tokens), each
with its gradient.

A case is a dict of plain values.  `prepare` makes its inputs on the GPU from a seed, `run` makes one pass: with `own` set
through the library's entry points, otherwise as elementary torch operations in 32 bits.  `exact` is the definition in 64 bits.

Shapes come from the synthetic workloads (synth/configs.py): gpt2_small (768 wide, 50257 tokens), paper_150m (1024 wide, 2816
in the feed-forward, 32000 tokens, 256 sequences of 1024 tokens over four workers = 65536 tokens a worker and step), llama_1b
(2048 / 5632 / 32000) and llama_3b (3200 / 8640 / 32000)."""

import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "i32": torch.int32, "i64": torch.int64}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4, "i32": 4, "i64": 8}


# ---------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # decoding: the rows of eight sequences' newest tokens, launch latency is what counts
        dict(name="embed_decode", op="embed", T=8, D=768, V=50257, table="bf16", out="bf16", ids="i64", scale=1.0),
        # training under mixed precision: fp32 master table, bf16 activations, one worker's batch of the 150M model
        dict(name="embed_train", op="embed", T=65536, D=1024, V=32000, table="fp32", out="bf16", ids="i64", scale=32.0),
        # gradient of a micro-batch of four sequences plus a ragged rest, large vocabulary: mostly rows that no token names
        dict(name="embed_grad_micro", op="embed_grad", T=4099, D=768, V=50257, grad="bf16", table="fp32", ids="i64", scale=1.0),
        # gradient of the whole batch of one worker of the 150M model: mostly rows that many tokens share
        dict(name="embed_grad_train", op="embed_grad", T=65536, D=1024, V=32000, grad="bf16", table="fp32", ids="i32", scale=32.0),
        # serving one token: both weight matrices are read once, nothing else matters
        dict(name="glu_token", op="glu", T=1, D=2048, F=5632, type="bf16", act="silu", save=False),
        # serving a ragged batch of tokens in half precision
        dict(name="glu_batch", op="glu", T=37, D=1024, F=2816, type="fp16", act="gelu", save=False),
        # training forward at the widest configured shape, gate and up projections kept for the backward pass
        dict(name="glu_train", op="glu", T=8192, D=3200, F=8640, type="bf16", act="silu", save=True),
        # training backward: gradients of the input and of both weight matrices
        dict(name="glu_grad_train", op="glu_grad", T=8192, D=2048, F=5632, type="bf16", act="silu"),
        # sampling step of one sequence: log probability and entropy of the drawn token with eight alternatives
        dict(name="logprobs_token", op="logprobs", T=1, V=50257, type="bf16", ids="i64", k=8, scale=1.25),
        # evaluation of a ragged batch on fp32 logits with five alternatives
        dict(name="logprobs_eval", op="logprobs", T=1333, V=32000, type="fp32", ids="i64", k=5, scale=1.0),
        # training loss on bf16 logits whose rows start at odd addresses (50257 values a row)
        dict(name="logprobs_train", op="logprobs", T=8192, V=50257, type="bf16", ids="i64", k=0, scale=1.0),
        # its gradient, entropy bonus included
        dict(name="logprobs_grad_train", op="logprobs_grad", T=8192, V=50257, type="bf16", ids="i64", scale=1.0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "glu", "glu", "glu_grad", "logprobs", "logprobs", "logprobs_grad"])
    ids = rng.choice(["i32", "i64"])
    if op in ("embed", "embed_grad"):
        T, D, V = _log(rng, 1, 65536), _log(rng, 64, 2048), _log(rng, 500, 50257)
        D = D // 8 * 8 if rng.random() < 0.75 else D
        T = min(T, 65536 * 1024 // D)
        scale = rng.choice([1.0, math.sqrt(D)])
        if op == "embed":
            return dict(op=op, T=T, D=D, V=V, table=rng.choice(["fp32", "bf16", "fp16"]), out=rng.choice(["bf16", "fp16", "fp32"]), ids=ids, scale=scale)
        return dict(op=op, T=T, D=D, V=V, grad=rng.choice(["bf16", "fp16", "fp32"]), table=rng.choice(["fp32", "fp32", "bf16"]), ids=ids, scale=scale)
    if op in ("glu", "glu_grad"):
        case = dict(op=op, T=_log(rng, 1 if op == "glu" else 32, 8192), D=8 * _log(rng, 32, 256), F=8 * _log(rng, 64, 704),
                    type=rng.choice(["bf16", "bf16", "fp16"]), act=rng.choice(["silu", "gelu"]))
        return dict(case, save=rng.random() < 0.5) if op == "glu" else case
    T, V, kind = _log(rng, 1, 8192), _log(rng, 1000, 50257), rng.choice(["bf16", "fp16", "fp32"])
    T = min(T, 8192 * 50257 // 2 // V) if kind == "fp32" else T
    case = dict(op=op, T=T, V=V, type=kind, ids=ids, scale=rng.choice([1.0, 0.7, 1.25]))
    return dict(case, k=rng.choice([0, 1, 5, 8, 20])) if op == "logprobs" else case


# --------------------------------------------------------------------------------------------------------------- inputs

def _tokens(case, g, dev):
    """Token ids whose frequency falls with the id as in text (id v has probability ln((v+2)/(v+1)) / ln(V+1)); one in fifty
    is -1, a place without a token (padding)."""
    V, T = case["V"], case["T"]
    u = torch.rand(T, generator=g, device=dev, dtype=torch.float64)
    ids = (torch.exp(u * math.log(V + 1)).long() - 1).clamp_(0, V - 1)
    ids[torch.rand(T, generator=g, device=dev) < 0.02] = -1
    return ids.to(TYPES[case["ids"]])


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))

    def normal(*shape, std=1.0, kind):
        return torch.randn(*shape, generator=g, device=dev).mul_(std).to(TYPES[kind])

    s, op, T = dict(case), case["op"], case["T"]
    if op == "embed":
        s["weight"] = normal(case["V"], case["D"], std=0.02, kind=case["table"])
        s["tokens"] = _tokens(case, g, dev)
        s["y"] = torch.empty(T, case["D"], dtype=TYPES[case["out"]], device=dev)
    elif op == "embed_grad":
        s["tokens"] = _tokens(case, g, dev)
        s["dy"] = normal(T, case["D"], std=0.1, kind=case["grad"])
        s["dweight"] = torch.empty(case["V"], case["D"], dtype=TYPES[case["table"]], device=dev)
    elif op in ("glu", "glu_grad"):
        D, F, kind = case["D"], case["F"], case["type"]
        s["x"] = normal(T, D, kind=kind)
        s["wg"], s["wu"] = (normal(F, D, std=D ** -0.5, kind=kind) for _ in range(2))
        if op == "glu":
            s["h"] = torch.empty(T, F, dtype=TYPES[kind], device=dev)
            s["gate"], s["up"] = (torch.empty_like(s["h"]) if case["save"] else None for _ in range(2))
        else:
            s["gate"], s["up"] = s["x"] @ s["wg"].t(), s["x"] @ s["wu"].t()
            s["dh"] = normal(T, F, std=0.1, kind=kind)
            s["dx"], s["dwg"], s["dwu"] = (torch.empty_like(s[k]) for k in ("x", "wg", "wu"))
    else:
        V = case["V"]
        s["logits"] = normal(T, V, std=2.0, kind=case["type"])
        s["tokens"] = _tokens(case, g, dev)
        # a trained model gives the token that came some of the mass
        at = s["tokens"].long().clamp(min=0).unsqueeze(1)
        s["logits"].scatter_add_(1, at, torch.rand(T, 1, generator=g, device=dev).mul_(14.0).to(s["logits"].dtype))
        f32 = lambda *shape: torch.empty(*shape, device=dev)  # noqa: E731
        if op == "logprobs":
            s["logp"], s["entropy"], s["lse"] = f32(T), f32(T), f32(T)
            s["top_ids"] = torch.empty(T, case["k"], dtype=torch.int32, device=dev) if case["k"] else None
            s["top_logp"] = f32(T, case["k"]) if case["k"] else None
        else:  # the statistics come from the forward pass
            z = s["logits"].float() * case["scale"]
            s["lse"] = torch.logsumexp(z, 1)
            z -= s["lse"].unsqueeze(1)
            s["entropy"] = -(z.exp() * z).sum(1)
            del z
            s["dlogp"] = torch.randn(T, generator=g, device=dev) * 0.5 - 1.0
            s["dentropy"] = torch.full((T,), -0.01, device=dev)
            s["dlogits"] = torch.empty_like(s["logits"])
    return s


# ----------------------------------------------------------------------------------------------------------- one pass

_ops = None


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    global _ops
    if _ops is None:
        from paper_2504_17672_b200 import binding
        _ops = binding.LmOps(torch.cuda.current_device())
    op = s["op"]
    if op == "embed":
        _ops.cocodc_lm_embed(s["weight"], s["tokens"], s["y"], scale=s["scale"])
        return s["y"]
    if op == "embed_grad":
        _ops.cocodc_lm_embed_grad(s["dy"], s["tokens"], s["dweight"], scale=s["scale"])
        return s["dweight"]
    if op == "glu":
        _ops.cocodc_lm_glu(s["x"], s["wg"], s["wu"], s["h"], gate=s["gate"], up=s["up"], act=s["act"])
        return {k: s[k] for k in ("h", "gate", "up") if s[k] is not None}
    if op == "glu_grad":
        _ops.cocodc_lm_glu_grad(s["dh"], s["gate"], s["up"], s["x"], s["wg"], s["wu"], s["dx"], s["dwg"], s["dwu"], act=s["act"])
        return {k: s[k] for k in ("dx", "dwg", "dwu")}
    if op == "logprobs":
        _ops.cocodc_lm_logprobs(s["logits"], s["tokens"], s["logp"], entropy=s["entropy"], lse=s["lse"], top_ids=s["top_ids"],
                                top_logp=s["top_logp"], scale=s["scale"])
        return {k: s[k] for k in ("logp", "entropy", "lse", "top_ids", "top_logp") if s[k] is not None}
    _ops.cocodc_lm_logprobs_grad(s["logits"], s["tokens"], s["lse"], s["entropy"], s["dlogp"], s["dentropy"], s["dlogits"], scale=s["scale"])
    return s["dlogits"]


def _act(g, kind):
    """The activation and its derivative."""
    if kind == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    a, b = math.sqrt(2.0 / math.pi), 0.044715
    t = torch.tanh(a * (g + b * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * a * (1.0 + 3.0 * b * g * g)


def _run_plain(s):
    op = s["op"]
    if op == "embed":
        t = s["tokens"].long()
        y = s["weight"][t.clamp(min=0)].float() * s["scale"]
        return (y * (t >= 0).unsqueeze(1)).to(s["y"].dtype)
    if op == "embed_grad":
        t = s["tokens"].long()
        dy = s["dy"].float() * (t >= 0).unsqueeze(1)
        dw = torch.zeros(s["dweight"].shape, device=dy.device)
        dw.index_add_(0, t.clamp(min=0), dy)
        return (dw * s["scale"]).to(s["dweight"].dtype)
    if op == "glu":
        x = s["x"].float()
        g, u = x @ s["wg"].float().t(), x @ s["wu"].float().t()
        out = {"h": _act(g, s["act"])[0] * u}
        if s["save"]:
            out.update(gate=g, up=u)
        return {k: v.to(s["x"].dtype) for k, v in out.items()}
    if op == "glu_grad":
        dh, g, u, x = s["dh"].float(), s["gate"].float(), s["up"].float(), s["x"].float()
        a, d = _act(g, s["act"])
        dg, du = dh * u * d, dh * a
        out = {"dx": dg @ s["wg"].float() + du @ s["wu"].float(), "dwg": dg.t() @ x, "dwu": du.t() @ x}
        return {k: v.to(s["x"].dtype) for k, v in out.items()}
    z, t = s["logits"].float() * s["scale"], s["tokens"].long()
    there, at = t >= 0, t.clamp(min=0).unsqueeze(1)
    if op == "logprobs":
        m = z.amax(1, keepdim=True)
        e = torch.exp(z - m)
        total = e.sum(1, keepdim=True)
        lse = m + torch.log(total)
        entropy = torch.log(total) - (e * (z - m)).sum(1, keepdim=True) / total
        zero = torch.zeros((), device=z.device)
        out = {"logp": torch.where(there, (z.gather(1, at) - lse).squeeze(1), zero), "entropy": entropy.squeeze(1), "lse": lse.squeeze(1)}
        if s["k"]:
            # an order on (value, lower index first) as whole numbers, so that ties have one answer
            bits = (s["logits"].float() + 0.0).view(torch.int32).long()
            key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) * (1 << 20) + ((1 << 20) - 1 - torch.arange(z.shape[1], device=z.device))
            best = torch.topk(key, s["k"], dim=1).indices
            out["top_ids"], out["top_logp"] = best.to(torch.int32), z.gather(1, best) - lse
        return out
    z -= s["lse"].unsqueeze(1)
    p = torch.exp(z)
    dz = -p * (s["dlogp"] * there).unsqueeze(1) - s["dentropy"].unsqueeze(1) * p * (z + s["entropy"].unsqueeze(1))
    dz.scatter_add_(1, at, (s["dlogp"] * there).unsqueeze(1))
    return (dz * s["scale"]).to(s["logits"].dtype)


# -------------------------------------------------------------------------------------------------------------- floors

def work(case):
    op, T = case["op"], case["T"]
    if op in ("embed", "embed_grad"):
        D, V = case["D"], case["V"]
        if op == "embed":  # the rows that some token names, once each
            p = 0.98 * np.diff(np.log(np.arange(1, V + 2))) / math.log(V + 1)
            rows = float(-np.expm1(T * np.log1p(-p)).sum())
            return {"bytes": T * D * BYTES[case["out"]] + rows * D * BYTES[case["table"]] + T * BYTES[case["ids"]], "flops": T * D}
        return {"bytes": T * D * BYTES[case["grad"]] + V * D * BYTES[case["table"]] + T * BYTES[case["ids"]], "flops": T * D}
    if op in ("glu", "glu_grad"):
        D, F, b = case["D"], case["F"], BYTES[case["type"]]
        if op == "glu":
            return {"bytes": b * (T * D + 2 * F * D + T * F * (3 if case["save"] else 1)), "flops": 4 * T * D * F}
        return {"bytes": b * (2 * T * D + 4 * F * D + 3 * T * F), "flops": 8 * T * D * F}
    V, b = case["V"], BYTES[case["type"]]
    if op == "logprobs":
        return {"bytes": T * V * b + T * (BYTES[case["ids"]] + 12 + 8 * case["k"]), "flops": 5 * T * V}
    return {"bytes": 2 * T * V * b + T * (BYTES[case["ids"]] + 16), "flops": 7 * T * V}


# -------------------------------------------------------------------------------------------------- the definition, 64 bits

def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    for k, v in list(s.items()):
        if isinstance(v, torch.Tensor) and v.is_floating_point() and k not in ("y", "dweight", "h", "dx", "dwg", "dwu", "dlogits", "logp", "top_logp", "logits"):
            s[k] = v.double()
    t = s["tokens"].long() if "tokens" in s else None
    if op == "embed":
        y = s["weight"].new_zeros(case["T"], case["D"])
        keep = t >= 0
        y[keep] = case["scale"] * s["weight"].index_select(0, t[keep])
        return y
    if op == "embed_grad":
        keep = t >= 0
        return s["dy"].new_zeros(case["V"], case["D"]).index_add_(0, t[keep], s["dy"][keep]).mul_(case["scale"])
    if op in ("glu", "glu_grad"):
        if op == "glu":
            g, u = torch.mm(s["x"], s["wg"].T), torch.mm(s["x"], s["wu"].T)
        else:
            g, u = s["gate"], s["up"]
        if case["act"] == "silu":
            sig = torch.sigmoid(g)
            value, slope = g * sig, sig + g * sig * (1 - sig)
        else:
            inner = math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
            value = g * (1 + torch.tanh(inner)) / 2
            slope = (1 + torch.tanh(inner)) / 2 + g / 2 / torch.cosh(inner) ** 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * g ** 2)
        if op == "glu":
            return {"h": value * u, "gate": g, "up": u} if case["save"] else {"h": value * u}
        dg, du = s["dh"] * u * slope, s["dh"] * value
        return {"dx": torch.mm(dg, s["wg"]) + torch.mm(du, s["wu"]), "dwg": torch.mm(dg.T, s["x"]), "dwu": torch.mm(du.T, s["x"])}
    rows, out = 1024, []
    for a in range(0, case["T"], rows):
        z = s["logits"][a:a + rows].double() * case["scale"]
        ids, n = t[a:a + rows], z.shape[0]
        here = (ids >= 0).nonzero().squeeze(1)
        if op == "logprobs":
            lse = torch.logsumexp(z, 1)
            lp = z - lse[:, None]
            logp = z.new_zeros(n)
            logp[here] = lp[here, ids[here]]
            got = [logp, -(lp.exp() * lp).sum(1), lse]
            if case["k"]:
                order = torch.sort(s["logits"][a:a + rows].double(), dim=1, descending=True, stable=True).indices[:, :case["k"]]
                got += [order.int(), lp.gather(1, order)]
            out.append(got)
        else:
            lp = z - s["lse"][a:a + rows, None]
            p, d1, d2 = lp.exp(), s["dlogp"][a:a + rows], s["dentropy"][a:a + rows]
            dz = -d2[:, None] * p * (lp + s["entropy"][a:a + rows, None])
            dz[here] -= d1[here, None] * p[here]
            dz[here, ids[here]] += d1[here]
            out.append(dz.mul_(case["scale"]))
    if op == "logprobs_grad":
        return torch.cat(out)
    names = ("logp", "entropy", "lse", "top_ids", "top_logp")
    return {k: torch.cat(v) for k, v in zip(names, zip(*out))}
