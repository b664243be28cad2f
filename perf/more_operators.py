"""Cases that measure the operators which complete a worker's local step: the root-mean-square norm with the residual's
addition (and its output in 8 bits), the output head with its loss, in pieces of the vocabulary and without keeping the
logits, each with its gradient, and the AdamW step over all tensors of a model with states in 32 or in 8 bits.

A case is a dict of plain values.  `prepare` makes its inputs on the GPU from a seed, `run` makes one pass: with `own` set
through the library's entry points, otherwise as elementary torch operations in 32 bits.  `exact` is the definition in 64 bits.

Shapes come from the synthetic workloads (synth/configs.py): gpt2_small (768 wide, 50257 tokens), paper_150m (1024 wide, 2816
in the feed-forward, 32000 tokens, 65536 tokens a worker and step), llama_1b (2048 / 5632 / 32000), llama_3b (3200 / 8640 / 32000),
and from the toy language model (128 / 344 / 509)."""

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "i32": torch.int32, "i64": torch.int64}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4, "i32": 4, "i64": 8}
EPS = 1e-5
E4M3 = torch.float8_e4m3fn
# AdamW: rates and decays of the paper's kind of run, one gradient scale for the whole step (clipping)
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP, CLIP = 1e-4, 0.9, 0.95, 1e-8, 0.1, 1000, 0.75


# ---------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # serving one token: launch latency is what counts
        dict(name="norm_token", op="norm", T=1, D=2048, type="bf16", sum="bf16", weight="bf16", residual=True, out="same"),
        # training forward of one worker of the 150M model: sum kept in fp32 as the residual stream, statistics for the backward pass
        dict(name="norm_train", op="norm", T=65536, D=1024, type="bf16", sum="fp32", weight="fp32", residual=True, out="same"),
        # a ragged batch at the widest configured shape whose next product takes 8 bits: scales per 128 columns
        dict(name="norm_8bit", op="norm", T=4099, D=3200, type="bf16", sum="bf16", weight="bf16", residual=True, out="group"),
        # training backward: the branch's gradient joins the residual stream's, and the weight's is summed over all tokens
        dict(name="norm_grad_train", op="norm_grad", T=65536, D=1024, type="bf16", sum="bf16", weight="fp32", stream=True),
        # serving one token: its log probability costs one read of the table
        dict(name="head_token", op="head", T=1, D=2048, V=32000, type="bf16", ids="i64", scale=1.0),
        # evaluation of a ragged batch in half precision over the large vocabulary, at a temperature
        dict(name="head_eval", op="head", T=1333, D=768, V=50257, type="fp16", ids="i32", scale=1.25),
        # training forward of a micro-batch of the 1B model
        dict(name="head_train", op="head", T=8192, D=2048, V=32000, type="bf16", ids="i64", scale=1.0),
        # gradient of a micro-batch of four sequences plus a ragged rest
        dict(name="head_grad_micro", op="head_grad", T=4099, D=768, V=50257, type="bf16", ids="i64", scale=1.0, zloss=False),
        # training backward of a micro-batch of the 1B model, with a penalty on the log-sum-exp
        dict(name="head_grad_train", op="head_grad", T=8192, D=2048, V=32000, type="bf16", ids="i64", scale=1.0, zloss=True),
        # the toy language model: eleven small tensors, launch latency is what counts
        dict(name="adamw_toy", op="adamw", L=1, D=128, F=344, V=509, grad="fp32", copy="bf16", bits=32),
        # the GPT-2-small-shaped model with fp32 gradients and states, parameters alone
        dict(name="adamw_gpt2", op="adamw", L=12, D=768, F=2048, V=50257, grad="fp32", copy="none", bits=32),
        # the 150M model with its token table, bf16 gradients, 8-bit states and a bf16 copy of the parameters for the next step
        dict(name="adamw_150m_8bit", op="adamw", L=12, D=1024, F=2816, V=32000, grad="bf16", copy="bf16", bits=8),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "head", "head", "head_grad", "adamw", "adamw"])
    kind = rng.choice(["bf16", "bf16", "fp16"])
    if op in ("norm", "norm_grad"):
        T, D = _log(rng, 1, 65536), _log(rng, 64, 4096)
        D = D // 8 * 8 if rng.random() < 0.8 else D
        T = min(T, 65536 * 1024 // D)
        kind = rng.choice([kind, kind, "fp32"])
        case = dict(op=op, T=T, D=D, type=kind, sum=rng.choice([kind, "fp32"]), weight=rng.choice([kind, "fp32"]))
        if op == "norm":
            return dict(case, residual=rng.random() < 0.7, out=rng.choice(["same", "same", "row", "group"]))
        return dict(case, stream=rng.random() < 0.7)
    if op in ("head", "head_grad"):
        T, D, V = _log(rng, 1 if op == "head" else 32, 8192), 8 * _log(rng, 16, 256), _log(rng, 1000, 50257)
        T = min(T, 8192 * 2048 * 32000 // (D * V))
        case = dict(op=op, T=T, D=D, V=V, type=kind, ids=rng.choice(["i32", "i64"]), scale=rng.choice([1.0, 0.7, 1.25]))
        return case if op == "head" else dict(case, zloss=rng.random() < 0.5)
    D, F, V = _log(rng, 64, 1024), _log(rng, 128, 2816), _log(rng, 500, 50257)
    L = _log(rng, 1, 12)
    if rng.random() < 0.7:
        D, F = max(8, D // 8 * 8), max(8, F // 8 * 8)
    return dict(op=op, L=L, D=D, F=F, V=V, grad=rng.choice(["fp32", "bf16", "fp16"]), copy=rng.choice(["none", "bf16", "fp16"]), bits=rng.choice([8, 32]))


# --------------------------------------------------------------------------------------------------------------- inputs

def _tensors(case):
    """(elements, weight decay) of every tensor: matrices first, then the norms' weights, which do not decay."""
    L, D, F, V = case["L"], case["D"], case["F"], case["V"]
    return [(V * D, DECAY)] + [(D * D, DECAY)] * (4 * L) + [(F * D, DECAY)] * (3 * L) + [(D, 0.0)] * (2 * L + 1)


def _tokens(case, g, dev):
    """Token ids whose frequency falls with the id as in text; one in fifty is -1, a place without a token."""
    V, T = case["V"], case["T"]
    u = torch.rand(T, generator=g, device=dev, dtype=torch.float64)
    ids = (torch.exp(u * math.log(V + 1)).long() - 1).clamp_(0, V - 1)
    ids[torch.rand(T, generator=g, device=dev) < 0.02] = -1
    return ids.to(TYPES[case["ids"]])


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))

    def normal(*shape, std=1.0, kind="fp32"):
        return torch.randn(*shape, generator=g, device=dev).mul_(std).to(TYPES[kind])

    s, op = dict(case), case["op"]
    f32 = lambda *shape: torch.empty(*shape, device=dev)  # noqa: E731
    if op in ("norm", "norm_grad"):
        T, D, kind = case["T"], case["D"], case["type"]
        s["weight_"] = (1.0 + 0.2 * normal(D)).to(TYPES[case["weight"]])
        if op == "norm":
            s["x"] = normal(T, D, kind=kind)
            s["r"] = normal(T, D, std=3.0, kind=case["sum"]) if case["residual"] else None
            s["total"] = torch.empty_like(s["r"]) if case["residual"] else None
            s["rstd"] = f32(T)
            s["y"] = torch.empty(T, D, dtype=TYPES[kind] if case["out"] == "same" else E4M3, device=dev)
            s["y_scale"] = None if case["out"] == "same" else f32(T, 1 if case["out"] == "row" else (D + 127) // 128)
        else:
            s["total"] = normal(T, D, std=3.0, kind=case["sum"])
            s["rstd"] = torch.rsqrt(s["total"].double().square().mean(1) + EPS).float()
            s["dy"] = normal(T, D, std=0.1, kind=kind)
            s["dstream"] = normal(T, D, std=0.1, kind=case["sum"]) if case["stream"] else None
            s["dx"] = torch.empty_like(s["total"])
            s["dweight"] = f32(D)
    elif op in ("head", "head_grad"):
        T, D, V, kind = case["T"], case["D"], case["V"], case["type"]
        s["table"] = normal(V, D, std=2.0 * D ** -0.5, kind=kind)
        s["tokens"] = _tokens(case, g, dev)
        # a trained model's hidden state points some way towards the token that came
        pull = torch.rand(T, 1, generator=g, device=dev).mul_(2.0)
        s["x"] = (normal(T, D) + pull * s["table"][s["tokens"].long().clamp(min=0)].float()).to(TYPES[kind])
        s["logp"], s["lse"] = f32(T), f32(T)
        if op == "head_grad":  # the statistics come from the forward pass
            for a in range(0, T, 2048):
                z = (s["x"][a:a + 2048].float() @ s["table"].float().t()) * case["scale"]
                s["lse"][a:a + 2048] = torch.logsumexp(z, 1)
                del z
            there = max(1, int((s["tokens"] >= 0).sum()))
            s["dlogp"] = torch.full((T,), -1.0 / there, device=dev) * (0.5 + torch.rand(T, generator=g, device=dev))
            s["dlse"] = 2e-4 / there * s["lse"] if case["zloss"] else None
            s["dx"], s["dtable"] = torch.empty_like(s["x"]), torch.empty_like(s["table"])
    else:
        sizes = _tensors(case)
        # one buffer for all tensors, each of which starts on a multiple of 256 elements; what lies between stays zero
        blocks = [(n + 255) // 256 for n, _ in sizes]
        starts = _running(blocks)
        N = 256 * sum(blocks)
        there = torch.zeros(N, dtype=torch.bool, device=dev)
        for (n, _), at in zip(sizes, starts):
            there[at:at + n] = True
        s["p"] = normal(N, std=0.02).mul_(there)
        spread = torch.exp(normal(sum(blocks))).repeat_interleave(256)      # some parts of a model see larger gradients than others
        s["g"] = (normal(N, std=1e-3) * spread).mul_(there).to(TYPES[case["grad"]])
        m, v = normal(N, std=3e-4) * spread * there, (normal(N).square() + 0.05) * (1e-6 * spread * spread) * there
        del spread, there
        if case["bits"] == 8:
            s["m"], s["m_scale"] = _to_8(m)
            s["v"], s["v_scale"] = _to_8(v.sqrt_())
        else:
            s["m"], s["v"] = m, v
        s["c"] = None if case["copy"] == "none" else s["p"].to(TYPES[case["copy"]])
        s["clip"] = torch.full((1,), CLIP, device=dev)
        s["seed"] = int(seed) & 0x7FFFFFFF
        s["decayed"] = sum(b for b, (_, d) in zip(blocks, sizes) if d > 0)                 # blocks of the tensors that decay
        s["blocks"] = torch.tensor(blocks, device=dev)
        if own:  # the step's handle on a model's tensors, made once by a program that trains it
            s["plan"] = _plan(s, [(at, n) for (n, _), at in zip(sizes, starts)], [d for _, d in sizes])
    return s


def _running(blocks):
    """Where each tensor starts, in elements."""
    at, out = 0, []
    for b in blocks:
        out.append(256 * at)
        at += b
    return out


def _to_8(x):
    """Blocks of 256 as 8-bit numbers times a scale that takes the largest to 448."""
    x = x.view(-1, 256)
    scale = (x.abs().amax(1) / 448.0).clamp_(min=1e-30)
    return (x / scale.unsqueeze(1)).to(E4M3).view(-1), scale


# ----------------------------------------------------------------------------------------------------------- one pass

_ops = None


def _library():
    global _ops
    if _ops is None:
        from paper_2504_17672_b200 import binding
        _ops = binding.LmOps(torch.cuda.current_device())
    return _ops


def _plan(s, places, decay):
    from paper_2504_17672_b200 import binding
    cut = lambda x: None if x is None else [x[at:at + n] for at, n in places]  # noqa: E731
    scales = lambda x: None if x is None else [x[at // 256:(at + n + 255) // 256] for at, n in places]  # noqa: E731
    return binding.AdamTensors(_library(), cut(s["p"]), cut(s["g"]), cut(s["m"]), cut(s["v"]), decay, copies=cut(s["c"]),
                               m_scales=scales(s.get("m_scale")), v_scales=scales(s.get("v_scale")))


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    ops, op = _library(), s["op"]
    if op == "norm":
        ops.cocodc_lm_norm(s["x"], s["weight_"], s["y"], residual=s["r"], total=s["total"], rstd=s["rstd"], y_scale=s["y_scale"], eps=EPS)
    elif op == "norm_grad":
        ops.cocodc_lm_norm_grad(s["dy"], s["total"], s["weight_"], s["rstd"], s["dx"], dweight=s["dweight"], dtotal=s["dstream"])
    elif op == "head":
        ops.cocodc_lm_head(s["x"], s["table"], s["tokens"], s["logp"], lse=s["lse"], scale=s["scale"])
    elif op == "head_grad":
        ops.cocodc_lm_head_grad(s["x"], s["table"], s["tokens"], s["lse"], s["dlogp"], s["dlse"], s["dx"], s["dtable"], scale=s["scale"])
    else:
        ops.cocodc_lm_adamw(s["plan"], LR, step=STEP, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, grad_scale=s["clip"], seed=s["seed"])
    return {k: s[k] for k in OUTPUTS[op] if s.get(k) is not None}


OUTPUTS = {"norm": ("y", "y_scale", "total", "rstd"), "norm_grad": ("dx", "dweight"), "head": ("logp", "lse"),
           "head_grad": ("dx", "dtable"), "adamw": ("p", "m", "v", "m_scale", "v_scale", "c")}


def _run_plain(s):
    op = s["op"]
    if op == "norm":
        out, z = {}, s["x"].float()
        if s["r"] is not None:
            out["total"] = (z + s["r"].float()).to(s["r"].dtype)
            z = out["total"].float()
        out["rstd"] = 1.0 / torch.sqrt((z * z).mean(1) + EPS)
        y = z * out["rstd"].unsqueeze(1) * s["weight_"].float()
        if s["y_scale"] is None:
            return dict(out, y=y.to(s["y"].dtype))
        T, D = y.shape
        width = D if s["out"] == "row" else 128
        y = torch.nn.functional.pad(y, (0, -D % width)).view(T, -1, width)
        scale = (y.abs().amax(2) / 448.0).clamp(min=1e-30)
        y = (y / scale.unsqueeze(2)).view(T, -1)[:, :D]
        return dict(out, y=y.to(E4M3), y_scale=scale)
    if op == "norm_grad":
        h = s["total"].float() * s["rstd"].unsqueeze(1)
        dy = s["dy"].float()
        dh = dy * s["weight_"].float()
        dx = (dh - h * (dh * h).mean(1, keepdim=True)) * s["rstd"].unsqueeze(1)
        if s["dstream"] is not None:
            dx = dx + s["dstream"].float()
        return {"dx": dx.to(s["dx"].dtype), "dweight": (dy * h).sum(0)}
    if op in ("head", "head_grad"):
        x, w, t = s["x"].float(), s["table"].float(), s["tokens"].long()
        there, at = t >= 0, t.clamp(min=0).unsqueeze(1)
        z = x @ w.t()
        z *= s["scale"]
        if op == "head":
            m = z.amax(1, keepdim=True)
            picked = z.gather(1, at).squeeze(1)
            lse = (m + torch.log(torch.exp(z - m).sum(1, keepdim=True))).squeeze(1)
            return {"logp": torch.where(there, picked - lse, torch.zeros_like(lse)), "lse": lse}
        z -= s["lse"].unsqueeze(1)
        z.exp_()
        d = s["dlogp"] * there
        z *= (-d if s["dlse"] is None else s["dlse"] - d).unsqueeze(1)
        z.scatter_add_(1, at, d.unsqueeze(1))
        z *= s["scale"]
        return {"dx": (z @ w).to(s["dx"].dtype), "dtable": (z.t() @ x).to(s["dtable"].dtype)}
    return _adamw_plain(s)


def _mix(x):
    """The 32-bit finaliser x ^= x >> 16; x *= 0x85EBCA6B; x ^= x >> 13; x *= 0xC2B2AE35; x ^= x >> 16 on numbers below 2^32.
    A product is taken in halves of the constant, so that it stays below 2^63."""
    mask = 0xFFFFFFFF

    def times(x, c):
        return (x * (c & 0xFFFF) + (((x * (c >> 16)) & 0xFFFF) << 16)) & mask

    x = times(x ^ (x >> 16), 0x85EBCA6B)
    x = times(x ^ (x >> 13), 0xC2B2AE35)
    return x ^ (x >> 16)


def _random_bits(s):
    """32 random bits for every element, which depend on the seed, the step, and the element's tensor, block and place."""
    dev, blocks = s["p"].device, s["blocks"]
    tensor = torch.arange(blocks.numel(), device=dev).repeat_interleave(blocks)
    number = torch.arange(tensor.numel(), device=dev) - (blocks.cumsum(0) - blocks).repeat_interleave(blocks)
    key = torch.full_like(tensor, s["seed"])
    for part in (STEP, tensor, number):
        key = _mix((key + 0x9E3779B9) & 0xFFFFFFFF) ^ part
    key = _mix((key + 0x9E3779B9) & 0xFFFFFFFF)
    return _mix((key.unsqueeze(1) + torch.arange(256, device=dev) * 0x9E3779B9) & 0xFFFFFFFF)


def _round_8(x, bits):
    """x in [0, 448] to an 8-bit number (3 bits of mantissa, 2^-9 apart below 2^-6), up with the probability of the part that is cut
    off: bits holds 16 random ones."""
    whole = torch.floor(x * 512.0 + bits.float() / 65536.0)                                       # below 2^-6
    cut = ((x.view(torch.int32) + (bits << 4).int()) >> 20) << 20                                  # the first 3 bits of the mantissa
    return torch.where(x < 2.0 ** -6, whole / 512.0, cut.view(torch.float32))


def _adamw_plain(s):
    """Every operation rounded on its own, in the order that the operator promises."""
    p, g = s["p"].view(-1, 256), s["g"].view(-1, 256).float() * s["clip"]
    if s["bits"] == 8:
        m = s["m"].view(-1, 256).float() * s["m_scale"].unsqueeze(1)
        v = (s["v"].view(-1, 256).float() * s["v_scale"].unsqueeze(1)).square_()
    else:
        m, v = s["m"].view(-1, 256), s["v"].view(-1, 256)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * (1 - BETA2)) * g
    root = torch.sqrt(v)
    step = (m * (LR / (1 - BETA1 ** STEP))) / (root * (1 / math.sqrt(1 - BETA2 ** STEP)) + ADAM_EPS)
    n = s["decayed"]
    p = torch.cat([p[:n] * (1 - LR * DECAY), p[n:]]) - step
    del step, g
    s["p"].copy_(p.view(-1))
    out = {"p": s["p"]}
    if s["c"] is not None:
        s["c"].copy_(s["p"])
        out["c"] = s["c"]
    del p
    if s["bits"] == 32:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
        return dict(out, m=s["m"], v=s["v"])
    del v
    r = _random_bits(s)
    most = m.abs().amax(1)
    s["m_scale"].copy_((most / 448.0).clamp(min=1e-30))
    inverse = (1.0 / s["m_scale"]).unsqueeze(1)
    codes = _round_8((m.abs() * inverse).clamp(max=448.0), r & 0xFFFF)
    s["m"].copy_(torch.where(m < 0, -codes, codes).view(-1).to(E4M3))
    del m
    s["v_scale"].copy_((root.amax(1) / 448.0).clamp(min=1e-30))
    inverse = (1.0 / s["v_scale"]).unsqueeze(1)
    codes = _round_8((root * inverse).clamp(max=448.0), r >> 16)
    codes = torch.where(root > 0, codes.clamp(min=2.0 ** -9), codes)                               # a root above zero stays above zero
    s["v"].copy_(codes.view(-1).to(E4M3))
    return dict(out, m=s["m"], v=s["v"], m_scale=s["m_scale"], v_scale=s["v_scale"])


# -------------------------------------------------------------------------------------------------------------- floors

def work(case):
    op = case["op"]
    if op in ("norm", "norm_grad"):
        n, b, r, w = case["T"] * case["D"], BYTES[case["type"]], BYTES[case["sum"]], BYTES[case["weight"]]
        if op == "norm":
            out = b if case["out"] == "same" else 1
            scales = 0 if case["out"] == "same" else 4 * case["T"] * (1 if case["out"] == "row" else (case["D"] + 127) // 128)
            return {"bytes": n * (b + out + (2 * r if case["residual"] else 0)) + case["D"] * w + 4 * case["T"] + scales, "flops": 5 * n}
        return {"bytes": n * (b + 2 * r + (r if case["stream"] else 0)) + case["D"] * (w + 4) + 4 * case["T"], "flops": 9 * n}
    if op in ("head", "head_grad"):
        T, D, V, b = case["T"], case["D"], case["V"], BYTES[case["type"]]
        if op == "head":
            return {"bytes": b * (T * D + V * D) + T * (BYTES[case["ids"]] + 8), "flops": 2 * T * D * V + 4 * T * V}
        return {"bytes": 2 * b * (T * D + V * D) + T * (BYTES[case["ids"]] + (12 if case["zloss"] else 8)), "flops": 6 * T * D * V + 5 * T * V}
    n = sum(k for k, _ in _tensors(case))
    states = 16 if case["bits"] == 32 else 4 + 16 / 256
    return {"bytes": n * (8 + BYTES[case["grad"]] + states + (0 if case["copy"] == "none" else 2)), "flops": 15 * n}


# -------------------------------------------------------------------------------------------------- the definition, 64 bits

def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "norm":
        total = s["x"].double() if s["r"] is None else s["x"].double() + s["r"].double()
        out = {} if s["r"] is None else {"total": total}
        if s["r"] is not None:  # the norm is taken of the sum as it is stored
            total = total.to(s["r"].dtype).double()
        norm = torch.linalg.vector_norm(total, dim=1)
        out["rstd"] = (norm ** 2 / case["D"] + EPS) ** -0.5
        y = torch.einsum("td,t,d->td", total, out["rstd"], s["weight_"].double())
        if case["out"] == "same":
            return dict(out, y=y)
        width = case["D"] if case["out"] == "row" else 128
        pieces = y.split(width, dim=1)
        scale = torch.stack([torch.linalg.vector_norm(q, ord=float("inf"), dim=1) for q in pieces], 1) / 448
        scale = torch.maximum(scale, torch.full_like(scale, 1e-30))
        return dict(out, y_scale=scale, y=torch.cat([_nearest_8(q / scale[:, i:i + 1]) for i, q in enumerate(pieces)], 1))
    if op == "norm_grad":
        x, r, w, dy = s["total"].double(), s["rstd"].double()[:, None], s["weight_"].double(), s["dy"].double()
        # y_i = w_i x_i r with r = (mean x^2 + eps)^(-1/2), so d r / d x_j = -r^3 x_j / D
        inner = torch.einsum("td,d,td->t", dy, w, x)[:, None]
        dx = dy * w * r - inner * r ** 3 / case["D"] * x
        return {"dx": dx if s["dstream"] is None else dx + s["dstream"].double(), "dweight": torch.einsum("td,td,t->d", dy, x, r[:, 0])}
    if op in ("head", "head_grad"):
        w, t, scale, T = s["table"].double(), s["tokens"].long(), case["scale"], case["T"]
        logp, lse, dx, dw = [], [], [], torch.zeros_like(w) if op == "head_grad" else None
        for a in range(0, T, 1024):
            x, ids = s["x"][a:a + 1024].double(), t[a:a + 1024]
            n, here = x.shape[0], (ids >= 0).nonzero().squeeze(1)
            z = torch.mm(x, w.T) * scale
            if op == "head":
                lse.append(torch.logsumexp(z, 1))
                picked = z.new_zeros(n)
                picked[here] = z[here, ids[here]] - lse[-1][here]
                logp.append(picked)
                continue
            p = torch.exp(z - s["lse"][a:a + 1024, None].double())
            up = s["dlogp"][a:a + 1024].double()
            dz = torch.zeros_like(p)
            dz[here] = -up[here, None] * p[here]
            dz[here, ids[here]] += up[here]
            if s["dlse"] is not None:
                dz += s["dlse"][a:a + 1024, None].double() * p
            dx.append(scale * torch.mm(dz, w))
            dw += scale * torch.mm(dz.T, x)
        return {"logp": torch.cat(logp), "lse": torch.cat(lse)} if op == "head" else {"dx": torch.cat(dx), "dtable": dw}
    return _adamw_exact(case, s)


def _nearest_8(x):
    """The nearest 8-bit number, ties to the even one."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -9))).clamp(min=-6)
    spacing = torch.exp2(e - 3)
    return torch.round(x / spacing) * spacing


def _adamw_exact(case, s):
    g = s["g"].double().view(-1, 256) * CLIP
    m, v = s["m"].double().view(-1, 256), s["v"].double().view(-1, 256)
    if case["bits"] == 8:
        m, v = m * s["m_scale"].double()[:, None], (v * s["v_scale"].double()[:, None]) ** 2
    m, v = torch.lerp(g, m, BETA1), torch.lerp(g ** 2, v, BETA2)
    decay = torch.zeros(m.shape[0], 1, dtype=torch.float64, device=m.device)
    decay[:s["decayed"]] = DECAY
    p = s["p"].double().view(-1, 256)
    p = p - LR * (decay * p + m / (1 - BETA1 ** STEP) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + ADAM_EPS))
    out = {"p": p.view(-1)}
    if s["c"] is not None:
        out["c"] = out["p"]
    del g
    if case["bits"] == 32:
        return dict(out, m=m.view(-1), v=v.view(-1))
    r = _random_bits(s)
    for name, x, bits in (("m", m, r & 0xFFFF), ("v", v.sqrt(), r >> 16)):
        top = torch.linalg.vector_norm(x, ord=float("inf"), dim=1) / 448
        top = torch.maximum(top, torch.full_like(top, 1e-30))
        y = x.abs() / top[:, None]
        spacing = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -9))).clamp(min=-6) - 3)
        y = torch.floor(y / spacing + bits.double() / 65536) * spacing
        if name == "v":
            y = torch.where(x > 0, y.clamp(min=2.0 ** -9), y)
        out[name], out[name + "_scale"] = (torch.sign(x) * y.clamp(max=448)).view(-1), top
    return out
