"""The operators between a language model's last hidden states and its fused gradient buffer, as measurable cases.

A training step ends in a softmax cross entropy over the vocabulary, whose weight is the largest layer of the plans in
``paper_2111_08617_amd.workloads``; its gradients join those of the other layers, all of them are clipped by their
global norm, and the clipped gradients go into the fused buffer that the quantizers take.

A case is a dict of plain values:
  op       "score"   loss and log-sum-exp of every token: evaluation, or scoring of candidates while serving
           "train"   the same with the gradients of the hidden states and of the weight
           "norm"    the global l2 norm of a list of gradient tensors
           "clip"    the norm, and the clipped gradients written into one fused buffer
  score and train: tokens, width (of a hidden state), vocab, dtype, ignored (share of tokens without a target),
           scale (of the loss, as mixed-precision training has it)
  norm and clip: plan (a workload's layer table, or "generic" with n, layers, layout), dtype ("mixed": types in turn),
           odd (1: tensors start at odd elements of larger buffers), out (type of the fused buffer), clip (max_norm as a share of
           the norm of what is clipped, roughly)
"""
import math

import numpy as np
import torch

own = False
IGNORE = -100
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    def head(name, op, tokens, width, vocab, dtype, ignored=0.0, scale=1.0):
        return {"name": name, "op": op, "tokens": tokens, "width": width, "vocab": vocab, "dtype": dtype, "ignored": ignored,
                "scale": scale}

    def grads(name, op, plan, dtype, odd=0, out="f32", clip=0.5, **more):
        return {"name": name, "op": op, "plan": plan, "dtype": dtype, "odd": odd, "out": out, "clip": clip, **more}

    return [
        # the log probability of one token that a GPT-2-medium sized model has just been given: latency
        head("score_one_f16", "score", 1, 1024, 50257, "f16"),
        # a batch of decoding sequences, one token each, on the 1.3 B decoder's head
        head("score_batch_bf16", "score", 32, 2048, 50257, "bf16"),
        # perplexity of one full context of that decoder
        head("score_context_bf16", "score", 2048, 2048, 50257, "bf16"),
        # evaluation in full precision on BERT-base's vocabulary, an odd number of tokens
        head("score_bert_f32", "score", 509, 768, 30522, "f32"),
        # a small model in full precision, every size odd: ragged tiles, rows off the 16-byte grid
        head("train_odd_f32", "train", 125, 519, 1003, "f32"),
        # masked-language-model training of BERT-base: 32 sequences of 128, targets at 15 % of the places
        head("train_masked_bf16", "train", 4096, 768, 30522, "bf16", ignored=0.85),
        # four contexts of GPT-2 medium in binary16 under a loss scale
        head("train_gpt2_f16", "train", 4096, 1024, 50257, "f16", scale=4096.0),
        # the largest: four contexts of the 1.3 B decoder
        head("train_decoder_bf16", "train", 8192, 2048, 50257, "bf16"),
        # the last few small gradients of a backward pass, starting anywhere: launches count
        grads("norm_few_f32", "norm", "tiny_mixed", "f32", odd=1),
        # the gradients of GPT-2 medium in binary16: 292 tensors
        grads("norm_gpt2_f16", "norm", "gpt2_medium", "f16"),
        # a CNN's gradients, clipped into the fused buffer: 161 tensors, most of them short
        grads("clip_resnet50_f32", "clip", "resnet50", "f32"),
        # the 1.3 B decoder's bfloat16 gradients, clipped into a binary32 fused buffer
        grads("clip_decoder_bf16", "clip", "decoder_1p3b", "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("score", "train", "norm", "clip"))
    if op in ("score", "train"):
        dtype = rng.choice(("f16", "bf16", "bf16", "f32"))
        tokens, width, vocab = _log(rng, 1, 8192), _log(rng, 64, 2048), _log(rng, 512, 50257)
        if rng.random() < 0.6:
            width = max(64, width // 64 * 64)
        while tokens * width * vocab > (3e10 if dtype == "f32" else 8.4e11):       # binary32 has a twentieth of the rate
            tokens = (tokens + 1) // 2
        return {"op": op, "tokens": tokens, "width": width, "vocab": vocab, "dtype": dtype,
                "ignored": rng.choice((0.0, 0.0, 0.1, 0.5, 0.85)), "scale": 512.0 if dtype == "f16" else 1.0}
    return {"op": op, "plan": "generic", "n": _log(rng, 1 << 12, 1 << 29), "layers": _log(rng, 1, 600), "layout": rng.randrange(1 << 20),
            "dtype": rng.choice(("f32", "f16", "bf16", "mixed")), "odd": rng.choice((0, 0, 1)),
            "out": rng.choice(("f32", "f32", "f16", "bf16")), "clip": rng.choice((0.1, 0.5, 2.0))}


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """Lengths of a case's tensors: a workload's layer table (its tensors in parameter order), or log-normal ones."""
    if case["plan"] != "generic":
        return _TABLES[case["plan"]]()
    rng = np.random.default_rng([23, int(case["layout"])])
    weight = rng.lognormal(0.0, 2.0, int(case["layers"]))
    sizes = np.floor(weight / weight.sum() * int(case["n"])).astype(np.int64)
    sizes[0] += int(case["n"]) - int(sizes.sum())
    return [int(s) for s in sizes]


def _gpt2(hidden, ffn, layers, vocab, context):
    block = [hidden, hidden, 3 * hidden * hidden, 3 * hidden, hidden * hidden, hidden, hidden, hidden, hidden * ffn, ffn,
             ffn * hidden, hidden]
    return [vocab * hidden, context * hidden] + block * layers + [hidden, hidden]


def _resnet50():
    sizes, inputs = [64 * 3 * 49, 64, 64], 64
    for planes, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
        for k in range(blocks):
            sizes += [planes * inputs, planes, planes, planes * planes * 9, planes, planes, planes * planes * 4, planes * 4, planes * 4]
            sizes += [planes * 4 * inputs, planes * 4, planes * 4] if k == 0 else []
            inputs = planes * 4
    return sizes + [1000 * 2048, 1000]


#: The layer tables of paper_2111_08617_amd.workloads, as lengths.
_TABLES = {
    "tiny_mixed": lambda: [5000, 37, 0, 64, 4096 + 13, 1, 512, 159, 1000, 3, 12345, 777, 2048],
    "resnet50": _resnet50,
    "gpt2_medium": lambda: _gpt2(1024, 4096, 24, 50257, 1024),
    "decoder_1p3b": lambda: _gpt2(2048, 8192, 24, 50257, 2048),
}


def _prepare_head(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    n, h, v, dtype = int(case["tokens"]), int(case["width"]), int(case["vocab"]), TYPES[case["dtype"]]
    weight = torch.randn(v, h, device="cuda", generator=g) * 0.02
    # tokens are distributed as in text: few of them are frequent
    targets = (torch.rand(n, device="cuda", generator=g) ** 3 * v).long().clamp_(max=v - 1)
    # normalised hidden states that point towards their targets, as a partly trained model's do
    hidden = torch.randn(n, h, device="cuda", generator=g) + weight[targets] * (5.0 / (0.0004 * h)) * torch.rand(n, 1, device="cuda", generator=g)
    if case["ignored"]:
        targets[1:][torch.rand(n - 1, device="cuda", generator=g) < case["ignored"]] = IGNORE
    counted = (targets != IGNORE).sum().clamp(min=1)
    dloss = torch.full((n,), float(case["scale"]), device="cuda") / counted
    out = {"case": case, "hidden": hidden.to(dtype), "weight": weight.to(dtype), "targets": targets, "dloss": dloss,
           "loss": torch.empty(n, device="cuda"), "lse": torch.empty(n, device="cuda")}
    if case["op"] == "train":
        out["dhidden"], out["dweight"] = torch.empty_like(out["hidden"]), torch.empty_like(out["weight"])
    return out


def _prepare_grads(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    lengths, types = _lengths(case), {"mixed": ("f32", "bf16", "f16")}.get(case["dtype"], (case["dtype"],))
    scales = (10.0 ** np.random.default_rng([29, int(seed)]).uniform(-4.0, -1.0, len(lengths))).tolist()   # a scale for each tensor
    total = sum(lengths)
    noise = torch.randn(min(total, 1 << 24) + 64, device="cuda", generator=g)
    grads, at = [], int(seed) % 17
    for k, (n, scale) in enumerate(zip(lengths, scales)):
        dtype = TYPES[types[k % len(types)]]
        buffer = torch.empty(n + 1, dtype=dtype, device="cuda")
        one = buffer[1:] if case["odd"] else buffer[:n]
        done = 0
        while done < n:
            at = at if at < noise.numel() else 0
            take = min(n - done, noise.numel() - at)
            one[done:done + take] = noise[at:at + take] * scale
            done, at = done + take, at + take
        grads.append(one)
    size = math.sqrt(sum(n * s * s for n, s in zip(lengths, scales)))
    out = {"case": case, "grads": grads, "max_norm": float(np.float32(case["clip"] * size)), "norm": torch.empty(1, device="cuda")}
    if case["op"] == "clip":
        out["fused"] = torch.empty(total, dtype=TYPES[case["out"]], device="cuda")
    return out


def prepare(case, seed):
    return (_prepare_head if case["op"] in ("score", "train") else _prepare_grads)(case, seed)


# ------------------------------------------------------------------ plain forms

def _plain_head(s):
    hidden, weight, targets = s["hidden"].float(), s["weight"].float(), s["targets"]
    counts = targets != IGNORE
    at = torch.where(counts, targets, 0)[:, None]
    z = hidden @ weight.t()
    top = z.max(dim=1, keepdim=True).values
    lse = top + torch.exp(z - top).sum(dim=1, keepdim=True).log()
    loss = torch.where(counts, (lse - z.gather(1, at))[:, 0], 0.0)
    out = {"loss": loss, "lse": torch.where(counts, lse[:, 0], 0.0)}
    if s["case"]["op"] == "train":
        d = torch.exp(z - lse)
        d.scatter_add_(1, at, torch.full_like(lse, -1.0))
        d = torch.where(counts[:, None], d * s["dloss"][:, None], 0.0)
        out["dhidden"] = (d @ weight).to(s["hidden"].dtype)
        out["dweight"] = (d.t() @ torch.where(counts[:, None], hidden, 0.0)).to(s["weight"].dtype)
    return out


def _plain_grads(s):
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt().reshape(1)
    if s["case"]["op"] == "norm":
        return {"norm": norm}
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    return {"norm": norm, "fused": torch.cat([(g.float() * factor).to(s["fused"].dtype) for g in s["grads"]])}


# ------------------------------------------------------------------ the framework's calls

def _own_head(s):
    from paper_2111_08617_amd import binding as cgx
    grad = s["case"]["op"] == "train"
    if "workspace" not in s:
        n, h = s["hidden"].shape
        size = cgx.cgx_head_workspace(n, h, s["weight"].shape[0], {"f32": cgx.F32, "f16": cgx.F16, "bf16": cgx.BF16}[s["case"]["dtype"]], grad)
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    cgx.cgx_head_loss(s["hidden"], s["weight"], s["targets"], s["loss"], s["lse"], s["workspace"], ignore=IGNORE)
    if not grad:
        return {"loss": s["loss"], "lse": s["lse"]}
    cgx.cgx_head_loss_grad(s["hidden"], s["weight"], s["targets"], s["lse"], s["dloss"], s["dhidden"], s["dweight"], s["workspace"],
                           ignore=IGNORE)
    return {"loss": s["loss"], "lse": s["lse"], "dhidden": s["dhidden"], "dweight": s["dweight"]}


def _own_grads(s):
    from paper_2111_08617_amd import binding as cgx
    if "workspace" not in s:
        s["workspace"] = torch.empty(cgx.cgx_grad_norm_workspace(), dtype=torch.uint8, device="cuda")
    cgx.cgx_grad_norm(s["grads"], s["norm"], s["workspace"])
    if s["case"]["op"] == "norm":
        return {"norm": s["norm"]}
    cgx.cgx_grad_clip(s["grads"], s["norm"], s["max_norm"], out=s["fused"])
    return {"norm": s["norm"], "fused": s["fused"]}


def run(state):
    if state["case"]["op"] in ("score", "train"):
        return (_own_head if own else _plain_head)(state)
    return (_own_grads if own else _plain_grads)(state)


# ------------------------------------------------------------------ what a pass needs, and its exact results

def work(case):
    if case["op"] in ("score", "train"):
        n, h, v, size = case["tokens"], case["width"], case["vocab"], SIZES[case["dtype"]]
        counted = max(1, round(n * (1.0 - case["ignored"])))          # tokens without a target need no products
        read = (counted * h + v * h) * size + n * 8
        if case["op"] == "score":
            return {"bytes": read + n * 8, "flops": 2 * counted * v * h}
        # logits, and both products of the gradient: what has to be computed, were the logits kept
        return {"bytes": read + n * 12 + (n * h + v * h) * size, "flops": 6 * counted * v * h}
    lengths, types = _lengths(case), {"mixed": ("f32", "bf16", "f16")}.get(case["dtype"], (case["dtype"],))
    read = sum(n * SIZES[types[k % len(types)]] for k, n in enumerate(lengths))
    if case["op"] == "norm":
        return {"bytes": read + 4, "flops": 2 * sum(lengths)}
    return {"bytes": read + sum(lengths) * SIZES[case["out"]] + 4, "flops": 3 * sum(lengths)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "clip"):
        squares = [float(torch.dot(part, part)) for g in s["grads"] for part in (p.double() for p in g.split(1 << 26)) if g.numel()]
        norm = math.sqrt(math.fsum(squares))
        out = {"norm": torch.tensor([norm], dtype=torch.float64, device="cuda")}
        if case["op"] == "clip":
            fused, at = torch.empty(s["fused"].numel(), dtype=torch.float64, device="cuda"), 0
            for g in s["grads"]:
                fused[at:at + g.numel()] = g
                at += g.numel()
            out["fused"] = fused.mul_(min(1.0, s["max_norm"] / norm) if norm else 1.0)
        return out
    weight, n = s["weight"].double(), int(case["tokens"])
    loss, lse = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    dhidden, dweight = torch.zeros(n, int(case["width"]), dtype=torch.float64, device="cuda"), torch.zeros_like(weight)
    rows = torch.nonzero(s["targets"] != IGNORE)[:, 0]
    for part in rows.split(1024):
        x, t = s["hidden"][part].double(), s["targets"][part]
        logp = torch.log_softmax(torch.mm(x, weight.t()), dim=1)
        loss[part] = -logp[torch.arange(len(part), device="cuda"), t]
        lse[part] = loss[part] + (x * weight[t]).sum(dim=1)
        if case["op"] == "train":
            p, g = logp.exp_(), s["dloss"][part].double()[:, None]
            dhidden[part] = g * (torch.mm(p, weight) - weight[t])
            dweight += torch.mm((g * p).t().contiguous(), x)
            dweight.index_add_(0, t, -g * x)
    out = {"loss": loss, "lse": lse}
    return {**out, "dhidden": dhidden, "dweight": dweight} if case["op"] == "train" else out
