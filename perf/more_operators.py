"""Fitting an acoustic model's output layer and holding it in four bits, case by
case.

The layer that Head.project computes, W x[n] + b, with up to 100000 labels:

loss      cross entropy of rows against their labels, straight from the hidden
          rows and the weights: loss[n] = log sum exp z[n] - z[n][target[n]],
          z = W x + b.  Rows whose target is no label (padding, frames that a
          first pass is not sure of) have loss 0.
grads     the same with the gradients of the rows, weights and bias for the
          gradient g[n] of each row's loss.
clip      the norm over many tensors' gradients, and the gradients times
          min(1, max_norm / norm), into other tensors (an optimizer's).
quantize  a matrix to microscaled 4-bit floating point: blocks of 32 values of a
          row share a power of two, 2^(floor(log2 max) - 2), and each is 0, 0.5, 1,
          1.5, 2, 3, 4 or 6 times it, with a sign (round to nearest, ties to the
          even code, more than 6 to 6); and the values that it stands for.
project4  out[n] = Wq q(x[n]) + b: a layer whose weights are held so, of rows that
          the call brings to that form.

A case is one call of one of them (quantize: and the values read back).  `own`
chooses between the plain forms here (elementary tensor operations in 32 bits)
and the framework's kernels.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _loss(name, N, D, P, dtype, grads, without):
    """N rows, a share `without` of them without a label."""
    return dict(name=name, op="grads" if grads else "loss", N=N, D=D, P=P, dtype=dtype, without=without)


def _clip(name, tensors, total, dtype, out, clipped):
    """`tensors` gradients of `total` values in all; `clipped`: whether their norm is above the largest allowed."""
    return dict(name=name, op="clip", tensors=tensors, total=total, dtype=dtype, out=out, clipped=clipped)


def _quantize(name, N, D, dtype):
    return dict(name=name, op="quantize", N=N, D=D, dtype=dtype)


def _project4(name, N, D, P, dtype, out):
    return dict(name=name, op="project4", N=N, D=D, P=P, dtype=dtype, out=out)


def listed():
    return [
        # how well a live stream's newest frame fits the label that it was decoded to: the smallest call
        _loss("loss_frame", 1, 512, 500, "bf16", False, 0.0),
        # held-out loss of 32 whole utterances
        _loss("loss_batch", 32_000, 1024, 6000, "bf16", False, 0.05),
        # a step on a few ragged utterances through a layer of odd sizes, in half precision
        _loss("grads_odd", 777, 1000, 3001, "f16", True, 0.1),
        # a step on 64 chunks of a second of audio, labels from a first pass
        _loss("grads_chunks", 2048, 1024, 6000, "bf16", True, 0.1),
        # a step of a word layer
        _loss("grads_words", 4096, 1024, 100_000, "bf16", True, 0.02),
        # a speaker's adapter and the bias
        _clip("clip_adapter", 3, 118_000, "f32", "f32", True),
        # a whole acoustic model, 16-bit gradients into the optimizer's 32-bit ones
        _clip("clip_model", 300, 250_000_000, "bf16", "f32", True),
        # a word layer's weights, once per model
        _quantize("quantize_words", 100_000, 1024, "bf16"),
        # a frame of one spoken command
        _project4("project4_frame", 1, 512, 500, "bf16", "f32"),
        # a frame of each of 64 live streams, a word layer
        _project4("project4_live", 64, 1024, 100_000, "bf16", "f32"),
        # a few ragged utterances through a layer of odd sizes
        _project4("project4_odd", 900, 1000, 3001, "f16", "f32"),
        # offline transcription: 64 whole utterances
        _project4("project4_batch", 64_000, 1024, 6000, "bf16", "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["loss", "grads", "grads", "clip", "quantize", "project4", "project4"])
    dtype = rng.choice(["bf16", "f16"])
    D = _log_int(rng, 64, 1536)
    if rng.random() < 0.6:  # most layers are multiples of eight, as the listed ones
        D = D // 8 * 8
    if op in ("loss", "grads"):
        P = _log_int(rng, 100, 100_000)
        N = _log_int(rng, 1, 32_000)
        while N * D * P > 4096 * 1024 * 100_000:  # no dearer than the largest listed one
            N = max(1, N // 2)
        c = _loss("", N, D, P, dtype, op == "grads", rng.choice([0.0, 0.1, 0.5]))
    elif op == "clip":
        tensors = _log_int(rng, 1, 600)
        c = _clip("", tensors, tensors + _log_int(rng, 1000, 200_000_000), *rng.choice(
            [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32")]), rng.random() < 0.7)
    elif op == "quantize":
        c = _quantize("", _log_int(rng, 1, 60_000), D, rng.choice(["bf16", "f16", "f32"]))
    else:
        P = _log_int(rng, 100, 100_000)
        N = _log_int(rng, 1, 64_000)
        while N * P > 64_000 * 6000:
            N = max(1, N // 2)
        c = _project4("", N, D, P, dtype, rng.choice(["f32", dtype]))
    return {k: v for k, v in c.items() if k != "name"}


# ------------------------------------------------------------------ inputs

def _normal(gen, shape, std, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device=DEVICE).mul_(std).to(dtype)


def _prepare_loss(case, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    N, D, P, dtype = case["N"], case["D"], case["P"], TYPES[case["dtype"]]
    weight = _normal(gen, (P, D), 2.5 / math.sqrt(D))
    target = torch.randint(0, P, (N,), generator=gen, device=DEVICE)
    # behind a layer norm, and towards the label by as much as a model that is half sure of it
    x = _normal(gen, (N, D), 1.0) + 4.5 / 2.5 * weight[target]
    rows = torch.rand(N, generator=gen, device=DEVICE)
    s = dict(op=case["op"], x=x.to(dtype), weight=weight.to(dtype), bias=_normal(gen, (P,), 1.0),
             target=torch.where(rows < case["without"], torch.full_like(target, -1), target).int())
    if case["op"] == "grads":  # the frames' confidences, over their number
        s["grad"] = (0.5 + 0.5 * torch.rand(N, generator=gen, device=DEVICE)) / N
    return s


def _sizes(case):
    """Values of each tensor: of all sizes, `total` together; they belong to the case."""
    share = np.exp(np.random.default_rng([case["tensors"], 7]).uniform(0, 6, case["tensors"]))
    sizes = np.maximum(1, (share / share.sum() * case["total"]).astype(np.int64))
    sizes[-1] += max(0, case["total"] - int(sizes.sum()))
    return sizes.tolist()


def _prepare_clip(case, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    sizes = _sizes(case)
    stds = np.exp(np.random.default_rng([seed, 1]).normal(-6.0, 1.0, len(sizes)))
    grads = [_normal(gen, (n,), float(s), TYPES[case["dtype"]]) for n, s in zip(sizes, stds)]
    flat = torch.empty(sum(sizes), dtype=TYPES[case["out"]], device=DEVICE)  # the optimizer's
    norm = math.sqrt(sum(n * float(s) ** 2 for n, s in zip(sizes, stds)))
    return dict(op="clip", grads=grads, flat=flat, out=list(flat.split(sizes)), max_norm=norm * (0.4 if case["clipped"] else 2.5))


def _prepare_quantize(case, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    size = torch.exp(_normal(gen, (case["N"], 1), 0.5))  # rows of different sizes
    return dict(op="quantize", x=(_normal(gen, (case["N"], case["D"]), 2.5 / math.sqrt(case["D"])) * size).to(TYPES[case["dtype"]]))


def _prepare_project4(case, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    D, dtype = case["D"], TYPES[case["dtype"]]
    s = dict(op="project4", x=_normal(gen, (case["N"], D), 1.0, dtype), bias=_normal(gen, (case["P"],), 1.0), out=TYPES[case["out"]])
    weight = _normal(gen, (case["P"], D), 2.5 / math.sqrt(D), dtype)
    # the layer as a program holds it
    if own:
        from paper_1804_03243_amd import wfstdec
        s["head"] = wfstdec.MicroHead(wfstdec.micro(weight), s["bias"])
    else:
        s["weight"] = _plain_micro(weight)
    return s


def prepare(case, seed):
    s = {"loss": _prepare_loss, "grads": _prepare_loss, "clip": _prepare_clip, "quantize": _prepare_quantize,
         "project4": _prepare_project4}[case["op"]](case, seed)
    if own:
        from paper_1804_03243_amd import wfstdec
        s["wf"] = wfstdec
    return s


# ------------------------------------------------------------- plain forms

def _plain_loss(s):
    x, w, t = s["x"].float(), s["weight"].float(), s["target"].long()
    z = x @ w.T + s["bias"]
    at = torch.arange(len(t), device=z.device)
    has = t >= 0
    label = torch.where(has, t, torch.zeros_like(t))
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    loss = torch.where(has, (top + total.log())[:, 0] - z[at, label], torch.zeros((), device=z.device))
    if s["op"] == "loss":
        return loss
    dz = e / total
    dz[at, label] -= 1.0
    dz *= torch.where(has, s["grad"], torch.zeros((), device=z.device))[:, None]
    return loss, (dz @ w).to(s["x"].dtype), (dz.T @ x).to(s["x"].dtype), dz.sum(0)


def _plain_clip(s):
    total = torch.zeros((), dtype=torch.float64, device=DEVICE)
    for g in s["grads"]:
        total += g.double().square().sum()
    norm = total.sqrt()
    factor = torch.clamp(s["max_norm"] / norm, max=1.0).float()
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * factor)
    return norm.float(), s["flat"]


def _plain_micro(x):
    """The values in 32 bits that a matrix's microscaled form stands for."""
    N, D = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -D % 32)).view(N, -1, 32)
    top = x.abs().amax(2, keepdim=True)
    power = torch.where(top > 0, torch.frexp(top).exponent - 3, 0).clamp(-126, 126)  # floor(log2 top) - 2
    unit = ((power + 127) << 23).view(torch.float32)  # 2^power
    y = x / unit
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    y = torch.clamp(torch.round(y / step) * step, -6.0, 6.0)
    return (y * unit).view(N, -1)[:, :D]


def _plain_project4(s):
    return (_plain_micro(s["x"]) @ s["weight"].T + s["bias"]).to(s["out"])


# ------------------------------------------------------------------- passes

def run(s):
    if not own:
        if s["op"] == "quantize":
            return _plain_micro(s["x"]).to(torch.bfloat16)
        return {"loss": _plain_loss, "grads": _plain_loss, "clip": _plain_clip, "project4": _plain_project4}[s["op"]](s)
    wf = s["wf"]
    if s["op"] == "loss":
        return wf.cross_entropy(s["x"], s["weight"], s["target"], s["bias"])
    if s["op"] == "grads":
        return wf.cross_entropy_grads(s["x"], s["weight"], s["target"], s["bias"], s["grad"])
    if s["op"] == "clip":
        return wf.clip_gradients(s["grads"], s["max_norm"], out=s["out"]), s["flat"]
    if s["op"] == "quantize":
        return wf.micro(s["x"]).values()
    return s["head"].project(s["x"], out_dtype=s["out"])


def work(case):
    """Every input once, every output once."""
    size = {"f32": 4, "f16": 2, "bf16": 2}
    e = size[case["dtype"]]
    if case["op"] == "clip":
        n = sum(_sizes(case))
        return {"bytes": n * (e + size[case["out"]]) + 4, "flops": 3 * n}
    N, D = case["N"], case["D"]
    if case["op"] == "quantize":  # the codes are written, and read for the values
        return {"bytes": N * D * (e + 2 * 17 / 32 + 2), "flops": 4 * N * D}
    P = case["P"]
    if case["op"] == "project4":
        return {"bytes": N * D * e + P * D * 17 / 32 + 4 * P + N * P * size[case["out"]], "flops": 2 * N * D * P}
    if case["op"] == "loss":
        return {"bytes": (N + P) * D * e + 4 * P + 8 * N, "flops": 2 * N * D * P}
    return {"bytes": 2 * (N + P) * D * e + 8 * P + 12 * N, "flops": 6 * N * D * P}


# ------------------------------------------------------------ in 64 bits

def exact(case, seed):
    """The same outputs from the definitions, in 64 bits."""

    def micro(x):
        """Each value to the nearest of the 15 that its block has, ties to the even code."""
        codes = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEVICE)
        between = (codes[1:] + codes[:-1]) / 2
        out = torch.zeros(x.shape, dtype=torch.float64, device=DEVICE)
        for c in range(0, x.shape[1], 32):
            v = x[:, c:c + 32].double()
            top = v.abs().amax(1, keepdim=True)
            mantissa = torch.tensor((1 << 52) - 1, device=DEVICE)
            unit = torch.where(top > 0, (top.view(torch.int64) & ~mantissa).view(torch.float64) / 4, 1.0)
            y = v.abs() / unit
            low = torch.bucketize(y, between)               # borders belong to the code below them
            high = torch.bucketize(y, between, right=True)  # and here to the one above
            out[:, c:c + 32] = torch.sign(v) * codes[torch.where(low % 2 == 0, low, high)] * unit
        return out

    if case["op"] == "quantize":
        return micro(_prepare_quantize(case, seed)["x"])
    if case["op"] == "clip":
        s = _prepare_clip(case, seed)
        flat = torch.cat([g.double() for g in s["grads"]])
        norm = torch.linalg.vector_norm(flat)
        return norm, flat * torch.clamp(s["max_norm"] / norm, max=1.0)
    if case["op"] == "project4":
        gen = torch.Generator(DEVICE).manual_seed(seed)
        D, dtype = case["D"], TYPES[case["dtype"]]  # (as prepare makes them)
        x = _normal(gen, (case["N"], D), 1.0, dtype)
        bias = _normal(gen, (case["P"],), 1.0)
        weight = _normal(gen, (case["P"], D), 2.5 / math.sqrt(D), dtype)
        return torch.addmm(bias.double(), micro(x), micro(weight).T)
    s = _prepare_loss(case, seed)
    x, w = s["x"].double(), s["weight"].double()
    z = torch.addmm(s["bias"].double(), x, w.T)
    has = s["target"] >= 0
    logp = torch.log_softmax(z, 1)
    label = s["target"].clamp(min=0).long()[:, None]
    loss = -logp.gather(1, label)[:, 0] * has
    if case["op"] == "loss":
        return loss
    dz = logp.exp().scatter_add_(1, label, -torch.ones(label.shape, dtype=torch.float64, device=DEVICE))
    dz *= (s["grad"].double() * has)[:, None]
    return loss, dz @ w, dz.T @ x, dz.sum(0)
