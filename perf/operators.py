"""Performance cases of the operators between a model's tensors and THC's flat vectors: the global norm of a gradient that
is held as many tensors, clipping by it, gathering the tensors into the padded vector that is compressed, scattering the
estimate back.  Four kinds of use, and the first and third together:

  norm     thc_grad_norm: the norm and the factor that clips by it
  clip     thc_grad_clip: the same, and the tensors scaled in place
  gather   thc_gather: tensors -> padded vector, with a factor from device memory
  scatter  thc_scatter: the estimate -> tensors, with a factor
  step     thc_grad_norm, then thc_gather with its factor: what a worker does before thc_compress

A case is a dict of plain values.  `layout` seeds the tensors' sizes: every second tensor is a short vector (a bias or a
norm's weight), the others share the rest.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _case(kind, count, total, dtype="f32", packed=False, norm="l2", clips=True, out="f32", log2_block=20, layout=1):
    c = {"kind": kind, "count": count, "total": total, "dtype": dtype, "packed": packed, "layout": layout}
    if kind in ("norm", "clip", "step"):
        c.update(norm=norm, clips=clips)
    if kind in ("gather", "step"):
        c.update(out=out)
    if kind in ("gather", "scatter", "step"):
        c.update(log2_block=log2_block)
    return c


def listed():
    def named(name, *a, **k):
        return dict(_case(*a, **k), name=name)

    return [
        # one bias: nothing but latency
        named("norm_bias", "norm", 1, 1600),
        # GPT-2-XL-shaped list of bf16 gradients, the largest norm
        named("norm_gpt2_xl", "norm", 580, 1_557_611_200, dtype="bf16"),
        # BERT-large-shaped list of loss-scaled f16 gradients: largest magnitude, as a check for overflow takes it
        named("norm_max_bert", "norm", 391, 336_000_000, dtype="f16", norm="max", clips=False),
        # a classifier's head, odd sizes one after another in one buffer: the smallest clipping
        named("clip_head", "clip", 5, 20_011, packed=True),
        # VGG16-shaped list, binary32: few and large tensors
        named("clip_vgg16", "clip", 32, 138_357_544),
        # BERT-large-shaped list, bf16 matrices and binary32 vectors, without gaps: starts on any element
        named("clip_bert_mixed", "clip", 391, 336_000_000, dtype="mixed", packed=True),
        # ResNet-50-shaped list in bf16 whose norm is below the limit, as in most steps of a run
        named("clip_below_limit", "clip", 161, 25_557_032, dtype="bf16", clips=False),
        # a small bucket of odd bf16 tensors widened into the vector of two blocks of 2^14
        named("gather_bucket_2p15", "gather", 12, 30_011, dtype="bf16", packed=True, log2_block=14),
        # GPT-2-XL-shaped list into its padded bf16 vector: the largest call
        named("gather_gpt2_xl", "gather", 580, 1_557_611_200, dtype="bf16", out="bf16", log2_block=22),
        # ResNet-50-shaped list: norm, then the clipped gradient as one block of 2^25
        named("step_resnet50", "step", 161, 25_557_032, log2_block=25),
        # VGG16-shaped estimate back to binary32 tensors
        named("scatter_vgg16", "scatter", 32, 138_357_544),
        # BERT-large-shaped estimate to f16 tensors that start on any element
        named("scatter_bert_f16", "scatter", 391, 336_000_000, dtype="f16", packed=True),
    ]


def draw(rng):
    kind = rng.choices(("norm", "clip", "gather", "scatter", "step"), (3, 3, 2, 2, 2))[0]
    dtype = rng.choice(("f32", "f32", "bf16", "bf16", "f16", "mixed"))
    total = max(1, int(2.0 ** rng.uniform(6.0, 29.0 if dtype in ("f32", "mixed") else 30.0)))
    count = max(1, min(total // 4, int(2.0 ** rng.uniform(0.0, 9.6))))
    log2_block = rng.choice((10, 12, 14, 16, 18, 20, 20, 20, 22))
    while log2_block > 10 and 1 << log2_block > 2 * total:
        log2_block -= 1
    return _case(kind, count, total, dtype, rng.random() < 0.4, "max" if rng.random() < 0.25 else "l2", rng.random() < 0.7,
                 rng.choice(("f32", "f32", "bf16")), log2_block, rng.randrange(1 << 16))


def _sizes(case):
    """Elements of each tensor: `count` positive numbers that add up to `total`."""
    count, total, rng = case["count"], case["total"], random.Random(case["layout"])
    short = [min(rng.choice((64, 250, 256, 512, 1000, 1024, 1600, 2048)), max(1, total // (2 * count))) for _ in range(count // 2)]
    weights = [math.exp(rng.gauss(0.0, 1.0)) for _ in range(count - count // 2)]
    rest = total - sum(short) - len(weights)
    long = [1 + int(rest * w / sum(weights)) for w in weights]
    long[0] += total - sum(short) - sum(long)
    sizes = [0] * count
    sizes[::2], sizes[1::2] = long, short
    return sizes


def _padded(case):
    block = 1 << case["log2_block"]
    return -(-case["total"] // block) * block


def prepare(case, seed):
    kind, gen = case["kind"], torch.Generator(device=DEV).manual_seed(seed)
    sizes = _sizes(case)
    # a tensor's own type, and its place in that type's buffer: without gaps, or on 128 elements as an allocator has them
    types = [("bf16", "f32")[i % 2] if case["dtype"] == "mixed" else case["dtype"] for i in range(len(sizes))]
    at, end = [], {}
    for n, t in zip(sizes, types):
        at.append(end.get(t, 0))
        end[t] = at[-1] + (n if case["packed"] else -(-n // 128) * 128)
    buffers = {t: torch.zeros(n, dtype=TYPES[t], device=DEV) for t, n in end.items()}
    tensors = [buffers[t][a:a + n] for t, a, n in zip(types, at, sizes)]
    s = {"kind": kind, "sizes": sizes, "tensors": tensors, "buffers": [buffers[t] for t in sorted(buffers)]}
    if kind != "scatter":
        for t, x in buffers.items():             # layers of different scales; f16 gradients carry a loss scale of 1024
            x.normal_(generator=gen)
            for k in range(8):
                part = x[x.numel() * k // 8:x.numel() * (k + 1) // 8]
                part.mul_(1e-3 * 10.0 ** (-1.0 + 2.0 * ((5 * k) % 8) / 7.0) * (1024.0 if t == "f16" else 1.0))
    if kind in ("norm", "clip", "step"):
        # the program's limit: three tenths of this gradient's norm, or four times it
        parts = torch.stack([x.double().square().sum() if case["norm"] == "l2" else x.double().abs().max() for x in tensors])
        v = float(parts.sum().sqrt() if case["norm"] == "l2" else parts.max())
        s.update(norm_kind=case["norm"], limit=v * (0.3 if case["clips"] else 4.0))
        s.update(norm=torch.empty(1, device=DEV), scale=torch.empty(1, device=DEV), ws=torch.empty(1 << 20, dtype=torch.uint8, device=DEV))
        s["next"] = 0.9999 if case["clips"] else 1.0   # the limit sinks a little, so that a clipped gradient is clipped again
    if kind in ("gather", "scatter", "step"):
        d = _padded(case)
        s.update(d=d, block=1 << case["log2_block"])
        if kind != "step":
            s["scale"] = torch.rand(1, generator=gen, device=DEV) * 0.5 + 0.25
        if kind == "scatter":
            s["flat"] = torch.zeros(d, device=DEV)
            s["flat"][:case["total"]].normal_(generator=gen).mul_(1e-2)
        else:
            s["flat"] = torch.empty(d, dtype=TYPES[case["out"]], device=DEV)
    return s


# ---------------------------------------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2302_08545_amd import api
    kind = s["kind"]
    if "list" not in s:          # a program describes its tensors once, as long as they stay where they are
        s["list"] = api.make_tensors(s["tensors"])
        if kind in ("gather", "scatter", "step"):
            s["P"] = api.make_params(s["d"], s["block"], 1, 4, 15, 2.0, 7, range(16),
                                     in_dtype=api.THC_DTYPE_BF16 if s["flat"].dtype == torch.bfloat16 else api.THC_DTYPE_F32)
    if kind == "gather":
        api.thc_gather(s["P"], s["list"], s["scale"], s["flat"])
        return {"flat": s["flat"]}
    if kind == "scatter":
        api.thc_scatter(s["P"], s["flat"], s["scale"], s["list"])
        return {"buffers": s["buffers"]}
    how = api.THC_NORM_L2 if s["norm_kind"] == "l2" else api.THC_NORM_MAX
    if kind == "clip":
        api.thc_grad_clip(s["list"], how, s["limit"], s["norm"], s["scale"], s["ws"])
        s["limit"] *= s["next"]
        return {"norm": s["norm"], "scale": s["scale"], "buffers": s["buffers"]}
    api.thc_grad_norm(s["list"], how, s["limit"], s["norm"], s["scale"], s["ws"])
    if kind == "norm":
        return {"norm": s["norm"], "scale": s["scale"]}
    api.thc_gather(s["P"], s["list"], s["scale"], s["flat"])
    return {"norm": s["norm"], "scale": s["scale"], "flat": s["flat"]}


# ---------------------------------------------------------------------------------------------- the plain form
def _joined(s):
    return torch.cat(s["tensors"]).float()


def _norm(s, x):
    v = (x * x).sum(dtype=torch.float64).sqrt() if s["norm_kind"] == "l2" else x.abs().max().double()
    scale = torch.where(v <= s["limit"], torch.ones_like(v), s["limit"] / v)
    return v.float().reshape(1), scale.float().reshape(1)


def _spread(s, x):
    return [t.copy_(part) for t, part in zip(s["tensors"], x.split(s["sizes"]))]


def _flat(s, x, scale):
    s["flat"][:x.numel()] = x * scale
    s["flat"][x.numel():] = 0
    return s["flat"]


def run(s):
    if own:
        return _own(s)
    kind = s["kind"]
    if kind == "scatter":
        _spread(s, s["flat"][:sum(s["sizes"])] * s["scale"])
        return {"buffers": s["buffers"]}
    x = _joined(s)
    if kind == "gather":
        return {"flat": _flat(s, x, s["scale"])}
    norm, scale = _norm(s, x)
    if kind == "clip":
        _spread(s, x * scale)
        s["limit"] *= s["next"]
        return {"norm": norm, "scale": scale, "buffers": s["buffers"]}
    if kind == "norm":
        return {"norm": norm, "scale": scale}
    return {"norm": norm, "scale": scale, "flat": _flat(s, x, scale)}


def work(case):
    """Every input once and every output once.  A gradient below its limit is read only."""
    sizes = _sizes(case)
    if case["dtype"] == "mixed":
        tensors = sum(sizes[::2]) * BYTES["bf16"] + sum(sizes[1::2]) * BYTES["f32"]
    else:
        tensors = case["total"] * BYTES[case["dtype"]]
    kind, n = case["kind"], case["total"]
    flat = {"scatter": 4 * n}.get(kind, _padded(case) * BYTES[case["out"]] if "out" in case else 0)
    written = tensors if kind == "clip" and case["clips"] else 0
    flops = {"norm": 2, "clip": 3 if written else 2, "step": 3}.get(kind, 1)
    return {"bytes": tensors + written + flat + 8, "flops": flops * n}


def exact(case, seed):
    """The definitions in 64 bits, tensor by tensor."""
    s = prepare(case, seed)
    wide = [t.double() for t in s["tensors"]]
    kind, found = case["kind"], {}
    if kind in ("norm", "clip", "step"):
        if case["norm"] == "l2":
            v = math.sqrt(math.fsum(float(torch.dot(w, w)) for w in wide))
        else:
            v = max(float(torch.maximum(w.max(), -w.min())) for w in wide)
        c = 1.0 if v <= s["limit"] else s["limit"] / v
        found = {"norm": torch.tensor([v], dtype=torch.float64), "scale": torch.tensor([c], dtype=torch.float64)}
    else:
        c = float(s["scale"])
    if kind in ("gather", "step"):
        flat = torch.zeros(s["d"], dtype=torch.float64, device=DEV)
        pos = 0
        for w in wide:
            torch.mul(w, c, out=flat[pos:pos + w.numel()])
            pos += w.numel()
        found["flat"] = flat
    if kind in ("clip", "scatter"):
        pos = 0
        buffers = {b.data_ptr(): b.double() for b in s["buffers"]}
        for t, w in zip(s["tensors"], wide):
            base = next(b for b in s["buffers"] if b.dtype == t.dtype)
            a = (t.data_ptr() - base.data_ptr()) // t.element_size()
            src = w if kind == "clip" else s["flat"][pos:pos + w.numel()].double()
            buffers[base.data_ptr()][a:a + w.numel()] = src * c
            pos += w.numel()
        found["buffers"] = [buffers[b.data_ptr()] for b in s["buffers"]]
    return found
