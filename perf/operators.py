"""The gradient norm, clipping and AdamW over a model's many tensors: the cases they are measured by.

A training step ends with three operators on the gradients that the aggregation (or a
backward pass) left: their global norm, their clipping by it, and the update of the
parameters.  Cases differ in the tensors' number, lengths, types and addresses: padded
buffers of one tensor each, or views of one flat buffer at any element address, as the
aggregated gradient of a round is cut into a model's tensors.
"""
from __future__ import annotations

import math
import random

import torch

own = False

LR, BETAS, EPS, DECAY = 3e-4, (0.9, 0.95), 1e-8, 0.1
CLIP_EPS = 1e-6                       # added to the norm under the clipping quotient
STEP = 1000                           # optimizer steps behind the state that a case begins with
LOSS_SCALE = 1024.0                   # fp16 gradients come multiplied by it
MOST_VALUES = 1.15e9                  # of the largest listed case
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


def _case(name, op, model, grad="fp32", **more):
    return dict({"name": name, "op": op, "model": model, "grad": grad, "packed": False}, **more)


def listed():
    blocks_1b = {"layers": 16, "width": 2048, "hidden": 8192, "vocab": 32_000}
    blocks_230m = {"layers": 12, "width": 1024, "hidden": 4096, "vocab": 32_000}
    return [
        # a toy model's six tensors (the 4,096 values of the smallest round): latency
        _case("norm_toy", "norm", "toy"),
        # the flat gradient that a round aggregated, cut into a ResNet-18's 62 tensors
        _case("norm_resnet18", "norm", "resnet18", packed=True),
        # a language model of 1.1 billion parameters in bf16, most rows of the embedding's gradient zero
        _case("norm_1b_bf16", "norm", "blocks", "bf16", **blocks_1b),
        # low-rank factors of a fine-tuned model: 256 small tensors, clipped into a second buffer
        _case("clip_adapters_bf16", "clip", "adapters", "bf16", out="bf16", clipped=True, inplace=False,
              layers=32, width=2048, rank=16),
        # the round's flat gradient, clipped into buffers of the tensors' own
        _case("clip_resnet18", "clip", "resnet18", out="fp32", clipped=True, inplace=False, packed=True),
        # bf16 gradients clipped into the fp32 buffers that an accumulation or a reduction reads
        _case("clip_230m_bf16_fp32", "clip", "blocks", "bf16", out="fp32", clipped=True, inplace=False,
              **blocks_230m),
        # the ordinary step of a run that has settled: the norm stays below the bound, in place
        _case("clip_230m_below", "clip", "blocks", out="fp32", clipped=False, inplace=True, **blocks_230m),
        # tensors of every length from 0 to millions at odd addresses, fp16 under a loss scale
        _case("clip_ragged_fp16", "clip", "ragged", "fp16", out="fp16", clipped=True, inplace=False, packed=True,
              count=301, longest=4_000_001),
        # the toy model's update
        _case("adamw_toy", "adamw", "toy", param="fp32", master=False, clipped=True),
        # a ResNet-18 updated with views of the aggregated gradient
        _case("adamw_resnet18", "adamw", "resnet18", param="fp32", master=False, clipped=True, packed=True),
        # mixed precision: bf16 parameters and gradients, fp32 master weights
        _case("adamw_230m_master", "adamw", "blocks", "bf16", param="bf16", master=True, clipped=True, **blocks_230m),
        # the largest: 1.1 billion parameters with master weights, 32 GB moved a step
        _case("adamw_1b_master", "adamw", "blocks", "bf16", param="bf16", master=True, clipped=False, **blocks_1b),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn_model(rng):
    model = rng.choice(["blocks", "blocks", "adapters", "ragged"])
    if model == "ragged":
        return {"model": model, "count": _log_uniform(rng, 1, 600), "longest": _log_uniform(rng, 50, 20_000_000)}
    width = _log_uniform(rng, 33, 2048)
    if model == "adapters":
        return {"model": model, "layers": rng.randint(1, 48), "width": width, "rank": _log_uniform(rng, 1, 128)}
    return {"model": model, "layers": rng.randint(1, 24), "width": width, "hidden": rng.randint(2 * width, 4 * width),
            "vocab": _log_uniform(rng, 100, 64_000)}


def draw(rng):
    while True:
        model = _drawn_model(rng)
        dims = [k for s in _shapes(model) for k in s]
        values = sum(math.prod(s) for s in _shapes(model))
        if 3072 not in dims and 1 <= values <= 0.8 * MOST_VALUES:
            break
    op = rng.choice(["norm", "clip", "adamw"])
    grad = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    case = dict(model, op=op, grad=grad, packed=rng.random() < 0.5)
    if op == "clip":
        inplace = rng.random() < 0.3
        case.update(out=grad if inplace else rng.choice([grad, grad, "fp32"]), clipped=not inplace, inplace=inplace)
    if op == "adamw":
        param = rng.choice(["fp32", grad])
        case.update(param=param, master=param != "fp32" and rng.random() < 0.7, clipped=rng.random() < 0.7)
    return case


# ------------------------------------------------------------------ tensors


def _resnet18():
    def conv(i, o, k):
        return [(o, i, k, k), (o,), (o,)]                  # with its normalisation
    shapes, c = conv(3, 64, 3), 64
    for o in (64, 128, 256, 512):
        shapes += conv(c, o, 3) + conv(o, o, 3) + (conv(c, o, 1) if o != c else []) + conv(o, o, 3) + conv(o, o, 3)
        c = o
    return shapes + [(10, 512), (10,)]


def _shapes(case):
    kind = case["model"]
    if kind == "toy":
        return [(32, 64), (32,), (60, 32), (60,), (4, 8), (4,)]
    if kind == "resnet18":
        return _resnet18()
    if kind == "ragged":
        rng = random.Random(case["count"] * 7919 + case["longest"])
        return [((0, 1, case["longest"])[i] if i < 3 else _log_uniform(rng, 1, case["longest"]),)
                for i in range(case["count"])][::-1]
    w = case["width"]
    if kind == "adapters":
        return [(case["rank"], w), (w, case["rank"])] * (4 * case["layers"])
    h = case["hidden"]
    layer = [(w,), (w, w), (w, w), (w, w), (w, w), (w,), (h, w), (h, w), (w, h)]
    return [(case["vocab"], w)] + layer * case["layers"] + [(w,)]


def _places(case, packed):
    """(offset, length, shape) of every tensor in one buffer, and the buffer's length: packed end to
    end, or each at a multiple of 256 values."""
    at, places = 0, []
    for shape in _shapes(case):
        places.append((at, math.prod(shape), shape))
        at += places[-1][1] if packed else -(-places[-1][1] // 256) * 256
    return places, max(at, 1)


def _views(buffer, places):
    return [buffer[o: o + n].view(s) for o, n, s in places]


def _gradients(case, seed, dev):
    """One buffer of gradients: a scale per tensor, most rows of an embedding zero, and a global norm of
    several times the bound 1 (clipped) or a fraction of it."""
    places, total = _places(case, case["packed"])
    gen = torch.Generator(dev).manual_seed(seed)
    values = max(1, sum(n for _, n, _ in places))
    level = (0.3 if case.get("clipped") is False else 5.0) / math.sqrt(values)
    level *= LOSS_SCALE if case["grad"] == "fp16" else 1.0
    spread = torch.randn(len(places), generator=torch.Generator().manual_seed(seed)).mul_(0.3).exp_().tolist()
    buffer = torch.zeros(total, dtype=TYPES[case["grad"]], device=dev)
    for (o, n, shape), k in zip(places, spread):
        x = torch.randn(shape, device=dev, generator=gen) * (level * k)
        if case["model"] == "blocks" and shape[0] == case["vocab"] and len(shape) == 2:
            x *= (torch.rand(shape[0], 1, device=dev, generator=gen) < 0.1)
        buffer[o: o + n] = x.reshape(-1).to(buffer.dtype)
    return buffer, places


def _scale(case):
    return 1.0 / LOSS_SCALE if case["grad"] == "fp16" else 1.0


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g, places = _gradients(case, seed, dev)
    s = {"case": case, "g": g, "grads": _views(g, places), "norm": torch.zeros(1, device=dev), "scale": _scale(case)}
    op = case["op"]
    if op == "norm":
        s["tensors"] = torch.zeros(len(places), device=dev)
    if op == "clip":
        if case["inplace"]:
            s["out"], s["outs"] = g, s["grads"]
        else:
            at, total = _places(case, False)
            s["out"] = torch.zeros(total, dtype=TYPES[case["out"]], device=dev)
            s["outs"] = _views(s["out"], at)
    if op == "adamw":
        # a flat optimizer shard packs its state as it packs its gradients; else every tensor has its own buffers
        at, total = _places(case, case["packed"] and case["model"] == "ragged")
        gen = torch.Generator(dev).manual_seed(seed + 1)
        level = 5.0 / math.sqrt(max(1, g.numel()))
        weights = torch.randn(total, device=dev, generator=gen).mul_(0.02)
        s["m"] = torch.randn(total, device=dev, generator=gen).mul_(0.1 * level)
        s["v"] = torch.rand(total, device=dev, generator=gen).add_(0.05).mul_(level * level)
        s["param"] = weights.to(TYPES[case["param"]])
        s["master"] = weights if case["master"] else None
        s["at"] = at
        s["decay"] = [DECAY if len(x[2]) > 1 else 0.0 for x in at]
        s["step"] = STEP
    if own:                                              # the handles that a program keeps beside its tensors
        import paper_2108_02416_gb300 as ap
        s["buf"] = ap.NormBuffers(dev)
        if op == "norm":
            s["list"] = ap.TensorList(s["grads"])
        elif op == "clip":
            s["list"] = ap.TensorList(s["grads"], None if case["inplace"] else s["outs"])
        else:
            views = {k: _views(s[k], s["at"]) for k in ("param", "m", "v", "master") if s[k] is not None}
            s["list"] = ap.ParamList(views["param"], s["grads"], views["m"], views["v"], masters=views.get("master"),
                                     weight_decay=s["decay"])
    return s


# ------------------------------------------------------------------ one pass


def _plain_norms(s):
    """Every tensor's norm and the global one, in 32 bits."""
    squares = torch.stack([g.float().square().sum() for g in s["grads"]])
    return squares.sqrt() * s["scale"], squares.sum().sqrt().view(1) * s["scale"]


def _plain_coef(norm):
    return (1.0 / (norm + CLIP_EPS)).clamp(max=1.0)


def _plain_update(p, master, g, m, v, coef, decay, step):
    h = g.reshape(-1).float() * coef
    m.mul_(BETAS[0]).add_(h * (1 - BETAS[0]))
    v.mul_(BETAS[1]).add_(h * h * (1 - BETAS[1]))
    x = p.float() if master is None else master
    x = x * (1 - LR * decay) - (LR / (1 - BETAS[0] ** step)) * m / ((v / (1 - BETAS[1] ** step)).sqrt() + EPS)
    p.copy_(x)
    if master is not None:
        master.copy_(x)


def _plain(s):
    case = s["case"]
    tensors, norm = _plain_norms(s)
    if case["op"] == "norm":
        return {"norm": norm, "tensors": tensors}
    coef = _plain_coef(norm) * s["scale"]
    if case["op"] == "clip":
        for g, out in zip(s["grads"], s["outs"]):
            out.copy_(g.float() * coef)
        return {"norm": norm, "out": s["out"]}
    s["step"] += 1
    for (o, n, _), g, decay in zip(s["at"], s["grads"], s["decay"]):
        p, m, v = (s[k][o: o + n] for k in ("param", "m", "v"))
        _plain_update(p, None if s["master"] is None else s["master"][o: o + n], g, m, v, coef, decay, s["step"])
    return {"norm": norm, "param": s["param"], "master": s["master"], "m": s["m"], "v": s["v"]}


def run(s):
    if not own:
        return _plain(s)
    import paper_2108_02416_gb300 as ap
    case, buf = s["case"], s["buf"]
    if case["op"] == "norm":
        ap.aspis_grad_norm(s["list"], buf.norm, buf.work, tensor_norms=s["tensors"], scale=s["scale"])
        return {"norm": buf.norm, "tensors": s["tensors"]}
    if case["op"] == "clip":
        ap.aspis_clip_grads(s["list"], 1.0, buf.norm, buf.work, scale=s["scale"])
        return {"norm": buf.norm, "out": s["out"]}
    s["step"] += 1
    ap.aspis_adamw(s["list"], s["step"], LR, BETAS, EPS, max_norm=1.0, norm=buf.norm, work=buf.work, scale=s["scale"])
    return {"norm": buf.norm, "param": s["param"], "master": s["master"], "m": s["m"], "v": s["v"]}


def work(case):
    shapes = _shapes(case)
    n, e = sum(math.prod(x) for x in shapes), BYTES[case["grad"]]
    if case["op"] == "norm":
        return {"bytes": n * e + 4 + 4 * len(shapes), "flops": 2 * n}
    if case["op"] == "clip":
        # below the bound, in place, there is nothing to write
        return {"bytes": n * (e + (0 if case["inplace"] and not case["clipped"] else BYTES[case["out"]])) + 4,
                "flops": 3 * n}
    weights = 8 + BYTES[case["param"]] if case["master"] else 2 * BYTES[case["param"]]
    return {"bytes": n * (e + weights + 16) + 4, "flops": 16 * n}


# ------------------------------------------------------------------ 64 bits


def exact(case, seed):
    """From the definitions, in 64 bits, on fresh inputs."""
    s = prepare(case, seed)
    dev = s["g"].device
    length = [float(torch.linalg.vector_norm(g.double())) * s["scale"] for g in s["grads"]]
    norm = math.sqrt(math.fsum(x * x for x in length))
    total = torch.tensor([norm], dtype=torch.float64, device=dev)
    if case["op"] == "norm":
        return {"norm": total, "tensors": torch.tensor(length, dtype=torch.float64, device=dev)}
    factor = min(1.0, 1.0 / (norm + CLIP_EPS)) * s["scale"]
    if case["op"] == "clip":
        out = s["out"].double()
        for (o, n, _), g in zip(_places(case, case["packed"] and case["inplace"])[0], s["grads"]):
            out[o: o + n] = g.reshape(-1).double() * factor
        return {"norm": total, "out": out}
    x = (s["param"] if s["master"] is None else s["master"]).double()
    m, v = s["m"].double(), s["v"].double()
    t = s["step"] + 1
    for (o, n, _), g, decay in zip(s["at"], s["grads"], s["decay"]):
        at = slice(o, o + n)
        h = g.reshape(-1).double() * factor
        m[at] = BETAS[0] * m[at] + (1 - BETAS[0]) * h
        v[at] = BETAS[1] * v[at] + (1 - BETAS[1]) * h ** 2
        first, second = m[at] / (1 - BETAS[0] ** t), v[at] / (1 - BETAS[1] ** t)
        x[at] -= LR * (decay * x[at] + first / (second ** 0.5 + EPS))
    return {"norm": total, "param": x, "master": None if s["master"] is None else x, "m": m, "v": v}
