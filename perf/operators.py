"""Workloads of the operators over a list of gradient tensors: the global norm, clipping by it, and
the clipped AdamW step, as a training loop calls them between the backward pass and the next forward.

A model's gradients do not lie in one flat vector: they are a list of tensors of its own shapes, some of
them views into a bucket, some of them columns of a wider matrix, weights in 16 bits and norms in 32.
`run` takes such a list through one operator, in its plain form or (where `own` is true) through the
library's call on the same tensors."""
import math
import random

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6  # added to the norm before the division, the convention of norm clipping
HP = dict(lr=4e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
STEP = 100
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
NORMS = {"2": 2.0, "1": 1.0, "inf": math.inf}


# ------------------------------------------------------------------------------------ tensor lists
def gpt2_small_shapes():
    """GPT-2 small: 148 tensors, 124,439,808 parameters."""
    w, vocab, ctx = 768, 50257, 1024
    block = [(w,), (w,), (w, 3 * w), (3 * w,), (w, w), (w,), (w,), (w,), (w, 4 * w), (4 * w,), (4 * w, w), (w,)]
    return [(vocab, w), (ctx, w)] + 12 * block + [(w,), (w,)]


def llama_1b_shapes():
    """A Llama-style decoder of 16 layers: 146 tensors, 1,235,814,400 parameters."""
    h, ff, vocab, kv = 2048, 8192, 128256, 512
    block = [(h, h), (kv, h), (kv, h), (h, h), (ff, h), (ff, h), (h, ff), (h,), (h,)]
    return [(vocab, h)] + 16 * block + [(h,)]


def ragged_shapes(tensors, elements):
    """`tensors` shapes of about `elements` values together, sizes spread over a factor of a hundred, odd
    ones among them, every fourth a vector; one tensor is empty and one holds a single value."""
    rng = random.Random(1000003 * tensors + elements)
    weight = [math.exp(rng.uniform(0.0, math.log(100.0))) for _ in range(tensors)]
    per = elements / sum(weight)
    shapes = []
    for i, x in enumerate(weight):
        n = max(2, int(x * per))
        rows = 1 if i % 4 == 3 else max(1, min(n // 2, int(math.sqrt(n) * rng.uniform(0.2, 2.0))))
        shapes.append((n,) if rows == 1 else (rows, max(1, n // rows)))
    if tensors > 2:
        shapes[1], shapes[2] = (0,), (1,)
    return shapes


def shapes_of(case):
    if case["shapes"] == "gpt2_small":
        return gpt2_small_shapes()
    if case["shapes"] == "llama_1b":
        return llama_1b_shapes()
    return ragged_shapes(case["tensors"], case["elements"])


def type_of(case, shape):
    """Vectors (norm weights, biases) may be kept in another type than matrices."""
    return case["vectors"] if len(shape) == 1 else case["dtype"]


# ------------------------------------------------------------------------------------------- cases
def _case(name, op, shapes, dtype, layout="separate", vectors=None, norm="2", out="", tensors=0, elements=0, scale=1.0):
    return {"name": name, "op": op, "shapes": shapes, "tensors": tensors, "elements": elements, "dtype": dtype,
            "vectors": vectors or dtype, "layout": layout, "norm": norm, "out": out, "scale": scale}


def listed():
    return [
        # the logged norm of a model small enough for a unit test or a probe: latency alone
        _case("norm_small", "norm", "ragged", "f32", tensors=20, elements=60_000),
        # low-rank adapters of every layer: very many small tensors of odd sizes, views into one bucket
        _case("norm_adapters", "norm", "ragged", "bf16", layout="bucket", tensors=1200, elements=24_000_000),
        # the largest gradient of a model, as a monitor of outliers reads it
        _case("norm_max_gpt2", "norm", "gpt2_small", "f32", norm="inf"),
        # the norm before the step of a 1.2B decoder, matrices in bf16 and norm weights in fp32
        _case("norm_llama", "norm", "llama_1b", "bf16", vectors="f32"),
        # clipping for a small model
        _case("clip_small", "clip", "ragged", "f32", out="f32", tensors=20, elements=60_000),
        # clipping between the backward pass and a bf16 exchange, gradients of separate allocations
        _case("clip_gpt2", "clip", "gpt2_small", "bf16", out="bf16"),
        # fp16 gradients under a loss scale, columns of fused matrices, unscaled into fp32 while clipping
        _case("clip_slices", "clip", "ragged", "f16", layout="slices", vectors="f32", out="f32", tensors=90, elements=30_000_001,
              scale=1.0 / 1024),
        # fp32 accumulated gradients of a 1.2B decoder, averaged over 8 micro-batches, clipped into bf16
        _case("clip_llama", "clip", "llama_1b", "f32", out="bf16", scale=1.0 / 8),
        # the whole step of a small model
        _case("step_small", "step", "ragged", "f32", tensors=20, elements=60_000),
        # the step over adapters: fp32 gradients, views into one bucket at odd offsets
        _case("step_adapters", "step", "ragged", "f32", layout="bucket", tensors=1200, elements=24_000_000),
        # the step of mixed-precision training: bf16 gradients, fp32 state, a bf16 copy of the weights
        _case("step_gpt2", "step", "gpt2_small", "bf16", out="bf16"),
        _case("step_llama", "step", "llama_1b", "bf16", vectors="f32", out="bf16", scale=1.0 / 8),
    ]


def draw(rng):
    op = rng.choice(("norm", "clip", "step"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    tensors = int(math.exp(rng.uniform(math.log(1), math.log(2000))))
    elements = int(math.exp(rng.uniform(math.log(300), math.log(4e8)))) | 1
    out = {"norm": "", "clip": rng.choice((dtype, "f32", "bf16")), "step": rng.choice(("", "bf16"))}[op]
    c = _case("", op, "ragged", dtype, layout=rng.choice(("separate", "bucket", "slices")), vectors=rng.choice((dtype, "f32")),
              norm=rng.choice(("2", "2", "2", "inf", "1")), out=out, tensors=tensors, elements=max(elements, 3 * tensors),
              scale=rng.choice((1.0, 1.0, 1.0 / 8, 1.0 / 1024)))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    """The gradient list as a backward pass leaves it, and what the operator's caller keeps beside it: the
    buffers that results go to and, for the library, its handle on the tensors."""
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    rng = random.Random(seed)
    shapes = shapes_of(case)
    sizes = [math.prod(s) for s in shapes]
    total = sum(sizes)

    # one noise scale for each tensor; the rows of the first matrix (an embedding) are mostly zero
    noise = torch.empty(max(total, 1), device=DEVICE).normal_(generator=gen)
    big = 1.0 / case["scale"]  # a loss scale, or a sum over micro-batches
    bucket = {t: torch.empty(0, device=DEVICE, dtype=TYPES[t]) for t in TYPES}
    if case["layout"] == "bucket":
        for t in TYPES:
            n = sum(size for size, s in zip(sizes, shapes) if type_of(case, s) == t)
            bucket[t] = torch.empty(n, device=DEVICE, dtype=TYPES[t])
    used = dict.fromkeys(TYPES, 0)
    grads, at, first = [], 0, True
    for s, n in zip(shapes, sizes):
        t = type_of(case, s)
        x = noise[at:at + n].view(s)
        x *= math.exp(rng.uniform(math.log(1e-4), math.log(3e-3))) * min(big, 1024.0)
        if first and len(s) == 2 and s[0] > 100:
            x *= (torch.rand(s[0], 1, device=DEVICE, generator=gen) < 0.4)
            first = False
        if case["layout"] == "bucket":
            g = bucket[t][used[t]:used[t] + n].view(s)
            used[t] += n
        elif case["layout"] == "slices" and len(s) == 2:
            g = torch.empty(s[0], 2 * s[1] + 8, device=DEVICE, dtype=TYPES[t])[:, s[1]:2 * s[1]]
        else:
            g = torch.empty(s, device=DEVICE, dtype=TYPES[t])
        g.copy_(x)
        grads.append(g)
        at += n
    del noise, x

    state = {"case": case, "grads": grads, "sizes": sizes, "max_norm": max_norm_of(case, total)}
    groups = [0 if len(s) == 2 else 1 for s in shapes]  # vectors take no weight decay
    state["hparams"] = [HP, dict(HP, weight_decay=0.0)]
    more = {}
    views = lambda flat: [v.view(s) for v, s in zip(flat.split(sizes), shapes)]  # noqa: E731
    if case["op"] == "clip":
        state["out"] = torch.empty(total, device=DEVICE, dtype=TYPES[case["out"]])
        more["out"] = views(state["out"])
    elif case["op"] == "step":
        state["p"] = torch.empty(total, device=DEVICE).normal_(generator=gen).mul_(0.02)
        state["m"] = torch.empty(total, device=DEVICE).normal_(generator=gen).mul_(1e-5)
        state["v"] = torch.empty(total, device=DEVICE).uniform_(1e-11, 1e-9, generator=gen)
        more.update(params=views(state["p"]), m=views(state["m"]), v=views(state["v"]), groups=groups)
        state["decay"] = [HP["weight_decay"] if k == 0 else 0.0 for k in groups]
        if case["out"]:
            state["p16"] = torch.empty(total, device=DEVICE, dtype=TYPES[case["out"]])
            more["params_bf16"] = views(state["p16"])
    if own:
        import paper_2412_21124_b200 as absnt
        state["tensors"] = absnt.GradTensors(grads, **more)
    return state


def max_norm_of(case, total):
    """Below the norm that the noise of prepare() has, so that the step is one that clips."""
    if case["norm"] == "inf":
        return 1e-3
    return 0.1 if case["norm"] == "2" else 1e-5 * max(total, 1)


# --------------------------------------------------------------------------------------- operators
def run(state):
    case = state["case"]
    if own:
        return run_own(state, case)
    norm, scale = case["norm"], case["scale"]
    size = [g.float().abs() for g in state["grads"]]
    zero = torch.zeros((), device=DEVICE)
    if norm == "2":
        each = torch.stack([(x * x).sum() for x in size])
        total, each = each.sum().sqrt(), each.sqrt()
    elif norm == "1":
        each = torch.stack([x.sum() for x in size])
        total = each.sum()
    else:
        each = torch.stack([x.max() if x.numel() else zero for x in size])
        total = each.max()
    del size
    total, each = total * scale, each * scale
    if case["op"] == "norm":
        return {"norm": total, "each": each}
    coef = torch.clamp(state["max_norm"] / (total + EPS), max=1.0)
    g = torch.cat([x.float().reshape(-1) for x in state["grads"]]) * (coef * scale)
    if case["op"] == "clip":
        state["out"].copy_(g)
        return {"norm": total, "coef": coef, "each": each, "out": state["out"]}
    p, m, v = state["p"], state["m"], state["v"]
    m.mul_(HP["beta1"]).add_(g, alpha=1 - HP["beta1"])
    v.mul_(HP["beta2"]).add_(g * g, alpha=1 - HP["beta2"])
    decay = torch.cat([x.new_full((n,), 1 - HP["lr"] * d) for x, n, d in zip(p.split(state["sizes"]), state["sizes"], state["decay"])])
    step = (m / (1 - HP["beta1"] ** STEP)) / ((v / (1 - HP["beta2"] ** STEP)).sqrt() + HP["eps"])
    p.mul_(decay).sub_(step, alpha=HP["lr"])
    outs = {"norm": total, "coef": coef, "each": each, "p": p, "m": m, "v": v}
    if case["out"]:
        state["p16"].copy_(p)
        outs["p16"] = state["p16"]
    return outs


def run_own(state, case):
    import paper_2412_21124_b200 as absnt
    t, norm, scale = state["tensors"], NORMS[case["norm"]], case["scale"]
    if case["op"] == "norm":
        absnt.abs_grad_norm(t, norm_type=norm, grad_scale=scale)
        return {"norm": t.norm, "each": t.norms}
    if case["op"] == "clip":
        absnt.abs_grad_clip(t, state["max_norm"], norm_type=norm, grad_scale=scale)
        return {"norm": t.norm, "coef": t.coef, "each": t.norms, "out": state["out"]}
    absnt.abs_grad_adamw(t, state["hparams"], STEP, state["max_norm"], norm_type=norm, grad_scale=scale)
    outs = {"norm": t.norm, "coef": t.coef, "each": t.norms, "p": state["p"], "m": state["m"], "v": state["v"]}
    if case["out"]:
        outs["p16"] = state["p16"]
    return outs


def work(case):
    """Bytes: each gradient read once, each result written once (for the step: parameters and moments read
    and written).  Operations: two a value for a norm, one for a scale, fifteen for an AdamW update."""
    shapes = shapes_of(case)
    n = sum(math.prod(s) for s in shapes)
    moved = sum(math.prod(s) * BYTES[type_of(case, s)] for s in shapes) + 4 * (len(shapes) + 2)
    flops = 2 * n
    if case["op"] == "clip":
        moved, flops = moved + n * BYTES[case["out"]], flops + n
    elif case["op"] == "step":
        moved, flops = moved + n * (24 + (BYTES[case["out"]] if case["out"] else 0)), flops + 15 * n
    return {"bytes": moved, "flops": flops}


def exact(case, seed):
    """The same from the definition in 64 bits, one tensor after the other."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    order = NORMS[case["norm"]]
    each = []
    for g in s["grads"]:
        a = g.double().reshape(-1)
        each.append(torch.linalg.vector_norm(a, order) if a.numel() else torch.zeros((), device=DEVICE, dtype=torch.float64))
    each = torch.stack(each) * case["scale"]
    total = torch.linalg.vector_norm(each, order)
    if case["op"] == "norm":
        return {"norm": total, "each": each}
    ratio = s["max_norm"] / (float(total) + EPS)
    coef = min(1.0, ratio)
    res = {"norm": total, "coef": torch.tensor(coef, dtype=torch.float64, device=DEVICE), "each": each}
    n = sum(s["sizes"])
    if case["op"] == "clip":
        res["out"] = torch.empty(n, dtype=torch.float64, device=DEVICE)
        for x, g in zip(res["out"].split(s["sizes"]), s["grads"]):
            x.copy_(g.reshape(-1)).mul_(coef * case["scale"])
        return res
    b1, b2 = HP["beta1"], HP["beta2"]
    at = 0
    for name in ("p", "m", "v"):
        res[name] = torch.empty(n, dtype=torch.float64, device=DEVICE)
    for g, size, decay in zip(s["grads"], s["sizes"], s["decay"]):
        here = slice(at, at + size)
        g = g.double().reshape(-1) * (coef * case["scale"])
        m = b1 * s["m"][here].double() + (1 - b1) * g
        v = b2 * s["v"][here].double() + (1 - b2) * g ** 2
        hat_m, hat_v = m / (1 - b1 ** STEP), v / (1 - b2 ** STEP)
        w = s["p"][here].double()
        res["p"][here] = w - HP["lr"] * (decay * w + hat_m / (hat_v.sqrt() + HP["eps"]))
        res["m"][here], res["v"][here] = m, v
        at += size
    if case["out"]:
        res["p16"] = res["p"]
    return res
