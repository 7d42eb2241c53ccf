"""Workloads of the two ends of a decoder's backward pass: the root-mean-square norm with the residual's
addition (16-bit output, or 8-bit with scales), its gradient with the weight's gradient kept apart for
every sample of a packed batch, and the distillation loss from a teacher's top logits with the gradient
on the student's.

The weight gradients of single samples are the rows that the per-sample norm test reads, the loss is the
mean over samples that this test presumes.  `run` takes inputs as a model's layers hold them through one
operator, in its plain form or (where `own` is true) through the library's call."""
import math
import random

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
         "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1, "e5m2": 1}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}


# ------------------------------------------------------------------------------------------- cases
def _norm(name, rows, heads, width, dtype, residual, out, group=0, power=False):
    """`heads` > 1: a view of rows x heads x width into the columns of a wider matrix; `residual`: the type
    of the stream that is added and handed on, or "" for none; 8-bit outputs: a scale for each `group`
    columns (0: the row), a power of two where `power` is true."""
    return {"name": name, "op": "norm", "rows": rows, "heads": heads, "width": width, "dtype": dtype, "residual": residual,
            "out": out, "group": group, "power": power}


def _grad(name, rows, heads, width, dtype, stream, samples, apart, add=True):
    """`stream`: the type of the norm's input; `samples` of ragged lengths in the packed rows (0: no table);
    `apart`: the weight's gradient of every sample as well; `add`: the residual's own gradient is added."""
    return {"name": name, "op": "grad", "rows": rows, "heads": heads, "width": width, "dtype": dtype, "stream": stream,
            "samples": samples, "apart": apart, "add": add}


def _loss(name, rows, vocab, top, dtype, samples, gradient, tail=False, temperature=1.0, kept=1.0):
    """`tail`: the teacher's log-sum-exp is known, so its mass outside the top counts; `kept`: the share of
    tokens whose loss counts (prompts are left out)."""
    return {"name": name, "op": "loss", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "samples": samples,
            "gradient": gradient, "tail": tail, "temperature": temperature, "kept": kept}


def listed():
    return [
        # eight sequences that generate: one token of each through a layer whose product takes 8 bits
        _norm("norm_tokens", 8, 1, 2048, "bf16", "bf16", "e4m3"),
        # a pretraining micro-batch of eight sequences of 2048 tokens, residual stream in fp32
        _norm("norm_layer", 16384, 1, 2048, "bf16", "f32", "bf16"),
        # the widest input of a layer's product (its hidden width), microscaled: a power of two for 32 values
        _norm("norm_scaled", 8192, 1, 8192, "bf16", "bf16", "e4m3", group=32, power=True),
        # the queries' norm, 32 heads of 64, columns of the fused projection
        _norm("norm_heads", 16384, 32, 64, "bf16", "", "bf16"),
        # the last norm of a model small enough for a unit test or a probe
        _grad("grad_small", 512, 1, 768, "f32", "f32", 0, False, add=False),
        # a layer of the micro-batch above, weight gradients of its eight samples for the norm test
        _grad("grad_layer", 16384, 1, 2048, "bf16", "f32", 8, True),
        # documents of uneven length packed into one batch, an odd width (a pruned model)
        _grad("grad_ragged", 9001, 1, 1537, "f16", "f16", 61, True),
        # the queries' norm backwards: a weight of 64 numbers shared by half a million rows
        _grad("grad_heads", 16384, 32, 64, "bf16", "bf16", 8, True, add=False),
        # a small model on the 50257-token vocabulary: few rows, where latency counts
        _loss("loss_small", 32, 50257, 8, "f32", 1, True),
        # evaluation of a student against stored teacher logits, no gradient
        _loss("loss_eval", 8192, 32000, 32, "f16", 8, False, temperature=2.0),
        # a micro-batch on the odd vocabulary, every row at another distance from a 16-byte boundary
        _loss("loss_gpt2", 4096, 50257, 50, "bf16", 16, True, temperature=2.0),
        # a packed batch on the 128256-token vocabulary with prompts left out, teacher's mass outside its top known
        _loss("loss_llama", 8192, 128256, 64, "bf16", 23, True, tail=True, kept=0.8),
    ]


def _spread(rng, low, high):
    return max(low, min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(("norm", "grad", "loss"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    if op == "loss":
        vocab = _spread(rng, 50, 160000)
        rows = _spread(rng, 1, min(16384, 8192 * 64128 // vocab))
        c = _loss("", rows, vocab, _spread(rng, 1, min(vocab // 8 + 1, 300)), dtype, min(rows, _spread(rng, 1, 64)), rng.random() < 0.7,
                  tail=rng.random() < 0.5, temperature=rng.choice((1.0, 2.0, 0.7)), kept=rng.choice((1.0, 0.8)))
    else:
        heads = rng.choice((1, 1, 1, 4, 32))
        width = rng.choice((64, 80, 100, 128, 192)) if heads > 1 else rng.choice((
            8 * _spread(rng, 8, 2000), 8 * _spread(rng, 8, 2000), _spread(rng, 40, 9000)))
        rows = _spread(rng, 1, min(40000, 60_000_000 // (width * heads)))
        stream = rng.choice((dtype, "f32"))
        if op == "norm":
            out = rng.choice((dtype, "bf16", "e4m3", "e4m3", "e5m2"))
            group = rng.choice((0, 32, 128)) if out in LARGEST else 0
            c = _norm("", rows, heads, width, dtype, rng.choice(("", stream)), out, group, out in LARGEST and rng.random() < 0.5)
        else:
            samples = min(rows, _spread(rng, 1, 64))
            c = _grad("", rows, heads, width, dtype, stream, samples, rng.random() < 0.7, rng.random() < 0.5)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ inputs
def _lengths(rng, rows, samples):
    """`samples` lengths from one token up whose sum is `rows`."""
    cuts = sorted(rng.sample(range(1, rows), samples - 1)) if samples > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [rows])]


def _view(case, gen, dtype, std, wide=False):
    """rows x heads x width values, or rows x width for one head; `wide`: columns of a wider matrix."""
    rows, heads, width = case["rows"], case["heads"], case["width"]
    if heads == 1:
        x = torch.empty(rows, width, device=DEVICE)
        return x.normal_(generator=gen).mul_(std).to(TYPES[dtype])
    x = torch.empty(rows, 3 * heads if wide else heads, width, device=DEVICE).normal_(generator=gen).mul_(std).to(TYPES[dtype])
    return x[:, :heads]


def prepare(case, seed):
    """What a layer holds before the call, and the buffers that it keeps for results."""
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    rng = random.Random(seed)
    state = {"case": case}
    if case["op"] == "loss":
        _prepare_loss(case, gen, rng, state)
        return state
    rows, heads, width = case["rows"], case["heads"], case["width"]
    shape = (rows, width) if heads == 1 else (rows, heads, width)
    state["weight"] = torch.empty(width, device=DEVICE).normal_(generator=gen).mul_(0.2).add_(1.0).to(TYPES[case["dtype"]])
    if case["op"] == "norm":
        state["x"] = _view(case, gen, case["dtype"], 0.7, wide=True)
        if case["residual"]:
            # a stream grows with depth and has a few channels far above the others
            r = torch.empty(shape, device=DEVICE).normal_(generator=gen).mul_(2.0)
            r[..., torch.randint(width, (max(1, width // 500),), device=DEVICE, generator=gen)] *= 20.0
            state["residual"] = r.to(TYPES[case["residual"]])
            state["sum"] = torch.empty_like(state["residual"])
        state["out"] = torch.empty(shape, device=DEVICE, dtype=TYPES[case["out"]])
        if case["out"] in LARGEST:
            groups = -(-width // case["group"]) if case["group"] else 1
            state["scales"] = torch.empty(shape[:-1] + (groups,), device=DEVICE,
                                          dtype=torch.float8_e8m0fnu if case["power"] else torch.float32)
        return state
    state["s"] = _view(case, gen, case["stream"], 2.0, wide=True)
    state["dy"] = _view(case, gen, case["dtype"], 0.01)
    state["add"] = _view(case, gen, case["stream"], 0.01) if case["add"] else None
    state["dx"] = torch.empty(shape, device=DEVICE, dtype=TYPES[case["stream"]])
    state["dweight"] = torch.empty(width, device=DEVICE)
    state["of"] = state["offsets"] = state["apart"] = None
    samples = case["samples"]
    if samples:
        lengths = _lengths(rng, rows, samples)
        state["of"] = torch.repeat_interleave(torch.arange(samples, device=DEVICE), torch.tensor(lengths, device=DEVICE))
        ends = torch.tensor([0] + lengths).cumsum(0)
        state["offsets"] = ends.to(torch.int32).to(DEVICE)
        if case["apart"]:
            state["apart"] = torch.empty(samples, width, device=DEVICE)
    if own:
        import paper_2412_21124_b200 as absnt
        state["work"] = absnt.alloc_rms_norm_work(state["s"], samples)
    return state


def _prepare_loss(case, gen, rng, state):
    """Student logits with peaks where the teacher has its top entries, which come sorted."""
    rows, vocab, top, samples = case["rows"], case["vocab"], case["top"], case["samples"]
    logits = torch.empty(rows, vocab, device=DEVICE).normal_(generator=gen).mul_(1.5)
    teacher = torch.empty(rows, top, device=DEVICE).normal_(generator=gen).mul_(2.0).sort(-1, descending=True).values
    teacher += 6.0
    first = torch.randint(vocab, (rows, 1), device=DEVICE, generator=gen)
    ids = (first + torch.randperm(vocab // 8 + 1, device=DEVICE, generator=gen)[:top] * 7 % vocab) % vocab
    logits.scatter_(1, ids, teacher + torch.empty_like(teacher).normal_(generator=gen))
    state["logits"] = logits.to(TYPES[case["dtype"]])
    state["ids"] = ids
    state["top"] = teacher.to(torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
    if case["tail"]:
        z = state["top"].float() / case["temperature"]
        rest = torch.empty(rows, device=DEVICE).uniform_(-4.0, -0.5, generator=gen)
        state["lse"] = torch.logsumexp(z, -1) - torch.log1p(-rest.exp())  # the top holds 1 - exp(rest) of the mass
    lengths = _lengths(rng, rows, samples)
    ends = torch.tensor([0] + lengths).cumsum(0)
    state["offsets"] = ends.to(torch.int32).to(DEVICE)
    state["of"] = torch.repeat_interleave(torch.arange(samples, device=DEVICE), torch.tensor(lengths, device=DEVICE))
    counts = torch.rand(rows, device=DEVICE, generator=gen) < case["kept"]
    each = torch.zeros(samples, device=DEVICE).index_add_(0, state["of"], counts.float()).clamp_(min=1.0)
    state["weights"] = counts / (samples * each[state["of"]])  # a mean over samples of means over tokens
    state["losses"] = torch.empty(rows, device=DEVICE)
    state["sample_losses"] = torch.empty(samples, device=DEVICE)
    if case["gradient"]:
        state["dlogits"] = torch.empty_like(state["logits"])
    state["scale"] = 65536.0 if case["dtype"] == "f16" else 1.0  # a loss scale


# --------------------------------------------------------------------------------------- operators
def run(state):
    case = state["case"]
    if own:
        return {"norm": own_norm, "grad": own_grad, "loss": own_loss}[case["op"]](state, case)
    return {"norm": plain_norm, "grad": plain_grad, "loss": plain_loss}[case["op"]](state, case)


def plain_norm(state, case):
    s, outs = state["x"].float(), {}
    if case["residual"]:
        s = s + state["residual"].float()
        outs["sum"] = s.to(TYPES[case["residual"]])
    y = s * torch.rsqrt((s * s).mean(-1, keepdim=True) + EPS) * state["weight"].float()
    if case["out"] not in LARGEST:
        outs["out"] = y.to(TYPES[case["out"]])
        return outs
    width = case["width"]
    group = case["group"] or width
    groups = -(-width // group)
    y = torch.nn.functional.pad(y, (0, groups * group - width)).view(y.shape[:-1] + (groups, group))
    scale = y.abs().amax(-1, keepdim=True) / LARGEST[case["out"]]
    scale = torch.where(scale == 0, 1.0, scale)
    if case["power"]:
        part, power = torch.frexp(scale)
        scale = torch.ldexp(torch.ones_like(scale), power - (part == 0.5).int())
    q = (y / scale).flatten(-2)[..., :width]
    outs["out"] = q.to(TYPES[case["out"]])
    outs["scales"] = scale.squeeze(-1).to(state["scales"].dtype)
    return outs


def plain_grad(state, case):
    s, dy, width = state["s"].float(), state["dy"].float(), case["width"]
    rstd = torch.rsqrt((s * s).mean(-1, keepdim=True) + EPS)
    g = dy * state["weight"].float()
    dx = rstd * (g - s * (rstd * rstd * (g * s).mean(-1, keepdim=True)))
    if case["add"]:
        dx = dx + state["add"].float()
    part = dy * (s * rstd)
    if case["heads"] > 1:
        part = part.sum(1)
    outs = {"dx": dx.to(TYPES[case["stream"]])}
    if case["apart"]:
        outs["apart"] = torch.zeros(case["samples"], width, device=DEVICE).index_add_(0, state["of"], part)
        outs["dweight"] = outs["apart"].sum(0)
    else:
        outs["dweight"] = part.sum(0)
    return outs


def plain_loss(state, case):
    tau, ids = case["temperature"], state["ids"]
    z = state["logits"].float() / tau
    z = z - z.amax(-1, keepdim=True)
    e = z.exp()
    total = e.sum(-1, keepdim=True)
    log_q = z.gather(1, ids) - total.log()
    t = state["top"].float() / tau
    if case["tail"]:
        log_p = t - state["lse"][:, None]
        p = log_p.exp()
        p_rest = (1.0 - p.sum(-1, keepdim=True)).clamp(min=0.0)
        q_rest = e.scatter(1, ids, 0.0).sum(-1, keepdim=True) / total
        losses = (p * (log_p - log_q)).sum(-1) + (p_rest * (p_rest / q_rest).log()).squeeze(-1)
    else:
        t = t - t.amax(-1, keepdim=True)
        log_p = t - t.exp().sum(-1, keepdim=True).log()
        p = log_p.exp()
        losses = (p * (log_p - log_q)).sum(-1)
    counts = state["weights"] != 0
    losses = torch.where(counts, tau * tau * losses, 0.0)
    each = torch.zeros(case["samples"], device=DEVICE).index_add_(0, state["of"], losses * state["weights"])
    outs = {"losses": losses, "sample_losses": each}
    if case["gradient"]:
        if case["tail"]:
            g = e * ((1.0 - p_rest / q_rest) / total)
            g = g.scatter(1, ids, log_q.exp() - p)
        else:
            g = (e / total).scatter(1, ids, log_q.exp() - p)
        outs["dlogits"] = (g * (tau * state["scale"] * state["weights"])[:, None]).to(TYPES[case["dtype"]])
    return outs


def own_norm(state, case):
    import paper_2412_21124_b200 as absnt
    absnt.abs_rms_norm(state["x"], state["weight"], state["out"], EPS, residual=state.get("residual"), sum_out=state.get("sum"),
                       scales_out=state.get("scales"), group=case["group"])
    return {k: state[k] for k in ("sum", "out", "scales") if k in state}


def own_grad(state, case):
    import paper_2412_21124_b200 as absnt
    absnt.abs_rms_norm_grad(state["dy"], state["s"], state["weight"], state["dx"], state["dweight"], EPS, dresidual=state["add"],
                            offsets=state["offsets"], dweight_samples=state["apart"], work=state["work"])
    outs = {"dx": state["dx"], "dweight": state["dweight"]}
    if case["apart"]:
        outs["apart"] = state["apart"]
    return outs


def own_loss(state, case):
    import paper_2412_21124_b200 as absnt
    absnt.abs_distill_loss(state["logits"], state["ids"], state["top"], state["losses"], temperature=case["temperature"],
                           teacher_lse=state.get("lse"), weights=state["weights"], offsets=state["offsets"],
                           sample_losses_out=state["sample_losses"], dlogits=state.get("dlogits"), grad_scale=state["scale"])
    return {k: state[k] for k in ("losses", "sample_losses", "dlogits") if k in state}


def work(case):
    """Bytes: each input read once, each result written once.  Operations: a value's share of the sums and
    products above, an exponential counted as one."""
    if case["op"] == "loss":
        rows, values = case["rows"], case["rows"] * case["vocab"]
        # rows that do not count need no reading; their gradient is still written
        moved = values * BYTES[case["dtype"]] * (case["kept"] + (1 if case["gradient"] else 0))
        moved += rows * case["top"] * (8 + (4 if case["dtype"] == "f32" else 2)) + 4 * rows * (3 if case["tail"] else 2) + 8 * case["samples"]
        return {"bytes": moved, "flops": values * case["kept"] * (6 if case["gradient"] else 4)}
    values, width = case["rows"] * case["heads"] * case["width"], case["width"]
    if case["op"] == "norm":
        each = BYTES[case["dtype"]] + BYTES[case["out"]] + (2 * BYTES[case["residual"]] if case["residual"] else 0)
        groups = -(-width // case["group"]) if case["group"] else 1
        scales = case["rows"] * case["heads"] * groups * (1 if case["power"] else 4) if case["out"] in LARGEST else 0
        return {"bytes": values * each + scales + width * BYTES[case["dtype"]], "flops": 6 * values}
    each = BYTES[case["dtype"]] + BYTES[case["stream"]] * (3 if case["add"] else 2)
    apart = 4 * case["samples"] * width if case["apart"] else 0
    return {"bytes": values * each + apart + width * (4 + BYTES[case["dtype"]]) + 4 * case["samples"], "flops": 13 * values}


def exact(case, seed):
    """The same from the definition in 64 bits, a stretch of rows at a time."""
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    return {"norm": _exact_norm, "grad": _exact_grad, "loss": _exact_loss}[case["op"]](state, case)


def _exact_norm(state, case):
    s = state["x"].double()
    outs = {}
    if case["residual"]:
        s = s + state["residual"].double()
        outs["sum"] = s
    y = s / (s.square().sum(-1, keepdim=True) / case["width"] + EPS).sqrt() * state["weight"].double()
    outs["out"] = y
    if case["out"] in LARGEST:
        out, scales = [], []
        for part in y.split(case["group"] or case["width"], dim=-1):
            scale = part.abs().max(-1, keepdim=True).values / LARGEST[case["out"]]
            scale[scale == 0] = 1.0
            if case["power"]:
                scale = 2.0 ** torch.ceil(torch.log2(scale))
            out.append((part / scale).to(TYPES[case["out"]]).double())
            scales.append(scale)
        outs["out"], outs["scales"] = torch.cat(out, -1), torch.cat(scales, -1)
    return outs


def _exact_grad(state, case):
    s, dy, w = state["s"].double(), state["dy"].double(), state["weight"].double()
    norm = (s.square().sum(-1, keepdim=True) / case["width"] + EPS).sqrt()
    unit = s / norm
    g = dy * w
    dx = (g - unit * (unit * g).sum(-1, keepdim=True) / case["width"]) / norm
    if case["add"]:
        dx = dx + state["add"].double()
    part = (dy * unit).reshape(case["rows"], -1, case["width"]).sum(1)
    outs = {"dx": dx, "dweight": part.sum(0)}
    if case["apart"]:
        ends = state["offsets"].tolist()
        outs["apart"] = torch.stack([part[a:b].sum(0) for a, b in zip(ends, ends[1:])])
    return outs


def _exact_loss(state, case):
    tau, rows, vocab = case["temperature"], case["rows"], case["vocab"]
    losses = torch.zeros(rows, device=DEVICE, dtype=torch.float64)
    grads = torch.empty(rows, vocab, device=DEVICE, dtype=torch.float64) if case["gradient"] else None
    weights = state["weights"].double()
    step = max(1, (1 << 27) // vocab)
    for a in range(0, rows, step):
        here = slice(a, a + step)
        ids, t = state["ids"][here], state["top"][here].double() / tau
        log_q = torch.log_softmax(state["logits"][here].double() / tau, -1)
        inside = torch.zeros_like(log_q, dtype=torch.bool).scatter_(1, ids, True)
        if case["tail"]:
            log_p = t - state["lse"][here].double()[:, None]
            rest = (1.0 - log_p.exp().sum(-1)).clamp(min=0.0)
            log_rest = torch.logsumexp(log_q.masked_fill(inside, -math.inf), -1)
            more = rest * (rest.log() - log_rest)
        else:
            log_p, more = torch.log_softmax(t, -1), 0.0
        p = log_p.exp()
        losses[here] = tau ** 2 * ((p * (log_p - log_q.gather(1, ids))).sum(-1) + more)
        if case["gradient"]:
            g = log_q.exp()
            if case["tail"]:
                g -= (rest[:, None] * (log_q - log_rest[:, None]).exp()).masked_fill(inside, 0.0)
            g.scatter_add_(1, ids, -p)
            grads[here] = g * (tau * state["scale"] * weights[here])[:, None]
    losses[weights == 0] = 0.0
    ends = state["offsets"].tolist()
    each = torch.stack([(losses[a:b] * weights[a:b]).sum() for a, b in zip(ends, ends[1:])])
    outs = {"losses": losses, "sample_losses": each}
    if case["gradient"]:
        outs["dlogits"] = grads
    return outs
