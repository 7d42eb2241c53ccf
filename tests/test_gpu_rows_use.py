"""The calls on rows as they are used together: a small decoder trained from a teacher's top logits, whose norm weights'
per-sample gradients go to the per-sample norm test; against autograd in fp64, one sample after the other.

Tolerance of the gradients: everything runs in fp32 here (e = 2^-24).  A gradient goes through two products with matrices
(at most 211 terms one after the other) and two norms on its way, each of which adds at most 256 e of the largest
magnitude to what the step before is off by, and so do the two products and norms forward: 8 x 256 e = 1.3e-4 of the
largest."""
import importlib.util
import os

import pytest
import torch

import paper_2412_21124_b200 as absnt

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"


def example():
    spec = importlib.util.spec_from_file_location("distilled_samples", os.path.join(ROOT, "examples", "distilled_samples.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_one_step_against_autograd():
    ex = example()
    vocab, width, top, samples = 211, 64, 5, 9
    model = ex.Decoder(vocab, width, torch.float32, DEV)
    tokens, offsets, ids, teacher, weights = ex.batch(samples, vocab, top, DEV, torch.Generator(device=DEV).manual_seed(3))
    logits = model.forward(tokens)
    losses, each = torch.empty(len(tokens), device=DEV), torch.empty(samples, device=DEV)
    absnt.abs_distill_loss(logits, ids, teacher, losses, weights=weights, offsets=offsets, sample_losses_out=each, dlogits=logits)
    grads, rows = model.backward(tokens, logits, offsets)

    def norm(s, w):
        return s / (s.square().mean(-1, keepdim=True) + ex.EPS).sqrt() * w

    def per_token(p):
        s1 = p["emb"][tokens]
        s2 = s1 + norm(s1, p["w1"]) @ p["lin"].t()
        log_q = torch.log_softmax(norm(s2, p["w2"]) @ p["head"].t(), -1).gather(1, ids)
        log_p = torch.log_softmax(teacher.double(), -1)
        return (log_p.exp() * (log_p - log_q)).sum(-1) * weights.double()

    params = {k: getattr(model, k).double().requires_grad_() for k in ("emb", "w1", "w2", "lin", "head")}
    token_losses = per_token(params)
    ref = dict(zip(params, torch.autograd.grad(token_losses.sum(), list(params.values()), retain_graph=True)))
    for k, g in grads.items():
        assert (g.double() - ref[k]).abs().max() <= 1.3e-4 * ref[k].abs().max(), k
    ends = offsets.tolist()
    for b, (a, e) in enumerate(zip(ends, ends[1:])):
        one = token_losses[a:e].sum()
        loss = float(one.detach())
        assert abs(float(each[b]) - loss) <= 1.3e-4 * loss
        parts = torch.autograd.grad(one, [params["w1"], params["w2"]], retain_graph=True)
        want = torch.cat(parts) * samples
        assert (rows[b].double() - want).abs().max() <= 1.3e-4 * want.abs().max()

    # the norm test on that matrix
    stats, gbar = absnt.alloc_persample_stats(samples, 2 * width, DEV), torch.empty(2 * width, device=DEV)
    b_next = torch.zeros(1, dtype=torch.int64, device=DEV)
    absnt.abs_persample_norm_test(rows, 0.5, stats, gbar, b_next)
    got = absnt.read_stats(stats)
    mean = rows.double().mean(0)
    assert abs(got["n2"] - float(mean.square().sum())) <= 1e-6 * got["n2"]
    assert abs(got["S"] - float((rows.double() - mean).square().sum())) <= 1e-6 * got["S"]
    assert (gbar.double() - torch.cat([ref["w1"], ref["w2"]])).abs().max() <= 1.3e-4 * gbar.abs().max()
    want = absnt.abs_decide(got["S"], got["n2"], samples - 1, 0.5, samples)
    assert int(b_next) == want[0]


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
def test_the_example_runs(dtype):
    history = example().run(steps=6, dtype=dtype, quiet=True)
    assert len(history) == 6
    sizes = [h[0] for h in history]
    assert sizes == sorted(sizes) and all(h[1] > 0 and h[2] > 0 for h in history)


def test_a_layer_captured_twice_in_one_graph():
    """Two layers of one graph, their own work areas, replayed: the same as run one by one."""
    gen = torch.Generator(device=DEV).manual_seed(0)
    rand = lambda *shape: torch.randn(*shape, device=DEV, generator=gen)  # noqa: E731
    layers = [dict(s=rand(500, 256), dy=rand(500, 256), w=rand(256), dx=torch.empty(500, 256, device=DEV),
                   dw=torch.empty(256, device=DEV)) for _ in range(2)]
    for x in layers:
        x["work"] = absnt.alloc_rms_norm_work(x["s"])

    def run():
        for x in layers:
            absnt.abs_rms_norm_grad(x["dy"], x["s"], x["w"], x["dx"], x["dw"], work=x["work"])
    run()
    want = [(x["dx"].clone(), x["dw"].clone()) for x in layers]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for x in layers:
        x["dx"].zero_(), x["dw"].zero_()
    graph.replay()
    for x, (dx, dw) in zip(layers, want):
        assert torch.equal(x["dx"], dx) and torch.equal(x["dw"], dw)
