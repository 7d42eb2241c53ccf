"""A training run whose batch size follows the per-sample norm test of its norm weights.

  python examples/distilled_samples.py [--steps 20]

A small decoder without attention learns a teacher's top logits.  Sequences of uneven length lie packed one behind
the other.  abs_distill_loss gives the loss of every sequence and the gradient on the logits, abs_rms_norm_grad
the norm weights' gradients of every sequence as columns of one matrix [sequences, weights], and
abs_persample_norm_test reads that matrix: how noisy the gradients of single sequences are decides how many
the next step takes.  The step itself is abs_grad_adamw on the tensors as they lie."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2412_21124_b200 as absnt  # noqa: E402

EPS = 1e-6


class Decoder:
    """embedding -> norm -> linear, added to the stream -> norm -> logits; gradients by hand"""

    def __init__(self, vocab, width, dtype, dev, seed=0):
        gen = torch.Generator(device=dev).manual_seed(seed)
        rand = lambda *shape, std: (torch.randn(*shape, device=dev, generator=gen) * std).to(dtype)  # noqa: E731
        self.width, self.dtype = width, dtype
        self.emb = rand(vocab, width, std=1.0)
        self.w1, self.w2 = (torch.ones(width, device=dev) + rand(width, std=0.1).float()).to(dtype), torch.ones(width, device=dev).to(dtype)
        self.lin, self.head = rand(width, width, std=width ** -0.5), rand(vocab, width, std=width ** -0.5)

    def forward(self, tokens):
        self.s1 = self.emb[tokens].float()  # the residual stream stays in fp32
        self.y1 = torch.empty_like(self.s1, dtype=self.dtype)
        absnt.abs_rms_norm(self.s1, self.w1, self.y1, EPS)
        mixed = self.y1 @ self.lin.t()
        self.s2, self.y2 = torch.empty_like(self.s1), torch.empty_like(self.y1)
        absnt.abs_rms_norm(mixed, self.w2, self.y2, EPS, residual=self.s1, sum_out=self.s2)
        return self.y2 @ self.head.t()

    def backward(self, tokens, dlogits, offsets):
        """Gradients of all tensors, and of the two norm weights for every sample: a matrix [samples, 2 width] whose
        rows are those of the samples' own losses."""
        samples, width = offsets.numel() - 1, self.width
        rows = torch.empty(samples, 2 * width, device=dlogits.device)
        work = absnt.alloc_rms_norm_work(self.s1, samples)
        dhead = dlogits.t() @ self.y2
        ds2, dw2 = torch.empty_like(self.s2), torch.empty(width, device=dlogits.device)
        absnt.abs_rms_norm_grad(dlogits @ self.head, self.s2, self.w2, ds2, dw2, EPS, offsets=offsets,
                                dweight_samples=rows[:, width:], sample_scale=samples, work=work)
        dmixed = ds2.to(self.dtype)
        dlin = dmixed.t() @ self.y1
        ds1, dw1 = torch.empty_like(self.s1), torch.empty(width, device=dlogits.device)
        absnt.abs_rms_norm_grad(dmixed @ self.lin, self.s1, self.w1, ds1, dw1, EPS, dresidual=ds2, offsets=offsets,
                                dweight_samples=rows[:, :width], sample_scale=samples, work=work)
        demb = torch.zeros_like(self.emb, dtype=torch.float32).index_add_(0, tokens, ds1)
        return {"emb": demb, "w1": dw1, "w2": dw2, "lin": dlin, "head": dhead}, rows


def batch(samples, vocab, top, dev, gen):
    """Packed sequences of 3 to 40 tokens, what a teacher says of them, and the tokens' weights: half of every sequence is
    prompt, and the loss is a mean over sequences of means over the rest."""
    lengths = torch.randint(3, 41, (samples,), device=dev, generator=gen)
    offsets = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)]).to(torch.int32)
    total = int(offsets[-1])
    tokens = torch.randint(vocab, (total,), device=dev, generator=gen)
    ids = (tokens[:, None] * 3 + torch.arange(top, device=dev) * 5) % vocab
    logits = 4.0 - 0.5 * torch.arange(top, device=dev).float().expand(total, top) + 0.1 * torch.randn(total, top, device=dev, generator=gen)
    of = torch.repeat_interleave(torch.arange(samples, device=dev), lengths)
    counts = (torch.arange(total, device=dev) - offsets[of]) >= lengths[of] // 2
    weights = counts / (samples * torch.zeros(samples, device=dev).index_add_(0, of, counts.float())[of])
    return tokens, offsets, ids, logits.contiguous(), weights


def run(steps=20, vocab=211, width=64, top=5, samples=8, most=64, eta=0.5, dtype=torch.bfloat16, dev="cuda", quiet=False):
    gen = torch.Generator(device=dev).manual_seed(1)
    model = Decoder(vocab, width, dtype, dev)
    names = ("emb", "w1", "w2", "lin", "head")
    master = {k: getattr(model, k).float() for k in names}
    state = [[torch.zeros_like(master[k]) for k in names] for _ in range(2)]
    hp = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0)
    gbar, b_next = torch.empty(2 * width, device=dev), torch.zeros(1, dtype=torch.int64, device=dev)
    history = []
    for step in range(1, steps + 1):
        tokens, offsets, ids, teacher, weights = batch(samples, vocab, top, dev, gen)
        logits = model.forward(tokens)
        losses, each = torch.empty(len(tokens), device=dev), torch.empty(samples, device=dev)
        absnt.abs_distill_loss(logits, ids, teacher, losses, weights=weights, offsets=offsets, sample_losses_out=each,
                               dlogits=logits)  # the gradient takes the logits' place
        grads, rows = model.backward(tokens, logits, offsets)
        stats = absnt.alloc_persample_stats(samples, 2 * width, dev)
        absnt.abs_persample_norm_test(rows, eta, stats, gbar, b_next)
        tensors = absnt.GradTensors([grads[k].contiguous() for k in names], params=[master[k] for k in names], m=state[0],
                                    v=state[1], params_bf16=[getattr(model, k) for k in names] if dtype == torch.bfloat16 else None)
        absnt.abs_grad_adamw(tensors, hp, step, max_norm=1.0)
        if dtype != torch.bfloat16:
            for k in names:
                getattr(model, k).copy_(master[k])
        history.append((samples, float(each.sum()), absnt.read_stats(stats)["T"]))
        if not quiet:
            print("step %2d  sequences %3d  loss %.4f  T %.1f" % ((step,) + history[-1]))
        samples = min(most, max(samples, int(b_next)))
    return history


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=20)
    run(ap.parse_args().steps)
