"""A small training run on lists of tensors: a bf16 model, fp32 master weights, gradients averaged over
micro-batches, clipped by their global norm and applied by AdamW, all on the tensors as they lie.

  python examples/clipped_training.py [--steps 60]

The model's own bf16 parameters are the working copy that abs_grad_adamw writes, and its .grad tensors
(kept in place between steps) are the gradients, so one GradTensors built before the loop serves every
step.  Matrices decay, vectors do not.  Every tenth step the norms of the single tensors are printed and
every gradient is clipped in place by its largest value first."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2412_21124_b200 as absnt  # noqa: E402


def make_model(width, dev):
    torch.manual_seed(0)
    return torch.nn.Sequential(
        torch.nn.Linear(16, width), torch.nn.GELU(), torch.nn.LayerNorm(width),
        torch.nn.Linear(width, width), torch.nn.GELU(), torch.nn.LayerNorm(width),
        torch.nn.Linear(width, 1)).to(dev)


def run(steps=60, width=256, batch=512, micro_batches=4, max_norm=1.0, dev="cuda", quiet=False):
    model = make_model(width, dev)
    master = [p.detach().clone() for p in model.parameters()]
    model.to(torch.bfloat16)
    params = list(model.parameters())
    for p in params:
        p.grad = torch.zeros_like(p)
    tensors = absnt.GradTensors(
        [p.grad for p in params], params=master, m=[torch.zeros_like(w) for w in master],
        v=[torch.zeros_like(w) for w in master], params_bf16=[p.detach() for p in params],
        groups=[0 if p.dim() == 2 else 1 for p in params])
    hp = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
    hparams = [hp, dict(hp, weight_decay=0.0)]

    gen = torch.Generator(device=dev).manual_seed(1)
    target = 0.3 * torch.randn(16, device=dev, generator=gen)
    losses, norms, coefs = [], [], []
    for step in range(1, steps + 1):
        loss_sum = torch.zeros((), device=dev)
        for _ in range(micro_batches):
            x = torch.randn(batch, 16, device=dev, generator=gen)
            y = torch.sin(x @ target)[:, None]
            loss = (model(x.bfloat16()).float() - y).square().mean()
            loss.backward()  # adds to the .grad tensors
            loss_sum += loss.detach()
        if step % 10 == 0:
            absnt.abs_grad_norm(tensors, norm_type=math.inf)
            largest = float(tensors.norm)
            absnt.abs_grad_clip(tensors, 0.5 * largest, norm_type=math.inf)
        # the mean over the micro-batches and the clipping are part of the update
        absnt.abs_grad_adamw(tensors, hparams, step, max_norm, grad_scale=1.0 / micro_batches)
        losses.append(loss_sum / micro_batches)
        norms.append(tensors.norm.clone())
        coefs.append(tensors.coef.clone())
        for p in params:
            p.grad.zero_()
        if step % 10 == 0 and not quiet:
            print("step %3d  loss %.4f  norm %.3f  coef %.3f  largest |g| %.3g  tensors %s" % (
                step, float(losses[-1]), float(norms[-1]), float(coefs[-1]), largest,
                " ".join("%.2g" % x for x in tensors.norms.tolist())))
    return (torch.stack(x).tolist() for x in (losses, norms, coefs))


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    run(ap.parse_args().steps)
