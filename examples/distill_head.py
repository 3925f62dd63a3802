"""Teaches a local head's vocabulary matrix from a teacher's top entries, and scores tokens before and after.

The teacher's rows of logits give, through token_logprobs, the K most likely tokens of every position with their log
probabilities: all that is kept of it.  The student's logits are rho W^T, with fixed low-rank states rho (in a local head
SiLU(W_rank h)); head_distill computes the loss and the gradient by W without storing them, and Adam keeps a float32 copy of
W.  (The K entries are not all of the teacher, so the loss, a part of a divergence, may fall below 0.)  At the end it is
computed once more from stored logits (distill_loss), and the log probability that the student gives the teacher's first
choice is compared with what it was.

    python examples/distill_head.py [--rows 1024] [--vocab 32003] [--rank 128] [--top-k 32] [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_07409_amd import binding as B  # noqa: E402


def first_choice_logprob(rho, w, first):
    """Mean log probability of the given tokens under the student, with its entropy."""
    stats, _, _ = B.token_logprobs((rho.float() @ w.float().T), first)
    return stats[:, 0].mean().item(), stats[:, 1].mean().item()


def run(rows=1024, vocab=32003, rank=128, top_k=32, steps=60, temperature=1.0, seed=0, quiet=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, device="cuda", generator=g)   # noqa: E731
    rho = normal(rows, rank).bfloat16()
    # a teacher that the student can follow: another matrix over the same states, and what the states do not say
    teacher = (rho.float() @ (normal(vocab, rank) * 3 / rank ** 0.5).T + 0.3 * normal(rows, vocab)).bfloat16()
    _, ids, logprobs = B.token_logprobs(teacher, top_k=top_k, temperature=temperature)
    del teacher

    master = torch.nn.Parameter(normal(vocab, rank) * 0.02)
    adam = torch.optim.Adam([master], lr=0.05)
    weight = torch.full((rows,), 1.0 / rows, device="cuda")   # the mean over the rows
    teach = dict(temperature=temperature, renormalise=False)
    before = first_choice_logprob(rho, master.detach().bfloat16(), ids[:, 0].contiguous())
    losses = []
    for step in range(steps):
        w = master.detach().bfloat16()
        loss, _, _, d_w = B.head_distill(rho, w, ids, logprobs, grad_loss=weight, want_grads=True, **teach)
        master.grad = d_w.float()
        adam.step()
        losses.append(loss.mean())
        if not quiet and step % 10 == 0:
            print(f"step {step:3d}  loss {losses[-1].item():.4f}", flush=True)
    w = master.detach().bfloat16()
    losses.append(B.head_distill(rho, w, ids, logprobs, **teach)[0].mean())
    losses = [x.item() for x in losses]
    stored = B.distill_loss(rho.float() @ w.float().T, ids, logprobs, **teach)[0].mean().item()
    after = first_choice_logprob(rho, w, ids[:, 0].contiguous())
    if not quiet:
        print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} (from stored logits {stored:.4f})")
        print(f"log probability of the teacher's first choice {before[0]:.3f} -> {after[0]:.3f}, entropy {before[1]:.3f} -> {after[1]:.3f}")
    return dict(losses=losses, stored=stored, before=before, after=after)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("rows", 1024), ("vocab", 32003), ("rank", 128), ("top-k", 32), ("steps", 60), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    run(**vars(ap.parse_args()))
