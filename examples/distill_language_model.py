"""Workers distil a small language model and exchange compressed updates.

R workers hold copies of a student, a bigram model with a tied embedding table and a bias per token, as rows of the
R x d batch that qs_bind takes.  A fixed teacher leaves, once, its top log probabilities for every token of the data
(qs_token_logp).  A local step of a worker is

    h      = embed(tokens, table)                       qs_embed, from the worker's own stretch of the batch
    logits = h table^T + bias                           torch
    loss, dlogits                                       qs_distill, the gradient in the logits' place
    dtable = dlogits^T h (+) embedding gradient of dlogits table, dbias      torch, qs_embed_grad accumulating
    the local step                                      qs_local_step, from the R x d gradients

and every `sync_every` steps qs_sync_round compresses the updates (Top_k, sign), aggregates and broadcasts.

    python examples/distill_language_model.py [--steps 60]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1906_02367_b200 import binding as B  # noqa: E402
from paper_1906_02367_b200 import lm  # noqa: E402


class Student:
    """Views of a flat (R, d) batch: the tied table (R, V, D) first, then the bias (R, V)."""

    def __init__(self, vocab, width):
        self.V, self.D = vocab, width
        self.d = vocab * width + vocab
        self.scale = math.sqrt(width)

    def views(self, flat):
        R = flat.shape[0]
        n = self.V * self.D
        return flat[:, :n].view(R, self.V, self.D), flat[:, n:]

    def gradient(self, flat, grad, tokens, ids, teacher_logp):
        """Loss per position (R N) and, in `grad`, every worker's gradient of its mean loss."""
        table, bias = self.views(flat)
        dtable, dbias = self.views(grad)
        R, N = tokens.shape
        h = lm.embed(tokens, table, scale=self.scale)
        logits = torch.baddbmm(bias[:, None, :], h, table.transpose(1, 2)).view(R * N, self.V)
        out = lm.distill(logits, ids, teacher_logp, tail=True, weight=1.0 / N, out=logits)
        dlogits = out.grad.view(R, N, self.V)
        torch.bmm(dlogits.transpose(1, 2), h, out=dtable)
        torch.sum(dlogits, 1, out=dbias)
        lm.embed_grad(tokens, torch.bmm(dlogits, table), self.V, scale=self.scale, accumulate=True, out=dtable)
        return out.loss


def teacher_entries(teacher, tokens, top):
    """A teacher's top log probabilities at every position: what travels instead of its logits."""
    logits = teacher[tokens.reshape(-1)]
    r = lm.token_logp(logits, top=top)
    return r.top_ids, r.top_logp


def run(R=4, vocab=1000, width=64, tokens=256, top=16, steps=60, sync_every=2, eta=20.0, seed=0, log=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    student = Student(vocab, width)
    teacher = torch.randn((vocab, vocab), generator=gen, device="cuda") * 2.5
    x = torch.randn(student.d, generator=gen, device="cuda") * 0.02
    xw = x.repeat(R, 1)
    mem = torch.zeros_like(xw)
    grad = torch.zeros_like(xw)
    ctx = B.Context(R, student.d, max(1, student.d // 50), 1, B.QS_TOPK, B.QS_SIGN_L1, seed=seed)
    ctx.bind(x, xw, mem)
    wire = ctx.new_wire()
    # every worker reads its own data, again and again
    data = torch.randint(0, vocab, (R, tokens), generator=gen, device="cuda")
    ids, teacher_logp = teacher_entries(teacher, data, top)
    losses = []
    for step in range(steps):
        loss = student.gradient(xw, grad, data, ids, teacher_logp)
        losses.append(loss.mean())
        if (step + 1) % sync_every:
            ctx.local_step(grad, eta)
        else:
            ctx.sync_round_step(wire, grad, eta)
        if log and step % 10 == 0:
            log(f"step {step:4d}  loss {float(losses[-1]):.4f}")
    if ctx.sync_status() != B.QS_OK:
        raise RuntimeError(ctx.last_error())
    # how the averaged model does: the teacher's favourite among the student's alternatives, and its entropy
    table, bias = student.views(x[None])
    h = lm.embed(data.view(-1), table[0], scale=student.scale)
    r = lm.token_logp(torch.addmm(bias[0], h, table[0].t()), ids[:, 0].contiguous(), top=5)
    agree = (r.top_ids == ids[:, :1]).any(1).float().mean()
    ctx.destroy()
    return {"losses": [float(v) for v in torch.stack(losses).cpu()], "in_top_5": float(agree), "entropy": float(r.entropy.mean()),
            "logp_of_favourite": float(r.logp.mean())}


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--workers", type=int, default=4)
    a = p.parse_args()
    got = run(R=a.workers, steps=a.steps, log=print)
    print(f"loss {got['losses'][0]:.4f} -> {got['losses'][-1]:.4f}; the teacher's favourite among the student's top 5 at "
          f"{100 * got['in_top_5']:.0f}% of the positions, mean entropy {got['entropy']:.3f}")
