"""Workers distil a small language model and exchange compressed updates.

R workers hold copies of a student, a bigram model with a tied embedding table and a bias per token, as rows of the
R x d batch that qs_bind takes.  A fixed teacher leaves, once, its top log probabilities for every token of the data
(qs_token_logp).  A local step of a worker is

    h      = embed(tokens, table)                       qs_embed, from the worker's own stretch of the batch
    logits = h table^T + bias                           torch
    loss, dlogits                                       qs_distill, the gradient in the logits' place
    dtable = dlogits^T h (+) embedding gradient of dlogits table, dbias      torch, qs_embed_grad accumulating
    the local step                                      qs_local_step, from the R x d gradients

and every `sync_every` steps qs_sync_round compresses the updates (Top_k, sign), aggregates and broadcasts.  With --blocks
there are residual blocks between the embedding and the logits, their parameters behind the others in the batch:

    h = h + dropout(gelu(norm(h) w1^T + b1) w2^T + b2)  qs_rms_norm, qs_linear, qs_dropout, and their gradients

    python examples/distill_language_model.py [--steps 60] [--blocks 2]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1906_02367_b200 import binding as B  # noqa: E402
from paper_1906_02367_b200 import layers, lm  # noqa: E402


class Student:
    """Views of a flat (R, d) batch: the tied table (R, V, D) first, then the bias (R, V), then per block the norm's weight (R, D),
    w1 (R, H, D), b1 (R, H), w2 (R, D, H) and b2 (R, D), H = 4 D."""

    def __init__(self, vocab, width, blocks=0, drop=0.1):
        self.V, self.D, self.H, self.blocks, self.drop = vocab, width, 4 * width, blocks, drop
        self.shapes = [(width,), (self.H, width), (self.H,), (width, self.H), (width,)]
        self.d = vocab * width + vocab + blocks * sum(math.prod(t) for t in self.shapes)
        self.scale = math.sqrt(width)

    def views(self, flat):
        R = flat.shape[0]
        n = self.V * self.D
        return flat[:, :n].view(R, self.V, self.D), flat[:, n:n + self.V]

    def block(self, flat, i):
        at, out = self.V * self.D + self.V + i * sum(math.prod(t) for t in self.shapes), []
        for t in self.shapes:
            out.append(flat[:, at:at + math.prod(t)].view(flat.shape[0], *t))
            at += math.prod(t)
        return out

    def start(self, flat):
        """Parameters of the blocks that a run starts from, in place: norms of one, biases of zero, w2 small."""
        for i in range(self.blocks):
            norm, w1, b1, w2, b2 = self.block(flat, i)
            norm.fill_(1.0), b1.zero_(), b2.zero_()
            w1.mul_(50.0 / math.sqrt(self.D)), w2.mul_(10.0 / math.sqrt(self.H))

    def hidden(self, flat, h, key=None):
        """The blocks' output, and what their gradients need; key (seed, round): with dropout."""
        saved = []
        for i in range(self.blocks):
            norm, w1, b1, w2, b2 = self.block(flat, i)
            n = layers.rms_norm(h, norm)
            a = layers.linear(n.out, w1, b1, activation="gelu", save=True)
            u = layers.linear(a.out, w2, b2, residual=None if key else h).out
            saved.append((n, a))
            h = layers.dropout(u, self.drop, key[0], round=key[1], layer=i, workers=True, residual=h) if key else u
        return h, saved

    def hidden_grad(self, flat, grad, dh, saved, key):
        """Gradients of the blocks into their stretches of `grad`; returns the embedding's."""
        for i in reversed(range(self.blocks)):
            norm, w1, b1, w2, b2 = self.block(flat, i)
            dnorm, dw1, db1, dw2, db2 = self.block(grad, i)
            n, a = saved[i]
            du = layers.dropout(dh, self.drop, key[0], round=key[1], layer=i, workers=True)
            da = layers.linear_grad(du, a.out, w2, bias=True, out_weight=dw2, out_bias=db2).x
            dn = layers.linear_grad(da, n.out, w1, a.pre, "gelu", bias=True, out_weight=dw1, out_bias=db1).x
            dh = layers.rms_norm_grad(dn, n.hidden, n.rstd, norm, grad_hidden=dh, out_weight=dnorm).hidden
        return dh

    def gradient(self, flat, grad, tokens, ids, teacher_logp, key=(0, 0)):
        """Loss per position (R N) and, in `grad`, every worker's gradient of its mean loss.  key: seed and round of the dropout."""
        table, bias = self.views(flat)
        dtable, dbias = self.views(grad)
        R, N = tokens.shape
        h, saved = self.hidden(flat, lm.embed(tokens, table, scale=self.scale), key)
        logits = torch.baddbmm(bias[:, None, :], h, table.transpose(1, 2)).view(R * N, self.V)
        out = lm.distill(logits, ids, teacher_logp, tail=True, weight=1.0 / N, out=logits)
        dlogits = out.grad.view(R, N, self.V)
        torch.bmm(dlogits.transpose(1, 2), h, out=dtable)
        torch.sum(dlogits, 1, out=dbias)
        dh = self.hidden_grad(flat, grad, torch.bmm(dlogits, table), saved, key)
        lm.embed_grad(tokens, dh, self.V, scale=self.scale, accumulate=True, out=dtable)
        return out.loss


def teacher_entries(teacher, tokens, top):
    """A teacher's top log probabilities at every position: what travels instead of its logits."""
    logits = teacher[tokens.reshape(-1)]
    r = lm.token_logp(logits, top=top)
    return r.top_ids, r.top_logp


def run(R=4, vocab=1000, width=64, tokens=256, top=16, steps=60, sync_every=2, eta=20.0, seed=0, blocks=0, log=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    student = Student(vocab, width, blocks)
    teacher = torch.randn((vocab, vocab), generator=gen, device="cuda") * 2.5
    x = torch.randn(student.d, generator=gen, device="cuda") * 0.02
    student.start(x[None])
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
        loss = student.gradient(xw, grad, data, ids, teacher_logp, key=(seed, step))
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
    h = lm.embed(data.view(1, -1), table, scale=student.scale)
    h = student.hidden(x[None], h)[0].view(-1, width)
    r = lm.token_logp(torch.addmm(bias[0], h, table[0].t()), ids[:, 0].contiguous(), top=5)
    agree = (r.top_ids == ids[:, :1]).any(1).float().mean()
    ctx.destroy()
    return {"losses": [float(v) for v in torch.stack(losses).cpu()], "in_top_5": float(agree), "entropy": float(r.entropy.mean()),
            "logp_of_favourite": float(r.logp.mean())}


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--workers", type=int, default=4)
    p.add_argument("--blocks", type=int, default=0)
    a = p.parse_args()
    got = run(R=a.workers, steps=a.steps, blocks=a.blocks, eta=2.0 if a.blocks else 20.0, log=print)
    print(f"loss {got['losses'][0]:.4f} -> {got['losses'][-1]:.4f}; the teacher's favourite among the student's top 5 at "
          f"{100 * got['in_top_5']:.0f}% of the positions, mean entropy {got['entropy']:.3f}")
