"""Plain 64-bit implementations of the language-model operators, on the CPU, written from their formulas."""
import numpy as np
import torch

NEG = float("-inf")


def order(z_row):
    """Columns by falling logit, equal logits by rising index; masked columns left out."""
    z = z_row.double().numpy() + 0.0
    live = np.nonzero(z > NEG)[0]
    return live[np.lexsort((live, -z[live]))]


def log_softmax(z, scale):
    """(log p, lse) in 64 bits; an empty row has log p = lse = -inf, a NaN or +inf in a row makes it all NaN."""
    y = z.double() * scale
    m = y.amax(1, keepdim=True)
    empty = (m == NEG)
    shift = torch.where(empty, torch.zeros_like(m), m)
    ls = (y - shift).exp().sum(1, keepdim=True).log()
    lse = shift + ls
    lse = torch.where(empty, torch.full_like(m, NEG), lse)
    lse = torch.where(torch.isnan(y).any(1, keepdim=True) | (m == float("inf")), torch.full_like(m, float("nan")), lse)
    # y - lse, with the two parts of lse apart: beside a maximum of -3e38 the other one would be lost
    lp = torch.where(empty, torch.full_like(y, NEG), torch.where(torch.isfinite(lse), (y - shift) - ls, y - lse))
    return lp, lse[:, 0]


def token_logp(z, tokens, scale, top):
    lp, lse = log_softmax(z, scale)
    n = z.shape[0]
    p = lp.exp()
    entropy = -torch.where(p > 0, p * lp, torch.where(torch.isnan(p), p, torch.zeros_like(p))).sum(1)
    logp = torch.zeros(n, dtype=torch.float64)
    for i in range(n):
        t = int(tokens[i])
        logp[i] = 0.0 if t < 0 else lp[i, t]
    ids = torch.full((n, top), -1, dtype=torch.int64)
    tl = torch.full((n, top), NEG, dtype=torch.float64)
    for i in range(n):
        if torch.isnan(lse[i]):
            tl[i] = float("nan")
            continue
        o = torch.from_numpy(order(z[i])[:top])
        ids[i, :len(o)] = o
        tl[i, :len(o)] = lp[i, o]
    return logp, lse, entropy, ids, tl


def token_logp_grad(z, tokens, scale, g, h):
    lp, lse = log_softmax(z, scale)
    p = lp.exp()
    logp0 = torch.where(p > 0, lp, torch.zeros_like(lp))
    ent = -(p * logp0).sum(1, keepdim=True)
    g = torch.where(tokens < 0, torch.zeros_like(g), g).double()[:, None]
    hot = torch.zeros_like(p)
    for i, t in enumerate(tokens.tolist()):
        if t >= 0:
            hot[i, t] = 1.0
    out = scale * (g * (hot - p) - h.double()[:, None] * p * (logp0 + ent))
    return torch.where((lse == NEG)[:, None], torch.zeros_like(out), out)


def teacher(ids, u, teacher_scale, tail):
    """q (N, K) and q_T (N)."""
    a = torch.where(ids < 0, torch.full_like(u, NEG, dtype=torch.float64), u.double() * teacher_scale)
    if tail:
        q = a.exp()
        return q, (1.0 - q.sum(1)).clamp_min(0.0)
    m = a.amax(1, keepdim=True)
    w = (a - torch.where(m == NEG, torch.zeros_like(m), m)).exp()
    s = w.sum(1, keepdim=True)
    return torch.where(s > 0, w / s.clamp_min(1e-300), torch.zeros_like(w)), None


def distill(z, ids, u, scale, teacher_scale, tail):
    """(loss, lse, log_tail)."""
    lp, lse = log_softmax(z, scale)
    q, rest = teacher(ids, u, teacher_scale, tail)
    n, k = ids.shape
    loss = torch.zeros(n, dtype=torch.float64)
    log_tail = torch.zeros(n, dtype=torch.float64)
    for i in range(n):
        for j in range(k):
            if q[i, j] > 0:
                loss[i] += q[i, j] * (q[i, j].log() - lp[i, ids[i, j]])
        if tail:
            keep = torch.ones(z.shape[1], dtype=torch.bool)
            keep[ids[i][ids[i] >= 0].long()] = False
            log_tail[i] = torch.logsumexp(lp[i][keep], 0) if keep.any() else NEG
            if rest[i] > 0:
                loss[i] += rest[i] * (rest[i].log() - log_tail[i])
    return loss, lse, log_tail if tail else None


def distill_grad(z, ids, u, scale, teacher_scale, tail, weight):
    lp, lse = log_softmax(z, scale)
    p = lp.exp()
    q, rest = teacher(ids, u, teacher_scale, tail)
    out = torch.zeros_like(p)
    for i in range(z.shape[0]):
        if lse[i] == NEG:
            continue
        qv = torch.zeros(z.shape[1], dtype=torch.float64)
        inside = torch.zeros(z.shape[1], dtype=torch.bool)
        for j in range(ids.shape[1]):
            t = int(ids[i, j])
            if t >= 0:
                qv[t] += q[i, j]
                inside[t] = True
        d = p[i] * q[i].sum() - qv
        if tail and rest[i] > 0:
            share = torch.where(inside | (lp[i] == NEG), torch.zeros_like(p[i]), (lp[i] - torch.logsumexp(torch.where(inside, torch.full_like(lp[i], NEG), lp[i]), 0)).exp())
            d = d + rest[i] * (p[i] - share)
        out[i] = weight[i].double() * scale * d
    return out


def embed_grad(tokens, g, vocab, scale):
    """(gradient, sum of magnitudes, places) per table row; tokens (N), g (N, D)."""
    out = torch.zeros((vocab, g.shape[1]), dtype=torch.float64)
    mag = torch.zeros_like(out)
    cnt = torch.zeros(vocab, dtype=torch.int64)
    for i, t in enumerate(tokens.tolist()):
        if t >= 0:
            out[t] += scale * g[i].double()
            mag[t] += abs(scale) * g[i].double().abs()
            cnt[t] += 1
    return out, mag, cnt
