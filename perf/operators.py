"""Measured cases of the language-model operators: embedding rows and their gradient, log probabilities of
given tokens with entropy and top alternatives, distillation from a teacher's top logits, in both directions.

Every case is one call that a training or serving loop makes.  `run` makes it either through the library
(`own`) or in a plain form of elementary torch operations in 32 bits; `exact` computes the same in 64 bits.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
IDS = {"i32": torch.int32, "i64": torch.int64}
NEG = float("-inf")


# ------------------------------------------------------------------ cases
def listed():
    return [
        # the input of one decoding step: a few sequences, one token each
        dict(name="embed_step", op="embed", workers=1, tokens=8, vocab=32000, width=1024, table="bf16", out="bf16",
             ids="i64", scale=32.0),
        # eight workers' micro-batches, each from its own fp32 copy of the model
        dict(name="embed_workers", op="embed", workers=8, tokens=4096, vocab=32000, width=1024, table="f32", out="bf16",
             ids="i64", scale=32.0),
        # a small model of odd width, one sequence
        dict(name="embed_grad_small", op="embed_grad", workers=1, tokens=509, vocab=8191, width=257, grad="f32", ids="i32",
             scale=1.0),
        # eight workers' gradients of their embedding tables
        dict(name="embed_grad_workers", op="embed_grad", workers=8, tokens=4096, vocab=32000, width=1024, grad="bf16",
             ids="i64", scale=32.0),
        # a large vocabulary and a long batch on one worker: the frequent tokens come thousands of times
        dict(name="embed_grad_large", op="embed_grad", workers=1, tokens=65536, vocab=128000, width=2048, grad="bf16",
             ids="i64", scale=1.0),
        # one token of one sequence, with the alternatives that a serving program reports
        dict(name="logp_step", op="logp", rows=1, vocab=128000, pad=0, type="bf16", ids="i64", top=8, scale=1.25),
        # a teacher's pass that keeps its top logits; odd vocabulary, rows padded with masked columns
        dict(name="logp_teacher", op="logp", rows=4096, vocab=50003, pad=173, type="bf16", ids="i64", top=64, scale=0.5),
        # log probabilities of a long batch at a large vocabulary, as policy training reads them
        dict(name="logp_large", op="logp", rows=8192, vocab=128000, pad=0, type="bf16", ids="i64", top=0, scale=1.0),
        # their gradient, with an entropy bonus, in 32 bits
        dict(name="logp_grad", op="logp_grad", rows=2048, vocab=32000, pad=0, type="f32", ids="i64", scale=1.0),
        # distillation of a small classifier head (the 1000 classes of the ResNet-50 table), with the tail bucket
        dict(name="distill_small", op="distill", rows=61, vocab=1000, pad=0, type="f32", ids="i32", top=8, teacher="f32",
             scale=0.5, tail=True, step=True),
        # the loss and its gradient of a training step at a large vocabulary
        dict(name="distill_step", op="distill", rows=6144, vocab=128000, pad=0, type="bf16", ids="i64", top=64, teacher="f32",
             scale=1.0, tail=False, step=True),
        # the backward pass alone, from weights that are known only after the loss
        dict(name="distill_grad", op="distill_grad", rows=2048, vocab=50003, pad=0, type="bf16", ids="i64", top=32,
             teacher="bf16", scale=0.5, tail=True),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm, odd more often than not."""
    v = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    if rng.random() < 0.6:
        v |= 1
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "logp", "logp_grad", "distill", "distill_grad"))
    ids = rng.choice(("i32", "i64"))
    if op in ("embed", "embed_grad"):
        workers = rng.choice((1, 1, 2, 4, 8))
        width = _spread(rng, 64, 4096)
        vocab = _spread(rng, 1000, max(1001, min(256000, 260_000_000 // (workers * width))))
        tokens = _spread(rng, 1, max(2, min(65536, 130_000_000 // (workers * width))))
        c = dict(op=op, workers=workers, tokens=tokens, vocab=vocab, width=width)
        if op == "embed":
            c.update(table=rng.choice(("f32", "bf16", "f16")), out=rng.choice(("f32", "bf16")))
        else:
            c.update(grad=rng.choice(("f32", "bf16")))
        return dict(c, ids=ids, scale=rng.choice((1.0, 16.0, 32.0)))
    vocab = _spread(rng, 1000, 256000)
    type_ = rng.choice(("f32", "bf16", "bf16", "f16"))
    rows = _spread(rng, 1, max(2, min(65536, 800_000_000 // (vocab * SIZE[type_]))))
    c = dict(op=op, rows=rows, vocab=vocab, pad=rng.choice((0, 0, 64, 173)), type=type_, ids=ids,
             scale=rng.choice((0.5, 1.0, 1.25)))
    if op == "logp":
        c.update(top=rng.choice((0, 1, 8, 20, 64)))
    if op in ("distill", "distill_grad"):
        c.update(top=rng.choice((1, 8, 32, 64, 100)), teacher=rng.choice(("f32", "bf16")), tail=rng.random() < 0.5)
    if op == "distill":
        c.update(step=rng.random() < 0.7)
    return c


# ------------------------------------------------------------------ inputs
def _tokens(shape, vocab, gen, dtype, padding=0.0):
    """Token ids as text has them: frequency falls as one over the rank, low ids first; some places are padding (-1)."""
    u = torch.rand(shape, generator=gen, device="cuda", dtype=torch.float64)
    t = torch.clamp((u * math.log(vocab + 1)).exp().long() - 1, 0, vocab - 1)
    if padding:
        t = torch.where(torch.rand(shape, generator=gen, device="cuda") < padding, -1, t)
    return t.to(dtype)


def _logits(case, gen, tokens):
    """Logits of a trained model: a broad floor and a raised given token; the last `pad` columns are masked, and rows
    are views of rows that long."""
    n, v, pad = case["rows"], case["vocab"], case["pad"]
    z = torch.empty((n, v + pad), device="cuda", dtype=TYPES[case["type"]])
    z.normal_(0.0, 2.5, generator=gen)
    up = torch.rand((n, 1), generator=gen, device="cuda") * 14.0
    z.scatter_(1, tokens.long().clamp_min(0)[:, None], up.to(z.dtype))
    z = z[:, :v]
    if pad:
        z[:, v - v // 50:] = NEG
    return z


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 17)
    s = dict(case=dict(case))
    op, idt = case["op"], IDS[case["ids"]]
    if op in ("embed", "embed_grad"):
        R, n, v, w = (case[k] for k in ("workers", "tokens", "vocab", "width"))
        s["tokens"] = _tokens((R, n), v, gen, idt, 0.02)
        if op == "embed":
            s["table"] = torch.empty((R, v, w), device="cuda", dtype=TYPES[case["table"]]).normal_(0.0, 0.02, generator=gen)
        else:
            s["grad_out"] = torch.empty((R, n, w), device="cuda", dtype=TYPES[case["grad"]]).normal_(0.0, 1e-3, generator=gen)
        return s
    n, v = case["rows"], case["vocab"]
    live = v - v // 50 if case["pad"] else v                      # columns that are not masked
    tokens = _tokens((n,), live, gen, idt, 0.02 if n > 16 else 0.0)
    s["logits"] = _logits(case, gen, tokens)
    if op in ("logp", "logp_grad"):
        s["tokens"] = tokens
    if op == "logp_grad":
        # what the forward pass left: the log of the sum and the entropy
        lse, h = _lse_entropy(s["logits"], case["scale"])
        s["lse"], s["entropy"] = lse, h
        s["grad_logp"] = torch.randn(n, generator=gen, device="cuda") / n
        s["grad_entropy"] = torch.full((n,), -0.01 / n, device="cuda")
    if op in ("distill", "distill_grad"):
        k = case["top"]
        # distinct ids, spread over the vocabulary; a teacher's values fall with the rank; a few rows have fewer
        start = torch.randint(0, live, (n, 1), generator=gen, device="cuda")
        step = 1 + torch.randint(0, max(1, live // k - 1), (n, 1), generator=gen, device="cuda")
        at = torch.arange(k, device="cuda")[None, :]
        ids = (start + step * at) % live
        t = torch.rand((n, k), generator=gen, device="cuda").sort(dim=1, descending=True).values * 6.0
        if case["tail"]:                                          # log probabilities that leave some of the mass
            left = 0.02 + 0.3 * torch.rand((n, 1), generator=gen, device="cuda")
            t = t - t.exp().sum(1, keepdim=True).log() + torch.log1p(-left)
        else:
            t = t + 8.0
        if k > 1 and n > 16:
            ids = torch.where((torch.rand((n, 1), generator=gen, device="cuda") < 0.03) & (at >= k // 2), -1, ids)
        s["ids"], s["teacher"] = ids.to(idt), t.to(TYPES[case["teacher"]])
        s["weight"] = torch.rand(n, generator=gen, device="cuda") / n
        if op == "distill_grad":
            s["lse"], _ = _lse_entropy(s["logits"], case["scale"])
            s["log_tail"] = _log_tail(s["logits"], s["ids"], case["scale"], s["lse"]) if case["tail"] else None
    return s


def _chunks(n, v, most=1 << 27):
    """Row ranges of at most `most` elements."""
    step = max(1, most // v)
    return [(a, min(n, a + step)) for a in range(0, n, step)]


def _lse_entropy(logits, scale):
    """What a forward pass leaves for the backward one, rounded from 64 bits."""
    lse, ent = [], []
    for a, b in _chunks(*logits.shape):
        z = logits[a:b].double() * scale
        m = z.amax(1, keepdim=True)
        e = (z - m).exp()
        s = e.sum(1, keepdim=True)
        lse.append((m + s.log())[:, 0])
        ent.append((s.log() - (e * (z - m).clamp_min(-1e30)).sum(1, keepdim=True) / s)[:, 0])
    return torch.cat(lse).float(), torch.cat(ent).float()


def _log_tail(logits, ids, scale, lse):
    out = []
    for a, b in _chunks(*logits.shape):
        p = (logits[a:b].double() * scale - lse[a:b, None].double()).exp()
        out.append((p * ~_member(ids[a:b], p.shape[1])).sum(1).log())
    return torch.cat(out).float()


def _member(ids, vocab):
    """True where a column is among the row's ids; negative ids name none."""
    m = torch.zeros((ids.shape[0], vocab + 1), dtype=torch.bool, device=ids.device)
    m.scatter_(1, torch.where(ids < 0, vocab, ids).long(), True)
    return m[:, :vocab]


# ------------------------------------------------------------------ one pass
def run(state):
    op = state["case"]["op"]
    return (_OWN if own else _PLAIN)[op](state, state["case"])


def _own_embed(s, c):
    from paper_1906_02367_b200 import lm
    return lm.embed(s["tokens"], s["table"], scale=c["scale"], dtype=TYPES[c["out"]])


def _own_embed_grad(s, c):
    from paper_1906_02367_b200 import lm
    return lm.embed_grad(s["tokens"], s["grad_out"], c["vocab"], scale=c["scale"])


def _own_logp(s, c):
    from paper_1906_02367_b200 import lm
    r = lm.token_logp(s["logits"], s["tokens"], scale=c["scale"], top=c["top"])
    return [r.logp, r.lse, r.entropy] + ([r.top_ids, r.top_logp] if c["top"] else [])


def _own_logp_grad(s, c):
    from paper_1906_02367_b200 import lm
    return lm.token_logp_grad(s["logits"], s["tokens"], s["lse"], s["grad_logp"], scale=c["scale"], entropy=s["entropy"],
                              grad_entropy=s["grad_entropy"])


def _own_distill(s, c):
    from paper_1906_02367_b200 import lm
    r = lm.distill(s["logits"], s["ids"], s["teacher"], scale=c["scale"], tail=c["tail"],
                   weight=s["weight"] if c["step"] else None)
    return [r.loss, r.lse] + ([r.log_tail] if c["tail"] else []) + ([r.grad] if c["step"] else [])


def _own_distill_grad(s, c):
    from paper_1906_02367_b200 import lm
    return lm.distill_grad(s["logits"], s["ids"], s["teacher"], s["lse"], s["weight"], scale=c["scale"], tail=c["tail"],
                           log_tail=s["log_tail"])


def _plain_embed(s, c):
    tok = s["tokens"].long()
    worker = torch.arange(tok.shape[0], device=tok.device)[:, None]
    rows = s["table"][worker, tok.clamp_min(0)].float() * c["scale"]
    return torch.where(tok[..., None] < 0, 0.0, rows).to(TYPES[c["out"]])


def _plain_embed_grad(s, c):
    tok, v = s["tokens"].long(), c["vocab"]
    R, n = tok.shape
    key = torch.where(tok < 0, R * v, tok + v * torch.arange(R, device=tok.device)[:, None])
    g = s["grad_out"].float().reshape(R * n, -1) * c["scale"]
    out = torch.zeros((R * v + 1, g.shape[1]), device=g.device)
    out.index_add_(0, key.reshape(-1), g)
    return out[: R * v].view(R, v, -1)


def _plain_logp(s, c):
    tok, k = s["tokens"].long(), c["top"]
    z = s["logits"].float() * c["scale"]
    m = z.amax(1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(1, keepdim=True)
    lse = m + total.log()
    logp = torch.where(tok < 0, 0.0, (z.gather(1, tok.clamp_min(0)[:, None]) - m - total.log())[:, 0])
    p = e / total
    entropy = -torch.where(p > 0, p * (z - lse), 0.0).sum(1)
    out = [logp, lse[:, 0], entropy]
    if k:
        # one whole number that orders by logit (larger first), then by index (lower first)
        bits = s["logits"].float().view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        key = order * (1 << 20) - torch.arange(z.shape[1], device=z.device)
        ids = z.shape[1] - 1 - (key.topk(k, dim=1).values + z.shape[1] - 1) % (1 << 20)
        out += [ids.to(s["tokens"].dtype), z.gather(1, ids) - m - total.log()]
    return out


def _plain_logp_grad(s, c):
    tok = s["tokens"].long()
    z = s["logits"].float() * c["scale"]
    logp = z - s["lse"][:, None]
    p = logp.exp()
    gl = torch.where(tok < 0, 0.0, s["grad_logp"])[:, None]
    g = -p * gl - s["grad_entropy"][:, None] * torch.where(p > 0, p * (logp + s["entropy"][:, None]), 0.0)
    g.scatter_add_(1, tok.clamp_min(0)[:, None], gl)
    return (g * c["scale"]).to(s["logits"].dtype)


def _teacher(s, c):
    """The teacher's probabilities of the given ids, their logs, and the mass that they leave."""
    t = torch.where(s["ids"] < 0, NEG, s["teacher"].float())
    if c["tail"]:
        q = t.exp()
        return q, t, (1.0 - q.sum(1)).clamp_min(0.0)
    m = t.amax(1, keepdim=True).clamp_min(-3e38)
    e = (t - m).exp()
    total = e.sum(1, keepdim=True).clamp_min(1e-38)
    return e / total, t - m - total.log(), None


def _plain_distill_grad_of(s, c, p, q, q_tail, p_tail):
    v = p.shape[1]
    a = q.sum(1)
    if c["tail"]:
        a = a + q_tail
        ratio = torch.where(q_tail > 0, q_tail / p_tail, 0.0)
        coef = a[:, None] - torch.where(_member(s["ids"], v), 0.0, ratio[:, None])
    else:
        coef = a[:, None]
    g = torch.cat([p * coef, torch.zeros_like(p[:, :1])], 1)
    g.scatter_add_(1, torch.where(s["ids"] < 0, v, s["ids"]).long(), -q)
    return (g[:, :v] * (s["weight"] * c["scale"])[:, None]).to(s["logits"].dtype)


def _plain_distill(s, c):
    z = s["logits"].float() * c["scale"]
    m = z.amax(1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(1, keepdim=True)
    lse = m + total.log()
    q, logq, q_tail = _teacher(s, c)
    logp = z.gather(1, s["ids"].long().clamp_min(0)) - lse
    loss = torch.where(q > 0, q * (logq - logp), 0.0).sum(1)
    out, p_tail = [lse[:, 0]], None
    if c["tail"]:
        # log of the share outside the ids, from both sums: near 1 the difference of two logs would cancel
        named = _member(s["ids"], z.shape[1])
        log_tail = -torch.log1p(torch.where(named, e, 0.0).sum(1) / torch.where(named, 0.0, e).sum(1))
        p_tail = log_tail.exp()
        loss = loss + torch.where(q_tail > 0, q_tail * (q_tail.log() - log_tail), 0.0)
        out.append(log_tail)
    out = [loss] + out
    if c["step"]:
        out.append(_plain_distill_grad_of(s, c, e / total, q, q_tail, p_tail))
    return out


def _plain_distill_grad(s, c):
    p = (s["logits"].float() * c["scale"] - s["lse"][:, None]).exp()
    q, _, q_tail = _teacher(s, c)
    return _plain_distill_grad_of(s, c, p, q, q_tail, s["log_tail"].exp() if c["tail"] else None)


_PLAIN = dict(embed=_plain_embed, embed_grad=_plain_embed_grad, logp=_plain_logp, logp_grad=_plain_logp_grad,
              distill=_plain_distill, distill_grad=_plain_distill_grad)
_OWN = dict(embed=_own_embed, embed_grad=_own_embed_grad, logp=_own_logp, logp_grad=_own_logp_grad, distill=_own_distill,
            distill_grad=_own_distill_grad)


# ------------------------------------------------------------------ what a pass cannot do without
def _distinct(tokens, vocab):
    """Distinct rows that `tokens` draws of _tokens name, in expectation."""
    edge = np.log(np.arange(1, vocab + 2)) / math.log(vocab + 1)
    return float(np.sum(-np.expm1(0.98 * tokens * np.log1p(-np.minimum(np.diff(edge), 1 - 1e-12)))))


def work(case):
    op, idb = case["op"], 4 if case["ids"] == "i32" else 8
    if op in ("embed", "embed_grad"):
        R, n, v, w = (case[k] for k in ("workers", "tokens", "vocab", "width"))
        if op == "embed":
            return dict(bytes=R * (n * idb + _distinct(n, v) * w * SIZE[case["table"]] + n * w * SIZE[case["out"]]), flops=R * n * w)
        return dict(bytes=R * (n * idb + n * w * SIZE[case["grad"]] + v * w * 4), flops=2 * R * n * w)
    n, v, b = case["rows"], case["vocab"], SIZE[case["type"]]
    if op == "logp":
        return dict(bytes=n * (v * b + idb + 12 + case["top"] * (idb + 4)), flops=6 * n * v)
    if op == "logp_grad":
        return dict(bytes=n * (2 * v * b + idb + 16), flops=6 * n * v)
    k = case["top"] * (idb + SIZE[case["teacher"]])
    if op == "distill":
        return dict(bytes=n * (v * b * (2 if case["step"] else 1) + k + 16), flops=(8 if case["step"] else 4) * n * v)
    return dict(bytes=n * (2 * v * b + k + 12), flops=4 * n * v)


# ------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    s, c = prepare(case, seed), case
    op = c["op"]
    if op == "embed":
        tok = s["tokens"].long()
        out = torch.zeros((*tok.shape, c["width"]), dtype=torch.float64, device=tok.device)
        r, i = (tok >= 0).nonzero(as_tuple=True)
        out[r, i] = s["table"].double()[r, tok[r, i]] * c["scale"]
        return out
    if op == "embed_grad":
        R, v, w = c["workers"], c["vocab"], c["width"]
        out = torch.zeros((R, v, w), dtype=torch.float64, device=s["tokens"].device)
        for r in range(R):                                       # runs of equal tokens: differences of running sums
            keep = (s["tokens"][r] >= 0).nonzero()[:, 0]
            tok, at = s["tokens"][r][keep].long().sort(stable=True)
            if not tok.numel():
                continue
            ids, count = tok.unique_consecutive(return_counts=True)
            run_ = s["grad_out"][r][keep[at]].double().cumsum(0)
            end = count.cumsum(0)
            upto = run_[end - 1]
            out[r, ids] = c["scale"] * torch.cat([upto[:1], upto[1:] - upto[:-1]])
        return out
    parts = [_EXACT[op](s, c, a, b) for a, b in _chunks(c["rows"], c["vocab"])]
    if isinstance(parts[0], torch.Tensor):
        return torch.cat(parts)
    return [None if p[0] is None else torch.cat(p) for p in zip(*parts)]


def _logp64(s, c, a, b):
    z = s["logits"][a:b].double() * c["scale"]
    return z, torch.log_softmax(z, 1)


def _exact_logp(s, c, a, b):
    z, lp = _logp64(s, c, a, b)
    tok = s["tokens"][a:b].long()
    row = torch.arange(b - a, device=tok.device)
    logp = torch.where(tok < 0, 0.0, lp[row, tok.clamp_min(0)])
    out = [logp, torch.logsumexp(z, 1), torch.special.entr(lp.exp()).sum(1)]
    if c["top"]:
        out += [None, lp.sort(1, descending=True).values[:, : c["top"]].clone()]
    return out


def _exact_logp_grad(s, c, a, b):
    # from the definition: the derivative of g . logp + h . entropy, the probabilities' own sums taken anew
    z, lp = _logp64(s, c, a, b)
    tok, p = s["tokens"][a:b].long(), lp.exp()
    ent = torch.special.entr(p).sum(1, keepdim=True)
    g = s["grad_logp"][a:b].double() * (tok >= 0)
    out = -p * g[:, None] + s["grad_entropy"][a:b].double()[:, None] * (torch.special.entr(p) - p * ent)
    row = (tok >= 0).nonzero()[:, 0]
    out[row, tok[row]] += g[row]
    return out * c["scale"]


def _dense_teacher64(s, c, a, b):
    """The teacher's distribution as a dense row, and the mass outside the ids."""
    ids, t = s["ids"][a:b].long(), s["teacher"][a:b].double()
    row, col = (ids >= 0).nonzero(as_tuple=True)
    w = torch.zeros((b - a, c["vocab"]), dtype=torch.float64, device=ids.device)
    w[row, ids[row, col]] = t[row, col].exp()
    inside = torch.zeros_like(w, dtype=torch.bool)
    inside[row, ids[row, col]] = True
    if c["tail"]:
        return w, inside, (1.0 - w.sum(1, keepdim=True)).clamp_min(0.0)
    return w / w.sum(1, keepdim=True), inside, None


def _exact_distill(s, c, a, b):
    z, lp = _logp64(s, c, a, b)
    q, inside, rest = _dense_teacher64(s, c, a, b)
    p = lp.exp()
    loss = torch.where(q > 0, torch.special.xlogy(q, q) - q * lp, 0.0).sum(1)
    out, log_tail = [torch.logsumexp(z, 1)], None
    if c["tail"]:
        log_tail = torch.logsumexp(lp.masked_fill(inside, NEG), 1)
        loss = loss + torch.special.xlogy(rest[:, 0], rest[:, 0]) - rest[:, 0] * log_tail
        out.append(log_tail)
    out = [loss] + out
    return out + [_distill_grad64(s, c, a, b, p, q, inside, rest)] if c["step"] else out


def _distill_grad64(s, c, a, b, p, q, inside, rest):
    g = p * q.sum(1, keepdim=True) - q
    if c["tail"]:                                                # the tail is one more class, whose mass is the sum of its members'
        out = p.masked_fill(inside, 0.0)
        g = g + rest * (p - out / out.sum(1, keepdim=True))
    return g * (s["weight"][a:b].double() * c["scale"])[:, None]


def _exact_distill_grad(s, c, a, b):
    _, lp = _logp64(s, c, a, b)
    return _distill_grad64(s, c, a, b, lp.exp(), *_dense_teacher64(s, c, a, b))


_EXACT = dict(logp=_exact_logp, logp_grad=_exact_logp_grad, distill=_exact_distill, distill_grad=_exact_distill_grad)
