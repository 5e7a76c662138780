"""Measured cases of the operators between a language model's two ends: root-mean-square norm with the residual's
addition (also with an output in 8 bits), dropout from the counter-based generator, and matrix products with bias,
activation and residual, with their gradients.

Every case is one call that a training or serving loop makes.  `run` makes it either through the library
(`own`) or in a plain form of elementary torch operations in 32 bits; `exact` computes the same in 64 bits.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}
EPS = 1e-6
E4M3_MAX = 448.0


# ------------------------------------------------------------------ cases
def listed():
    return [
        # the norm in front of a layer in one decoding step: a few sequences, one token each
        dict(name="norm_step", op="norm", workers=1, rows=8, width=2048, type="bf16", weight="bf16", residual=True, quantize=False),
        # a prompt's rows on their way into a product in 8 bits
        dict(name="norm_8bit", op="norm", workers=1, rows=8192, width=4096, type="bf16", weight="bf16", residual=True, quantize=True),
        # the backward pass of eight workers' micro-batches, weights from the fp32 batch, with the residual stream's gradient
        dict(name="norm_grad_workers", op="norm_grad", workers=8, rows=4096, width=1024, type="bf16", weight="f32", residual=True),
        # a small model of odd width in 32 bits, one sequence
        dict(name="norm_grad_small", op="norm_grad", workers=1, rows=509, width=257, type="f32", weight="f32", residual=False),
        # one sequence of a small model
        dict(name="dropout_small", op="dropout", workers=1, rows=61, width=1000, type="f32", residual=False, p=0.25),
        # eight workers' micro-batches, added to the residual stream
        dict(name="dropout_workers", op="dropout", workers=8, rows=4096, width=1024, type="bf16", residual=True, p=0.1),
        # a product of one decoding step: bound by the weights
        dict(name="linear_step", op="linear", workers=1, rows=8, inner=2048, width=8192, type="bf16", weight="bf16", bias=False,
             residual=False, activation="silu", save=False),
        # eight workers' first product of a residual block, each with its own fp32 copy of the weights, kept for the backward pass
        dict(name="linear_workers", op="linear", workers=8, rows=4096, inner=1024, width=4096, type="bf16", weight="f32", bias=True,
             residual=False, activation="silu", save=True),
        # a small model in 32 bits: odd sizes, the second product with the residual
        dict(name="linear_small", op="linear", workers=1, rows=509, inner=257, width=1000, type="f32", weight="f32", bias=True,
             residual=True, activation=None, save=False),
        # a long prompt through a wide layer in 8 bits, a scale per row of both sides
        dict(name="linear_8bit", op="linear8", workers=1, rows=8192, inner=4096, width=16384, out="bf16", bias=True, residual=False,
             activation="gelu"),
        # the backward pass of eight workers' product, the weights' gradient in 32 bits
        dict(name="linear_grad_workers", op="linear_grad", workers=8, rows=4096, inner=1024, width=4096, type="bf16", weight="f32",
             activation="relu", grad="f32"),
        # the same of a small model in 32 bits
        dict(name="linear_grad_small", op="linear_grad", workers=1, rows=509, inner=257, width=1000, type="f32", weight="f32",
             activation="gelu", grad="f32"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm, odd more often than not."""
    v = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    if rng.random() < 0.6:
        v |= 1
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(("norm", "norm_grad", "dropout", "linear", "linear", "linear8", "linear_grad", "linear_grad"))
    type_ = rng.choice(("bf16", "bf16", "f16", "f32"))
    workers = 1 if op == "linear8" else rng.choice((1, 1, 2, 4, 8))
    if op in ("norm", "norm_grad", "dropout"):
        width = _spread(rng, 64, 8192)
        if rng.random() < 0.4:
            width = (width + 63) // 64 * 64
        rows = _spread(rng, 1, max(2, min(65536, 100_000_000 // (workers * width * SIZE[type_]))))
        c = dict(op=op, workers=workers, rows=rows, width=width, type=type_, residual=rng.random() < 0.6)
        if op == "dropout":
            return dict(c, p=rng.choice((0.1, 0.25, 0.5)))
        c["weight"] = rng.choice((type_, "f32"))
        if op == "norm":
            c["quantize"] = rng.random() < 0.4
        return c
    width, inner = _spread(rng, 64, 16384), _spread(rng, 64, 8192)
    if rng.random() < 0.5:                                        # most models' sizes are whole multiples
        width, inner = (width + 63) // 64 * 64, (inner + 63) // 64 * 64
    # a third of the largest listed case at most, a product in 32 bits less: several times the work
    most = (3e10 if type_ == "f32" and op != "linear8" else 1.8e11) / (workers * width * inner)
    rows = _spread(rng, 1, max(2, min(16384, int(most))))
    c = dict(op=op, workers=workers, rows=rows, inner=inner, width=width)
    activation = rng.choice((None, "relu", "silu", "gelu"))
    if op == "linear8":
        return dict(c, out=rng.choice(("bf16", "f16", "f32")), bias=rng.random() < 0.5, residual=rng.random() < 0.5, activation=activation)
    c.update(type=type_, weight=rng.choice((type_, "f32")))
    if op == "linear":
        return dict(c, bias=rng.random() < 0.5, residual=rng.random() < 0.5, activation=activation, save=rng.random() < 0.4)
    # with a smooth activation the gradient in front of it is rounded to 16 bits: then the weights' gradient comes in 16 bits too
    grad = "f32" if type_ == "f32" or activation in (None, "relu") else type_
    return dict(c, activation=activation, grad=grad)


# ------------------------------------------------------------------ inputs
def _shape(case, width):
    return (case["workers"], case["rows"], width) if case["workers"] > 1 else (case["rows"], width)


def _weight_shape(case, *shape):
    return (case["workers"], *shape) if case["workers"] > 1 else shape


def _normal(gen, shape, dtype, std=1.0, mean=0.0):
    return torch.empty(shape, device="cuda", dtype=dtype).normal_(mean, std, generator=gen)


def _to_8bit(v):
    """Values in 8 bits and the scale of each row."""
    scale = (v.abs().amax(-1) / E4M3_MAX).clamp_min(2.0 ** -126)
    return (v / scale[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 29)
    s = dict(case=dict(case))
    op = case["op"]
    dt = TYPES[case["type"]] if "type" in case else None
    if op in ("norm", "norm_grad", "dropout"):
        shape = _shape(case, case["width"])
        if op == "dropout":
            s["x"] = _normal(gen, shape, dt)
            s["residual"] = _normal(gen, shape, dt) if case["residual"] else None
            s["seed"], s["round"], s["layer"] = int(seed) * 7919 + (1 << 40), 3 + int(seed), 2
            return s
        s["weight"] = _normal(gen, _weight_shape(case, case["width"]), TYPES[case["weight"]], 0.1, 1.0)
        if op == "norm":
            s["x"] = _normal(gen, shape, dt)
            s["residual"] = _normal(gen, shape, dt, 2.0) if case["residual"] else None
        else:
            s["hidden"] = _normal(gen, shape, dt, 2.0)
            s["rstd"] = (s["hidden"].double().square().mean(-1) + EPS).rsqrt().float()
            s["grad"] = _normal(gen, shape, dt, 1e-2)
            s["grad_hidden"] = _normal(gen, shape, dt, 1e-2) if case["residual"] else None
        return s
    n, k, r = case["width"], case["inner"], case["rows"]
    if op == "linear8":
        s["x"], s["x_scale"] = _to_8bit(_normal(gen, (r, k), torch.float32))
        s["weight"], s["weight_scale"] = _to_8bit(_normal(gen, (n, k), torch.float32, k ** -0.5))
        s["bias"] = _normal(gen, (n,), torch.float32, 0.1) if case["bias"] else None
        s["residual"] = _normal(gen, (r, n), TYPES[case["out"]]) if case["residual"] else None
        return s
    s["x"] = _normal(gen, _shape(case, k), dt)
    s["weight"] = _normal(gen, _weight_shape(case, n, k), TYPES[case["weight"]], k ** -0.5)
    if op == "linear":
        s["bias"] = _normal(gen, _weight_shape(case, n), TYPES[case["weight"]], 0.1) if case["bias"] else None
        s["residual"] = _normal(gen, _shape(case, n), dt) if case["residual"] else None
    else:
        s["grad"] = _normal(gen, _shape(case, n), dt, 1e-2)
        s["pre"] = _normal(gen, _shape(case, n), dt) if case["activation"] else None
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    op = state["case"]["op"]
    return (_OWN if own else _PLAIN)[op](state, state["case"])


def _values(q, scale, dtype):
    """What 8 bits with a scale per row stand for."""
    return (q.float() * scale[..., None]).to(dtype)


def _own_norm(s, c):
    from paper_1906_02367_b200 import layers
    r = layers.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS, quantize=c["quantize"])
    out = [_values(r.out, r.scale, torch.bfloat16), r.scale] if c["quantize"] else [r.out]
    return out + [r.rstd] + ([r.hidden] if c["residual"] else [])


def _own_norm_grad(s, c):
    from paper_1906_02367_b200 import layers
    r = layers.rms_norm_grad(s["grad"], s["hidden"], s["rstd"], s["weight"], grad_hidden=s["grad_hidden"])
    return [r.hidden, r.weight]


def _own_dropout(s, c):
    from paper_1906_02367_b200 import layers
    return layers.dropout(s["x"], c["p"], s["seed"], round=s["round"], layer=s["layer"], residual=s["residual"], workers=c["workers"] > 1)


def _own_linear(s, c):
    from paper_1906_02367_b200 import layers
    r = layers.linear(s["x"], s["weight"], s["bias"], activation=c["activation"], residual=s["residual"], save=c["save"])
    return [r.out] + ([r.pre] if c["save"] else [])


def _own_linear8(s, c):
    from paper_1906_02367_b200 import layers
    return layers.linear(s["x"], s["weight"], s["bias"], activation=c["activation"], residual=s["residual"], x_scale=s["x_scale"],
                         weight_scale=s["weight_scale"], dtype=TYPES[c["out"]]).out


def _own_linear_grad(s, c):
    from paper_1906_02367_b200 import layers
    r = layers.linear_grad(s["grad"], s["x"], s["weight"], pre=s["pre"], activation=c["activation"], bias=True, dtype=TYPES[c["grad"]])
    return [r.x, r.weight, r.bias]


def _plain_norm(s, c):
    h = s["x"].float()
    if c["residual"]:
        h = (h + s["residual"].float()).to(s["x"].dtype)
        kept, h = h, h.float()
    rstd = 1.0 / (h.square().mean(-1) + EPS).sqrt()
    w = s["weight"].float()
    y = h * rstd[..., None] * (w[:, None] if c["workers"] > 1 else w)
    if c["quantize"]:
        scale = (y.abs().amax(-1) / E4M3_MAX).clamp_min(2.0 ** -126)
        q = (y / scale[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        out = [_values(q, scale, torch.bfloat16), scale]
    else:
        out = [y.to(s["x"].dtype)]
    return out + [rstd] + ([kept] if c["residual"] else [])


def _plain_norm_grad(s, c):
    w = s["weight"].float()
    g, n = s["grad"].float(), s["hidden"].float() * s["rstd"][..., None]
    wg = g * (w[:, None] if c["workers"] > 1 else w)
    dh = s["rstd"][..., None] * (wg - n * (wg * n).mean(-1, keepdim=True))
    if c["residual"]:
        dh = dh + s["grad_hidden"].float()
    return [dh.to(s["hidden"].dtype), (g * n).sum(-2)]


LOW = 0xFFFFFFFF


def _words(count, worker, seed, round_, layer, device):
    """The first `count` random words of each worker: Philox4x32-10, four words a counter, in whole numbers of 64 bits."""
    q = torch.arange((count + 3) // 4, device=device)
    c = [q, torch.full_like(q, worker), torch.full_like(q, round_ & LOW), torch.full_like(q, layer << 16 | (round_ >> 32 & 0xFF) << 8 | 2)]
    k0, k1 = seed & LOW, seed >> 32 & LOW
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32 & LOW) ^ c[1] ^ k0, b & LOW, (a >> 32 & LOW) ^ c[3] ^ k1, a & LOW]
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    return torch.stack(c, 1).reshape(-1)[:count]


def _plain_dropout(s, c):
    x = s["x"]
    count = c["rows"] * c["width"]
    border = int(c["p"] * 2.0 ** 32)
    keep = torch.stack([_words(count, w, s["seed"], s["round"], s["layer"], x.device) >= border for w in range(c["workers"])]).view(x.shape)
    out = torch.where(keep, x.float() * (1.0 / (1.0 - c["p"])), 0.0)
    return (out if s["residual"] is None else out + s["residual"].float()).to(x.dtype)


def _act(z, activation):
    if activation == "relu":
        return torch.where(z > 0, z, 0.0)
    if activation == "silu":
        return z / (1.0 + (-z).exp())
    if activation == "gelu":
        return 0.5 * z * (1.0 + (z * 0.5 ** 0.5).erf())
    return z


def _act_slope(z, activation):
    if activation == "relu":
        return (z > 0).float()
    if activation == "silu":
        p = 1.0 / (1.0 + (-z).exp())
        return p * (1.0 + z * (1.0 - p))
    return 0.5 * (1.0 + (z * 0.5 ** 0.5).erf()) + z * (-0.5 * z * z).exp() * (2.0 * math.pi) ** -0.5


def _plain_after(z, s, c, dtype):
    if s["bias"] is not None:
        b = s["bias"].float()
        z = z + (b[:, None] if c["workers"] > 1 else b)
    y = _act(z, c["activation"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return [y.to(dtype)] + ([z.to(dtype)] if c.get("save") else [])


def _plain_linear(s, c):
    dt = s["x"].dtype
    return _plain_after(s["x"].float() @ s["weight"].to(dt).float().transpose(-1, -2), s, c, dt)


def _plain_linear8(s, c):
    z = (s["x"].float() @ s["weight"].float().t()) * s["x_scale"][:, None] * s["weight_scale"]
    return _plain_after(z, s, c, TYPES[c["out"]])[0]


def _plain_linear_grad(s, c):
    dt = s["x"].dtype
    dz = s["grad"].float()
    if c["activation"]:
        dz = dz * _act_slope(s["pre"].float(), c["activation"])
    bias = dz.sum(-2)
    dz = dz.to(dt).float()                                        # the products' operand
    return [(dz @ s["weight"].to(dt).float()).to(dt), (dz.transpose(-1, -2) @ s["x"].float()).to(TYPES[c["grad"]]), bias]


_PLAIN = dict(norm=_plain_norm, norm_grad=_plain_norm_grad, dropout=_plain_dropout, linear=_plain_linear, linear8=_plain_linear8,
              linear_grad=_plain_linear_grad)
_OWN = dict(norm=_own_norm, norm_grad=_own_norm_grad, dropout=_own_dropout, linear=_own_linear, linear8=_own_linear8,
            linear_grad=_own_linear_grad)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, R, n, w = (case[k] for k in ("op", "workers", "rows", "width"))
    e = R * n * w
    if op in ("norm", "norm_grad", "dropout"):
        b = SIZE[case["type"]]
        if op == "dropout":
            return dict(bytes=e * b * (3 if case["residual"] else 2), flops=2 * e)
        weight = R * w * SIZE[case["weight"]]
        if op == "norm":
            out = e * 1 + 4 * R * n if case["quantize"] else e * b
            return dict(bytes=e * b * (3 if case["residual"] else 1) + out + weight + 4 * R * n, flops=5 * e)
        return dict(bytes=e * b * (4 if case["residual"] else 3) + weight + 4 * R * n + 4 * R * w, flops=9 * e)
    k = case["inner"]
    if op == "linear_grad":
        b = SIZE[case["type"]]
        moved = e * b * (2 if case["activation"] else 1) + 2 * R * n * k * b + R * w * k * (SIZE[case["weight"]] + SIZE[case["grad"]]) + 4 * R * w
        return dict(bytes=moved, flops=4 * e * k)
    b_in, b_w, b_out = (1, 1, SIZE[case["out"]]) if op == "linear8" else (SIZE[case["type"]], SIZE[case["weight"]], SIZE[case["type"]])
    outs = 1 + bool(case["residual"]) + bool(case.get("save"))
    b_bias = (4 if op == "linear8" else b_w) if case["bias"] else 0
    scales = 4 * (n + w) if op == "linear8" else 0
    return dict(bytes=R * n * k * b_in + R * w * k * b_w + e * b_out * outs + R * w * b_bias + scales, flops=2 * e * k)


# ------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    s, c = prepare(case, seed), case
    return _EXACT[c["op"]](s, c)


def _per_worker(t, c):
    return list(t) if c["workers"] > 1 else [t]


def _join(parts, c):
    return torch.stack(parts) if c["workers"] > 1 else parts[0]


def _exact_norm(s, c):
    outs = []
    for i, x in enumerate(_per_worker(s["x"], c)):
        h = x.double()
        if c["residual"]:
            h = (h + _per_worker(s["residual"], c)[i].double()).to(x.dtype).double()
        size = torch.linalg.vector_norm(h, dim=-1, keepdim=True)
        length = (size * size / c["width"] + EPS).sqrt()
        y = h / length * _per_worker(s["weight"], c)[i].double()
        if c["quantize"]:
            # the 8 bits round where they round: the values themselves are what they come near to
            outs.append((y, torch.linalg.vector_norm(y, ord=math.inf, dim=-1) / E4M3_MAX, 1.0 / length[..., 0], h))
        else:
            outs.append((y, 1.0 / length[..., 0], h))
    got = [_join(list(p), c) for p in zip(*outs)]
    if c["quantize"]:
        got[0] = None                                             # (a step of 8 bits is no error of the norm)
    return got if c["residual"] else got[:-1]


def _exact_norm_grad(s, c):
    outs = []
    for i, h in enumerate(_per_worker(s["hidden"], c)):
        g, rstd = _per_worker(s["grad"], c)[i].double(), _per_worker(s["rstd"], c)[i].double()[:, None]
        v = g * _per_worker(s["weight"], c)[i].double()
        h = h.double()
        along = (v * h).sum(1, keepdim=True) * rstd.pow(3) / c["width"]
        dh = v * rstd - h * along
        if c["residual"]:
            dh = dh + _per_worker(s["grad_hidden"], c)[i].double()
        outs.append((dh, torch.einsum("nd,nd,n->d", g, h, rstd[:, 0])))
    return [_join(list(p), c) for p in zip(*outs)]


def _words_apart(count, worker, seed, round_, layer):
    """The generator once more, on the host in numpy's unsigned numbers."""
    u = np.uint64
    low, half = u(LOW), u(32)
    x0 = np.arange((count + 3) // 4, dtype=u)
    x1, x2 = np.full_like(x0, worker), np.full_like(x0, round_ % 2 ** 32)
    x3 = np.full_like(x0, layer * 65536 + (round_ // 2 ** 32) % 256 * 256 + 2)
    key = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]
    for _ in range(10):
        m0, m1 = x0 * u(0xD2511F53), x2 * u(0xCD9E8D57)
        x0, x1, x2, x3 = (m1 >> half) ^ x1 ^ u(key[0]), m1 & low, (m0 >> half) ^ x3 ^ u(key[1]), m0 & low
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack([x0, x1, x2, x3], 1).reshape(-1)[:count]


def _exact_dropout(s, c):
    count, outs = c["rows"] * c["width"], []
    for i, x in enumerate(_per_worker(s["x"], c)):
        words = _words_apart(count, i, s["seed"], s["round"], s["layer"])
        dropped = torch.from_numpy(words < np.uint64(math.floor(c["p"] * 4294967296))).to(x.device).view(x.shape)
        y = (x.double() / (1.0 - c["p"])).masked_fill(dropped, 0.0)
        outs.append(y if s["residual"] is None else y + _per_worker(s["residual"], c)[i].double())
    return _join(outs, c)


def _act64(z, activation):
    if activation == "relu":
        return z.relu()
    if activation == "silu":
        return z * torch.special.expit(z)
    return z * torch.special.ndtr(z) if activation == "gelu" else z


def _exact_linear(s, c):
    outs = []
    for i, x in enumerate(_per_worker(s["x"], c)):
        w = _per_worker(s["weight"], c)[i].to(x.dtype).double()
        z = torch.einsum("mk,nk->mn", x.double(), w)
        if s["bias"] is not None:
            z += _per_worker(s["bias"], c)[i].double()
        y = _act64(z, c["activation"])
        if s["residual"] is not None:
            y = y + _per_worker(s["residual"], c)[i].double()
        outs.append((y, z))
    got = [_join(list(p), c) for p in zip(*outs)]
    return got if c["save"] else got[:1]


def _exact_linear8(s, c):
    out = []
    for a in range(0, c["rows"], 2048):
        x = s["x"][a:a + 2048].double() * s["x_scale"][a:a + 2048, None].double()
        z = torch.einsum("mk,nk->mn", x, s["weight"].double() * s["weight_scale"][:, None].double())
        if s["bias"] is not None:
            z += s["bias"].double()
        z = _act64(z, c["activation"])
        if s["residual"] is not None:
            z = z + s["residual"][a:a + 2048].double()
        out.append(z)
    return torch.cat(out)


def _exact_linear_grad(s, c):
    outs = []
    for i, x in enumerate(_per_worker(s["x"], c)):
        dz = _per_worker(s["grad"], c)[i].double()
        if c["activation"]:
            z = _per_worker(s["pre"], c)[i].double().requires_grad_()
            with torch.enable_grad():
                (slope,) = torch.autograd.grad(_act64(z, c["activation"]).sum(), z)
            dz = dz * slope
        bias = dz.sum(0)
        dz = dz.to(x.dtype).double()
        w = _per_worker(s["weight"], c)[i].to(x.dtype).double()
        outs.append((torch.einsum("mn,nk->mk", dz, w), torch.einsum("mn,mk->nk", dz, x.double()), bias))
    return [_join(list(p), c) for p in zip(*outs)]


_EXACT = dict(norm=_exact_norm, norm_grad=_exact_norm_grad, dropout=_exact_dropout, linear=_exact_linear, linear8=_exact_linear8,
              linear_grad=_exact_linear_grad)
