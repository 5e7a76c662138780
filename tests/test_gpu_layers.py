"""The operators of a residual block on the GPU, against plain implementations in 64 bits.

Bounds: a result rounded to its type is off by at most half a step, U[type] of its magnitude; a sum of n terms in fp32 is off
by at most n 2^-23 of the sum of magnitudes, whether additions round to nearest or cut (the matrix unit cuts); products of
16- and 8-bit elements are exact in fp32.
"""
import numpy as np
import pytest
import torch

import layers_reference as ref

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}        # a step among the smallest numbers
E = 2.0 ** -23


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.fixture
def L():
    from paper_1906_02367_b200 import layers
    return layers


def rand(shape, dtype=F32, seed=0, std=1.0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)


def wide(t, pad, offset=0):
    """The same values as a view of rows that are `pad` elements longer, `offset` elements into memory."""
    rows = t.reshape(-1, t.shape[-1])
    buf = torch.full((offset + rows.shape[0] * (t.shape[-1] + pad) + 8,), 7.0, device="cuda", dtype=F32).to(t.dtype)
    v = buf[offset:offset + rows.shape[0] * (t.shape[-1] + pad)].view(rows.shape[0], -1)[:, :t.shape[-1]]
    v.copy_(rows)
    return v.view(*t.shape[:-1], t.shape[-1]) if t.dim() == 2 else v.unflatten(0, t.shape[:-1])


def near(got, want, slack, dtype):
    """|got - want| <= slack + half a step of `dtype`."""
    got, want = got.double(), want.double()
    bad = (got - want).abs() > slack + U[dtype] * want.abs() * (1 + 2 * U[dtype]) + U[dtype] * slack + TINY[dtype]
    assert not bool(bad.any()) and bool(torch.isfinite(got).all()), (int(bad.sum()), float((got - want).abs().max()))


# ------------------------------------------------------------------ norm
NORM_SHAPES = [(1, 1), (3, 7), (1, 257), (5, 64), (9, 256), (33, 520), (2, 1000), (7, 2048), (4, 4097), (3, 8192), (2, 16384), (2, 20000), (1, 40008)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,width", NORM_SHAPES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm(L, dtype, rows, width, residual):
    x, res = rand((rows, width), dtype, 1, 3.0), rand((rows, width), dtype, 2, 2.0) if residual else None
    w = rand((width,), F32 if width % 2 else dtype, 3, 0.2, 1.0)
    r = L.rms_norm(x, w, res, eps=1e-5)
    y, h, rstd = ref.rms_norm(x, w, res, 1e-5)
    assert torch.equal(r.hidden.double(), h)
    # the mean of squares is off by (width + 3) 2^-23 at most, its root by half of that; then three roundings
    rel = (width / 2 + 6) * E
    near(r.rstd, rstd, rel * rstd, F32)
    near(r.out, y, (rel + 3 * E) * y.abs(), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width", [(1, 1), (5, 64), (4, 257), (7, 2048), (3, 4100), (2, 20000)])
def test_norm_in_8_bits(L, dtype, rows, width):
    x, res, w = rand((rows, width), dtype, 1, 3.0), rand((rows, width), dtype, 2), rand((width,), F32, 3, 0.2, 1.0)
    x[0] = 0.0
    res[0] = 0.0
    r = L.rms_norm(x, w, res, quantize=True)
    y, _, _ = ref.rms_norm(x, w, res, 1e-6)
    check_8_bits(r.out, r.scale, y, (width / 2 + 9) * E)


def check_8_bits(q, scale, y, rel):
    """Scales are max / 448; every element is one of the two 8-bit values around y / scale, the nearer one but for what
    fp32 leaves open next to a middle."""
    want = (y.abs().amax(-1) / 448).clamp_min(2.0 ** -126)
    near(scale, want, (rel + 2 * E) * want, F32)
    table = ref.e4m3_values().to(y.device)
    at = y / scale.double()[..., None]
    i = torch.searchsorted(table, at.abs().clamp_max(448.0).contiguous()).clamp(1, len(table) - 1)
    lo, hi = table[i - 1], table[i]
    best = torch.minimum((at.abs() - lo).abs(), (hi - at.abs()).abs())
    off = (q.double().abs() - at.abs()).abs()
    assert bool((off <= best + 2 * (rel + 4 * E) * at.abs() + 1e-30).all())
    assert bool(((q.double() == 0) | (torch.sign(q.double()) == torch.sign(at))).all())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_quantize(L, dtype):
    for rows, width in ((1, 1), (3, 16), (5, 1001), (2, 5000)):
        x = rand((rows, width), dtype, 4, 0.02)
        q = L.quantize(x)
        check_8_bits(q.values, q.scale, x.double(), 0.0)
    tiny = torch.full((2, 8), 2.0 ** -140, device="cuda")
    q = L.quantize(tiny)
    assert bool((q.scale == 2.0 ** -126).all()) and bool(torch.isfinite(q.values.float()).all())
    odd = torch.ones((3, 64), device="cuda", dtype=dtype)
    odd[0, 5], odd[1, 9] = float("nan"), float("-inf")
    q = L.quantize(odd)
    assert torch.isnan(q.scale).tolist() == [True, True, False] and bool((q.values[2].float() == 448).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,rows,width", [(2, 5, 257), (4, 3, 2048), (3, 9, 64), (2, 1, 20000)])
def test_norm_of_workers_with_strided_weights_and_rows(L, dtype, R, rows, width):
    """Weights as stretches of a batch's rows, activations as views of longer rows, results in their inputs' places."""
    batch = rand((R, width + 11), F32, 5, 0.2, 1.0)
    w = batch[:, 3:3 + width]
    x, res = wide(rand((R, rows, width), dtype, 6), 8), wide(rand((R, rows, width), dtype, 7), 24)
    y, h, rstd = ref.rms_norm(x, w, res, 1e-6)
    r = L.rms_norm(x, w, res, hidden=res, out=x)
    assert r.out is x and r.hidden is res and torch.equal(res.double(), h)
    near(x, y, ((width / 2 + 9) * E) * y.abs(), dtype)
    assert bool((res._base[..., -8:] == 7).all())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 7), (130, 64), (509, 257), (40, 520), (33, 1024), (17, 4096), (5, 4097), (3, 16384), (2, 20008)])
@pytest.mark.parametrize("stream", [False, True])
def test_norm_grad(L, dtype, rows, width, stream):
    h, g = rand((rows, width), dtype, 1, 2.0), rand((rows, width), dtype, 2, 0.1)
    gh = rand((rows, width), dtype, 3, 0.1) if stream else None
    w = rand((width,), F32, 4, 0.2, 1.0)
    rstd = ref.rms_norm(h, w, None, 1e-6)[2].float()
    r = L.rms_norm_grad(g, h, rstd, w, grad_hidden=gh)
    dh, dw, size = ref.rms_norm_grad(g, h, rstd, w, gh)
    n = h.double() * rstd.double()[:, None]
    wg = g.double() * w.double()
    # the mean's terms: (width + 4) 2^-23 of their magnitudes
    slack = rstd.double()[:, None] * (4 * E * wg.abs() + n.abs() * (width + 6) * E * (wg * n).abs().mean(-1, keepdim=True)) + 2 * E * dh.abs()
    near(r.hidden, dh, slack + (2 * E * gh.double().abs() if stream else 0), dtype)
    near(r.weight, dw, (rows + 3) * E * size, F32)


def test_norm_grad_of_workers_into_a_gradient_batch(L):
    R, rows, width = 3, 50, 257
    batch = torch.full((R, width + 20), 5.0, device="cuda")
    w = rand((R, width), F32, 1, 0.1, 1.0)
    h, g = wide(rand((R, rows, width), BF16, 2), 7, 1), rand((R, rows, width), BF16, 3)
    rstd = ref.rms_norm(h, w, None, 1e-6)[2].float()
    _, dw, size = ref.rms_norm_grad(g, h, rstd, w, None)
    out = batch[:, 5:5 + width]
    L.rms_norm_grad(g, h, rstd, w, out_weight=out)
    near(out, dw, (rows + 3) * E * size, F32)
    keep = out.clone()
    r = L.rms_norm_grad(g, h, rstd, w, out_weight=out, accumulate=True, out=g)
    near(out, 2 * dw, 2 * (rows + 4) * E * size, F32)
    assert r.hidden is g and bool((batch[:, :5] == 5).all()) and bool((batch[:, 5 + width:] == 5).all())
    empty = torch.zeros((R, 0, width), device="cuda", dtype=BF16)
    none = torch.zeros((R, 0), device="cuda")
    L.rms_norm_grad(empty, empty, none, w, out_weight=out, accumulate=True)
    assert not torch.equal(out, keep)
    L.rms_norm_grad(empty, empty, none, w, out_weight=out)
    assert bool((out == 0).all())


def test_norm_of_odd_values(L):
    x = torch.ones((4, 300), device="cuda")
    x[1, 7], x[2, 8] = float("nan"), float("inf")
    r = L.rms_norm(x, None)
    assert bool(torch.isnan(r.out[1]).all()) and bool(torch.isnan(r.out[2, 8])) and bool((r.out[2, :8] == 0).all())
    near(r.out[0], torch.full((300,), (1 + 1e-6) ** -0.5, device="cuda"), 300 * E, F32)


def test_norm_gradient_against_differences(L):
    h, w, g = rand((4, 33), F32, 1), rand((33,), F32, 2, 0.2, 1.0), rand((4, 33), F32, 3)
    r = L.rms_norm(h, w)
    got = L.rms_norm_grad(g, h, r.rstd, w)
    loss = lambda hh, ww: (ref.rms_norm(hh, ww, None, 1e-6)[0] * g.double()).sum()  # noqa: E731
    h64, w64, step = h.double(), w.double(), 1e-5
    for i in range(0, 132, 13):
        d = torch.zeros(132, device="cuda", dtype=torch.float64)
        d[i] = step
        d = d.view(4, 33)
        assert abs(float((loss(h64 + d, w64) - loss(h64 - d, w64)) / (2 * step)) - float(got.hidden.view(-1)[i])) < 1e-5
    for i in range(0, 33, 5):
        d = torch.zeros(33, device="cuda", dtype=torch.float64)
        d[i] = step
        assert abs(float((loss(h64, w64 + d) - loss(h64, w64 - d)) / (2 * step)) - float(got.weight[i])) < 1e-5


# ------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape,workers", [((1,), False), ((3, 5), False), ((61, 100), False), ((2, 7, 33), True), ((3, 4, 64), True), ((2, 1, 12), True)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(L, dtype, shape, workers, residual):
    x, res = rand(shape, dtype, 1), rand(shape, dtype, 2) if residual else None
    key = dict(round=(5 << 32) + 9, layer=40000)
    got = L.dropout(x, 0.3, 0x123456789ABCDEF, worker=6, workers=workers, residual=res, **key)
    want = ref.dropout(x, 0.3, 0x123456789ABCDEF, key["round"], key["layer"], 6, res, workers)
    near(got, want, 2 * E * (x.double().abs() * 1.5), dtype)
    if not residual:
        assert torch.equal(got == 0, want == 0)


@pytest.mark.parametrize("pad,offset,width", [(8, 0, 64), (3, 0, 64), (0, 1, 64), (5, 2, 33), (4, 4, 12), (8, 8, 20)])
def test_dropout_does_not_depend_on_the_layout(L, pad, offset, width):
    x, res = rand((2, 9, width), BF16, 1), rand((2, 9, width), BF16, 2)
    want = L.dropout(x, 0.5, 11, residual=res, workers=True)
    xs, rs = wide(x, pad, offset), wide(res, pad, offset)
    out = wide(torch.zeros_like(x), pad, offset)
    assert torch.equal(L.dropout(xs, 0.5, 11, residual=rs, workers=True, out=out), want)
    assert torch.equal(L.dropout(xs, 0.5, 11, residual=rs, workers=True, out=rs), want)
    if pad:
        assert bool((out._base[offset:offset + 18 * (width + pad)].view(18, -1)[:, width:] == 7).all())


def test_dropout_of_odd_values_and_probabilities(L):
    x = torch.full((4096,), float("nan"), device="cuda")
    y = L.dropout(x, 0.5, 3)
    kept = torch.isnan(y)
    assert bool((y[~kept] == 0).all()) and abs(float(kept.float().mean()) - 0.5) < 0.05      # 6 deviations: 6 * 0.5 / 64
    x = rand((4096,), F32, 1)
    assert torch.equal(L.dropout(x, 0.0, 3), x)
    # the gradient is the same call: the same places, the same factor
    g = torch.ones_like(x)
    assert torch.equal(L.dropout(g, 0.25, 7, layer=1) * x, L.dropout(x, 0.25, 7, layer=1))
    for other in (dict(seed=8), dict(layer=2), dict(round=1), dict(worker=1), dict(round=1 << 32)):
        a = {**dict(seed=7, layer=1), **other}
        assert not torch.equal(L.dropout(g, 0.25, a.pop("seed"), **a), L.dropout(g, 0.25, 7, layer=1))


def test_dropout_of_a_long_row(L):
    """Element numbers past 2^32 (a counter above 2^30): the last words of a long row."""
    n = (1 << 32) // 64 + 5
    x = torch.ones((1, 70, n), device="cuda", dtype=BF16)
    y = L.dropout(x, 0.5, 1)
    at = 69 * n + n - 64
    k = torch.from_numpy(_tail_words(at, 64) >= np.uint64(1 << 31)).cuda()
    assert torch.equal(y.view(-1)[at:] != 0, k)


def _tail_words(first, count):
    """words(..)[first:first + count] for seed 1, without the ones before."""
    out = []
    for q in range(first // 4, (first + count + 3) // 4):
        c, k = [q, 0, 0, 2], [1, 0]
        for _ in range(10):
            p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
            c = [p1 >> 32 ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, p0 >> 32 ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
            k = [k[0] + 0x9E3779B9 & 0xFFFFFFFF, k[1] + 0xBB67AE85 & 0xFFFFFFFF]
        out += c
    return np.array(out[first % 4:][:count], dtype=np.uint64)


# ------------------------------------------------------------------ products
def check_linear(L, x, w, bias=None, activation=None, residual=None, dtype=None, save=True, **more):
    dtype = dtype or x.dtype
    K = x.shape[-1]
    r = L.linear(x, w, bias, activation=activation, residual=residual, save=save, dtype=dtype, **more)
    z, size = ref.product(x, w.to(x.dtype))
    # (fp32: the three parts leave out 3 2^-24 of the terms, and six products are added for one)
    slack = ((K + 8) * E * 1.05 + 4 * E) * size
    if bias is not None:
        b = bias.double() if bias.dim() == 1 else bias.double().view(bias.shape[0], *([1] * (x.dim() - 2)), -1)
        z = z + b
        slack = slack + 2 * E * (size + b.abs())
    if save:
        near(r.pre, z, slack, dtype)
    y = ref.activate(z, activation)
    # slopes are below 1.13; the functions themselves: a few roundings of their terms
    slack = 1.13 * slack + (8 * E * (z.abs() + 1) if activation in ("silu", "gelu") else 0)
    if residual is not None:
        y = y + residual.double()
        slack = slack + 2 * E * y.abs()
    near(r.out, y, slack, dtype)
    return r


SIZES = [(1, 1, 1), (3, 5, 7), (1, 64, 64), (128, 128, 64), (130, 257, 65), (64, 1000, 257), (256, 256, 128), (300, 520, 1000), (509, 1000, 257),
         (1, 4096, 1024), (17, 2048, 4096), (1025, 257, 129), (700, 72, 3000)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear(L, dtype, M, N, K):
    check_linear(L, rand((M, K), dtype, 1), rand((N, K), dtype, 2, K ** -0.5))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("R,M,N,K", [(1, 4000, 2100, 200), (1, 8192, 4096, 136), (2, 1500, 3001, 257), (5, 900, 1100, 64)])
def test_linear_of_many_tiles(L, dtype, R, M, N, K):
    """More tiles than blocks, in both directions: every accumulator and every slot of the ring is used again."""
    x, w, g = rand((R, M, K), dtype, 1), rand((R, N, K), dtype, 2, K ** -0.5), rand((R, M, N), dtype, 3, 0.1)
    check_linear(L, x, w, rand((R, N), F32, 3), "relu", rand((R, M, N), dtype, 4))
    r = L.linear_grad(g, x, w, dtype=dtype)
    dx, size = ref.product(g, w.transpose(1, 2))
    near(r.x, dx, ((N + 8) * E * 1.05 + 4 * E) * size, dtype)
    dw, size = ref.product(g.transpose(1, 2), x.transpose(1, 2))
    near(r.weight, dw, ((M + 8) * E * 1.05 + 4 * E) * size, dtype)
    v, u = L.quantize(x[0].float()), L.quantize(w[0].float())
    z, size = ref.product(v.values.float(), u.values.float())
    s = v.scale.double()[:, None] * u.scale.double()
    near(L.linear(v.values, u.values, x_scale=v.scale, weight_scale=u.scale, dtype=dtype).out, z * s, ((K + 8) * E + 4 * E) * size * s, dtype)


@pytest.mark.parametrize("activation", [None, "relu", "silu", "gelu"])
@pytest.mark.parametrize("M,N,K", [(5, 24, 33), (200, 264, 192), (190, 261, 130)])
@pytest.mark.parametrize("dtype,w_dtype,out", [(BF16, F32, BF16), (F16, F16, F32), (F32, F32, F32)])
def test_linear_epilogue(L, activation, M, N, K, dtype, w_dtype, out):
    check_linear(L, rand((M, K), dtype, 1), rand((N, K), w_dtype, 2, K ** -0.5), rand((N,), w_dtype, 3), activation, rand((M, N), out, 4), out)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R,M,N,K,shift", [(2, 100, 300, 200, 0), (3, 33, 65, 129, 1), (8, 4, 520, 256, 4), (2, 300, 256, 512, 2)])
def test_linear_of_workers_from_a_batch(L, dtype, R, M, N, K, shift):
    """Weights and biases as stretches of a batch's fp32 rows, at places of any alignment."""
    batch = rand((R, shift + N * K + N + 5), F32, 1, K ** -0.5)
    w = batch[:, shift:shift + N * K].view(R, N, K)
    bias = batch[:, shift + N * K:shift + N * K + N]
    check_linear(L, rand((R, M, K), dtype, 2), w, bias, "silu")


@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (16, 8)])
def test_linear_of_strided_rows(L, pad, offset):
    M, N, K = 150, 200, 168
    x, w, res = wide(rand((M, K), BF16, 1), pad, offset), wide(rand((N, K), BF16, 2, K ** -0.5), pad, offset), wide(rand((M, N), BF16, 3), pad, offset)
    out, pre = wide(torch.zeros((M, N), device="cuda", dtype=BF16), pad, offset), wide(torch.zeros((M, N), device="cuda", dtype=BF16), pad, offset)
    check_linear(L, x, w, None, "relu", res, out=out, pre=pre)
    if pad:
        for t in (out, pre):
            assert bool((t._base[offset:offset + M * (N + pad)].view(M, -1)[:, N:] == 7).all())
    want = L.linear(x, w, activation="relu", residual=res).out
    L.linear(x, w, activation="relu", residual=res, out=res)
    assert torch.equal(res, want)


@pytest.mark.parametrize("M,N,K", [(1, 64, 64), (3, 5, 7), (130, 264, 192), (300, 520, 1000), (8, 2048, 4096), (257, 130, 129)])
@pytest.mark.parametrize("out", [BF16, F32])
def test_linear_in_8_bits(L, M, N, K, out):
    x, w = L.quantize(rand((M, K), F32, 1)), L.quantize(rand((N, K), F32, 2, K ** -0.5))
    bias, res = rand((N,), F32, 3), rand((M, N), out, 4)
    r = L.linear(x.values, w.values, bias, activation="gelu", residual=res, x_scale=x.scale, weight_scale=w.scale, dtype=out, save=True)
    z, size = ref.product(x.values.float(), w.values.float())
    s = x.scale.double()[:, None] * w.scale.double()
    z, slack = z * s + bias.double(), ((K + 8) * E + 4 * E) * size * s
    slack = slack + 2 * E * (z.abs() + bias.double().abs())
    near(r.pre, z, slack, out)
    near(r.out, ref.activate(z, "gelu") + res.double(), 1.13 * slack + 8 * E * (z.abs() + 1) + 2 * E * res.double().abs(), out)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (5, 3, 7), (128, 64, 64), (200, 264, 192), (509, 1000, 257), (64, 2048, 1024), (1030, 257, 129), (4097, 64, 72)])
def test_linear_grad(L, dtype, M, N, K):
    x, w, g = rand((M, K), dtype, 1), rand((N, K), F32, 2, K ** -0.5), rand((M, N), dtype, 3, 0.1)
    r = L.linear_grad(g, x, w, bias=True)
    dx, size = ref.product(g, w.to(dtype).t())
    near(r.x, dx, ((N + 8) * E * 1.05 + 4 * E) * size, dtype)
    dw, size = ref.product(g.t(), x.t())
    near(r.weight, dw, ((M + 8) * E * 1.05 + 4 * E) * size, F32)
    near(r.bias, g.double().sum(0), M * E * g.double().abs().sum(0), F32)
    half = L.linear_grad(g, x, w, need_x=False, dtype=dtype)
    assert half.x is None and half.bias is None
    near(half.weight, dw, ((M + 8) * E * 1.05 + 4 * E) * size, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("activation", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("R,M,N", [(1, 1, 1), (2, 100, 261), (3, 33, 264), (1, 2000, 64)])
def test_activation_grad(L, dtype, activation, R, M, N):
    g, z = rand((R, M, N), dtype, 1), rand((R, M, N), dtype, 2, 2.0)
    z[0, 0, 0] = 0.0
    dz, db = L.activation_grad(g, z, activation, bias=True, workers=True)
    want = g.double() * ref.slope(z.double(), activation)
    slack = 8 * E * g.double().abs() * (1 + z.double().abs()) if activation != "relu" else 0 * want
    near(dz, want, slack, dtype)
    near(db, want.sum(1), (slack + M * E * want.abs()).sum(1), F32)


def test_linear_grad_of_workers_into_a_gradient_batch(L):
    R, M, N, K, shift = 3, 70, 130, 65, 3
    flat, grad = rand((R, shift + N * K + N), F32, 1, 0.1), torch.full((R, shift + N * K + N), 5.0, device="cuda")
    cut = lambda t: (t[:, shift:shift + N * K].view(R, N, K), t[:, shift + N * K:])  # noqa: E731
    w, _ = cut(flat)
    dw, db = cut(grad)
    x, g, z = rand((R, M, K), BF16, 2), rand((R, M, N), BF16, 3), rand((R, M, N), BF16, 4)
    r = L.linear_grad(g, x, w, z, "relu", bias=True, out_weight=dw, out_bias=db)
    dz = g.double() * (z > 0)
    assert torch.equal(r.pre.double(), dz)
    want, size = ref.product(dz.transpose(1, 2), x.transpose(1, 2))
    near(dw, want, (M + 8) * E * 1.05 * size, F32)
    near(db, dz.sum(1), M * E * dz.abs().sum(1), F32)
    assert bool((grad[:, :shift] == 5).all())
    L.linear_grad(g, x, w, z, "relu", bias=True, out_weight=dw, out_bias=db, accumulate=True)
    near(dw, 2 * want, 2 * (M + 10) * E * 1.05 * size, F32)
    near(db, 2 * dz.sum(1), 2 * (M + 2) * E * dz.abs().sum(1), F32)
    before = grad.clone()
    L.linear_grad(g[:, :0], x[:, :0], w, z[:, :0], "relu", bias=True, out_weight=dw, out_bias=db, accumulate=True)
    assert torch.equal(grad, before)
    r = L.linear_grad(g[:, :0], x[:, :0], w, z[:, :0], "relu", bias=True, out_weight=dw, out_bias=db)
    assert bool((dw == 0).all()) and bool((db == 0).all()) and r.x.shape == (R, 0, K) and bool((grad[:, :shift] == 5).all())


@pytest.mark.parametrize("activation", [None, "silu", "gelu"])
def test_linear_gradients_against_differences(L, activation):
    M, N, K, step = 6, 9, 40, 1e-5
    x, w, b, g = rand((M, K), F32, 1), rand((N, K), F32, 2, K ** -0.5), rand((N,), F32, 3), rand((M, N), F32, 4)
    y = L.linear(x, w, b, activation=activation, save=True)
    got = L.linear_grad(g, x, w, y.pre, activation, bias=True)
    loss = lambda x_, w_, b_: float((ref.activate(x_ @ w_.t() + b_, activation) * g.double()).sum())  # noqa: E731
    at = [t.double() for t in (x, w, b)]
    for which, grad in ((0, got.x), (1, got.weight), (2, got.bias)):
        for i in range(0, grad.numel(), 7):
            d = torch.zeros(grad.numel(), device="cuda", dtype=torch.float64)
            d[i] = step
            up, down = list(at), list(at)
            up[which], down[which] = at[which] + d.view(at[which].shape), at[which] - d.view(at[which].shape)
            # (third derivatives below 10, step^2 / 6 of them; fp32 sums of up to 40 terms of size 1)
            assert abs((loss(*up) - loss(*down)) / (2 * step) - float(grad.view(-1)[i])) < 2e-5


def test_linear_of_no_rows(L):
    assert L.linear(torch.zeros((0, 64), device="cuda"), torch.zeros((8, 64), device="cuda")).out.shape == (0, 8)


def test_linear_of_odd_values(L):
    """NaN and infinities stay in the rows and columns that they enter."""
    for dtype in (BF16, F32):
        x, w = rand((150, 256), dtype, 1), rand((140, 256), dtype, 2)
        want = L.linear(x, w).out
        x[3, 5], x[70, 9] = float("nan"), float("inf")
        got = L.linear(x, w).out
        assert bool(torch.isnan(got[3]).all()) and not bool(torch.isfinite(got[70]).any())
        keep = [i for i in range(150) if i not in (3, 70)]
        assert torch.equal(got[keep], want[keep])


def test_linear_twice_gives_the_same_bits(L):
    for M, N, K in ((64, 512, 4096), (509, 1000, 257), (2000, 300, 1000)):
        x, w = rand((M, K), BF16, 1), rand((N, K), F32, 2)
        assert torch.equal(L.linear(x, w).out, L.linear(x, w).out)
        g = rand((M, N), BF16, 3)
        a, b = L.linear_grad(g, x, w, bias=True), L.linear_grad(g, x, w, bias=True)
        assert torch.equal(a.x, b.x) and torch.equal(a.weight, b.weight) and torch.equal(a.bias, b.bias)
