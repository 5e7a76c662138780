"""Language-model operators against plain 64-bit implementations: sizes, types, strides and masks at which they can go
wrong.  Tolerances follow from the arithmetic: EPS is half a unit in the last place of fp32; a sum of n terms is off by at most
n EPS of the terms' magnitudes, an exponential by 2^-21 (two units of the hardware's, and the rounding of its
argument), a result by half a unit of its own type."""
import math

import pytest
import torch

from tests import lm_reference as ref

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}
NEG, NAN = float("-inf"), float("nan")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def lm():
    from paper_1906_02367_b200 import lm as module
    return module


def gen(seed):
    return torch.Generator().manual_seed(seed)


def near(got, want, tol):
    """Within tol (a number or a tensor) element by element; infinities and NaN at the same places."""
    got, want = got.double().cpu(), want.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fin = torch.isfinite(want)
    assert torch.equal(fin, torch.isfinite(got)) and torch.equal(got[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)])
    tol = torch.as_tensor(tol, dtype=torch.float64).expand(want.shape)
    worst = ((got - want).abs() - tol)[fin]
    assert not worst.numel() or float(worst.max()) <= 0.0, f"over the tolerance by {float(worst.max()):.3g}"


def view(t, pad, offset):
    """The same rows inside a larger buffer: `pad` more columns per row, the first element `offset` elements in."""
    n, v = t.shape
    buf = torch.full((offset + n * (v + pad) + 8,), 77.0, dtype=t.dtype, device="cuda")
    out = torch.as_strided(buf, (n, v), (v + pad, 1), offset)
    out.copy_(t)
    return out, buf


def sum_tol(V):
    """Relative error of a sum of V exponentials, generously split into at most V / 128 terms in a row and a tree."""
    return (V / 128 + 40) * EPS + 2.0 ** -21


# ------------------------------------------------------------------ embedding
@pytest.mark.parametrize("table_type,out_type", [(F32, F32), (F32, BF16), (BF16, BF16), (F16, F32), (BF16, F16), (F32, F16)])
@pytest.mark.parametrize("R,N,V,D,ids", [(1, 1, 1, 1, torch.int64), (1, 7, 5, 3, torch.int32), (3, 65, 33, 64, torch.int64), (1, 300, 1000, 257, torch.int32),
                                         (2, 9, 50, 2056, torch.int64), (8, 16, 11, 40, torch.int64)])
def test_embed_rows(R, N, V, D, ids, table_type, out_type):
    g = gen(R * 1000 + N)
    table = torch.randn((R, V, D), generator=g).to(table_type)
    tok = torch.randint(-1, V, (R, N), generator=g).to(ids)
    want = torch.where(tok[..., None] < 0, torch.zeros(()), torch.stack([table[r].float()[tok[r].long().clamp_min(0)] for r in range(R)]) * 1.7).to(out_type)
    got = lm().embed(tok.cuda(), table.cuda(), scale=1.7, dtype=out_type)
    assert torch.equal(got.cpu(), want)          # one product, one rounding
    if R == 1:
        got = lm().embed(tok[0].cuda(), table[0].cuda(), scale=1.7, dtype=out_type)
        assert torch.equal(got.cpu(), want[0])
    shared = lm().embed(tok.cuda(), table[0].cuda(), scale=1.7, dtype=out_type)
    assert torch.equal(shared[0].cpu(), want[0])


@pytest.mark.parametrize("offset", [0, 1, 2, 3, 4])
@pytest.mark.parametrize("pad", [0, 1, 4])
def test_embed_from_a_stretch_of_the_workers_rows(offset, pad):
    """Tables at any offset of an R x d fp32 batch, rows of any stride; results into rows of any stride."""
    R, N, V, D = 3, 37, 29, 24
    g = gen(offset * 10 + pad)
    d = offset + V * (D + pad) + 5
    batch = torch.randn((R, d), generator=g).cuda()
    table = torch.as_strided(batch, (R, V, D), (d, D + pad, 1), offset)
    tok = torch.randint(0, V, (R, N), generator=g)
    want = torch.stack([table.cpu()[r][tok[r]] for r in range(R)]) * 0.5
    assert torch.equal(lm().embed(tok.cuda(), table, scale=0.5).cpu(), want)
    out, buf = view(torch.zeros(R * N, D), pad, offset)
    lm().embed(tok.cuda(), table, scale=0.5, out=torch.as_strided(buf, (R, N, D), (N * (D + pad), D + pad, 1), offset))
    assert torch.equal(out.cpu(), want.view(R * N, D))
    rest = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(rest, (R * N, D), (D + pad, 1), offset).fill_(False)
    assert bool((buf[rest] == 77.0).all())       # nothing beside the rows was written


def test_ids_past_the_end_are_reported_and_harmless():
    m = lm()
    from paper_1906_02367_b200 import binding as B
    V, D = 6, 8
    table = torch.ones(V, D).cuda()
    tok = torch.tensor([0, V, 5, 2**40], dtype=torch.int64).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = m.embed(tok, table, status=status).cpu()
    assert int(status) == B.QS_INVALID_ARG and bool(torch.isnan(out[[1, 3]]).all()) and bool((out[[0, 2]] == 1).all())
    status.zero_()
    grad = m.embed_grad(tok, torch.ones(4, D).cuda(), V, status=status).cpu()
    assert int(status) == B.QS_INVALID_ARG and float(grad.sum()) == 2 * D and float(grad[0].sum()) == D and float(grad[5].sum()) == D
    z = torch.zeros(4, V).cuda()
    status.zero_()
    r = m.token_logp(z, tok, status=status)
    assert int(status) == B.QS_INVALID_ARG and torch.isnan(r.logp.cpu()).tolist() == [False, True, False, True]
    status.zero_()
    g = m.token_logp_grad(z, tok, r.lse, status=status).cpu()
    assert int(status) == B.QS_INVALID_ARG and torch.isnan(g).any(1).tolist() == [False, True, False, True]
    ids = torch.tensor([[0, 1], [1, V], [-1, 3], [2**40, 0]]).cuda()
    status.zero_()
    r = m.distill(z, ids, torch.zeros(4, 2).cuda(), weight=1.0, status=status)
    assert int(status) == B.QS_INVALID_ARG and torch.isnan(r.loss.cpu()).tolist() == [False, True, False, True]
    assert torch.isnan(r.grad.cpu()).all(1).tolist() == [False, True, False, True] and torch.isnan(r.grad.cpu()).any(1).tolist() == [False, True, False, True]
    status.zero_()
    g = m.distill_grad(z, ids, torch.zeros(4, 2).cuda(), r.lse, 1.0, status=status).cpu()
    assert int(status) == B.QS_INVALID_ARG and torch.isnan(g).all(1).tolist() == [False, True, False, True]
    m.embed(tok.clamp_max(5), table, status=status.zero_())
    assert int(status) == 0


def _tokens(kind, N, V, g):
    if kind == "uniform":
        return torch.randint(-1, V, (N,), generator=g)
    if kind == "one":
        return torch.full((N,), V - 1)
    if kind == "padding":
        return torch.full((N,), -1)
    if kind == "rising":
        return torch.arange(N) % V
    if kind == "falling":
        return V - 1 - torch.arange(N) % V
    return torch.clamp((torch.rand(N, generator=g) * math.log(V + 1)).exp().long() - 1, 0, V - 1)    # zipf


GRAD_CASES = [(1, 0, 5, 8, "uniform"), (1, 1, 1, 1, "one"), (1, 1, 70000, 8, "one"), (1, 33, 7, 5, "uniform"), (2, 100, 1000, 64, "zipf"),
              (1, 1023, 511, 33, "zipf"), (1, 1024, 512, 16, "falling"), (1, 1025, 513, 16, "rising"), (3, 2500, 262145, 8, "uniform"),
              (1, 5000, 40, 257, "zipf"), (1, 4096, 9, 64, "one"), (2, 300, 77, 1030, "padding"), (1, 9000, 300000, 12, "zipf"),
              (8, 40, 3000, 100, "zipf"), (1, 3000, 2, 2050, "uniform"), (1, 20000, 3, 4, "one")]


@pytest.mark.parametrize("R,N,V,D,kind", GRAD_CASES)
@pytest.mark.parametrize("type_,ids", [(F32, torch.int64), (BF16, torch.int32), (F16, torch.int64)])
def test_embed_gradient(R, N, V, D, kind, type_, ids):
    g = gen(N + V)
    tok = torch.stack([_tokens(kind, N, V, g) for _ in range(R)]).to(ids)
    go = torch.randn((R, N, D), generator=g).to(type_)
    got = lm().embed_grad(tok.cuda(), go.cuda(), V, scale=0.75)
    again = lm().embed_grad(tok.cuda(), go.cuda(), V, scale=0.75)
    assert torch.equal(got, again)               # no order of blocks in the sums
    base = torch.randn((R, V, D), generator=g)
    acc = lm().embed_grad(tok.cuda(), go.cuda(), V, scale=0.75, accumulate=True, out=base.cuda())
    for r in range(R):
        want, mag, cnt = ref.embed_grad(tok[r], go[r], V, 0.75)
        tol = (cnt[:, None] + 2) * EPS * mag
        near(got[r], want, tol)
        near(acc[r], want + base[r].double(), tol + 2 * EPS * (mag + base[r].abs()))
        assert torch.equal(acc[r].cpu()[cnt == 0], base[r][cnt == 0])


@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 1), (4, 4), (2, 3)])
def test_embed_gradient_into_the_workers_gradient_batch(offset, pad):
    R, N, V, D = 3, 200, 50, 20
    g = gen(offset + pad)
    d = offset + V * (D + pad) + 3
    batch = torch.full((R, d), 5.0, device="cuda")
    out = torch.as_strided(batch, (R, V, D), (d, D + pad, 1), offset)
    tok = torch.randint(0, 30, (R, N), generator=g)
    wide = torch.randn((R * N, D + pad), generator=g).cuda()
    go = torch.as_strided(wide, (R, N, D), (N * (D + pad), D + pad, 1))
    lm().embed_grad(tok.cuda(), go, V, out=out)
    for r in range(R):
        want, mag, cnt = ref.embed_grad(tok[r], go[r].cpu(), V, 1.0)
        near(out[r], want, (cnt[:, None] + 2) * EPS * mag)
    rest = torch.ones_like(batch, dtype=torch.bool)
    torch.as_strided(rest, (R, V, D), (d, D + pad, 1), offset).fill_(False)
    assert bool((batch[rest] == 5.0).all())


@pytest.mark.parametrize("offset", [0, 1, 2, 3])
@pytest.mark.parametrize("V,D", [(1, 4), (1, 5), (2, 7), (3000, 4), (700, 37), (20, 1030), (9, 4100)])
@pytest.mark.parametrize("few", [True, False])
def test_embed_gradient_beside_other_values(offset, V, D, few):
    """Rows side by side at any distance from a 16-byte boundary: named rows between rows of zeros, nothing beside the table."""
    R, N = 3, 6 if few else 1500
    g = gen(V + D + offset)
    d = offset + V * D + 5
    batch = torch.full((R, d), 5.0, device="cuda")
    out = torch.as_strided(batch, (R, V, D), (d, D, 1), offset)
    tok = torch.randint(0, V, (R, N), generator=g) // 3 * 3
    go = torch.randn((R, N, D), generator=g).to(BF16)
    for type_ in (F32, BF16):
        out.fill_(7.0)
        lm().embed_grad(tok.cuda(), go.to(type_).cuda(), V, out=out)
        acc = torch.full((R, d), 0.5, device="cuda")
        lm().embed_grad(tok.cuda(), go.to(type_).cuda(), V, out=torch.as_strided(acc, (R, V, D), (d, D, 1), offset), accumulate=True)
        for r in range(R):
            want, mag, cnt = ref.embed_grad(tok[r], go[r], V, 1.0)
            tol = (cnt[:, None] + 2) * EPS * mag
            near(out[r], want, tol)
            near(torch.as_strided(acc, (R, V, D), (d, D, 1), offset)[r], want + 0.5, tol + 2 * EPS * (mag + 0.5))
        rest = torch.ones_like(batch, dtype=torch.bool)
        torch.as_strided(rest, (R, V, D), (d, D, 1), offset).fill_(False)
        assert bool((batch[rest] == 5.0).all()) and bool((acc[rest] == 0.5).all())


def test_embed_gradient_is_the_transpose_of_embed():
    """<embed(tok, W), G> = <W, embed_grad(tok, G)>, and the difference of the product along one entry."""
    N, V, D = 50, 20, 12
    g = gen(3)
    tok, G, W = torch.randint(-1, V, (N,), generator=g).cuda(), torch.randn((N, D), generator=g).cuda(), torch.randn((V, D), generator=g).cuda()
    left = (lm().embed(tok, W, scale=2.0).double() * G.double()).sum()
    right = (W.double() * lm().embed_grad(tok, G, V, scale=2.0).double()).sum()
    assert abs(float(left - right)) <= 2e-6 * N * D


# ------------------------------------------------------------------ log probabilities
ROWS = [(1, 1), (1, 2), (3, 7), (2, 31), (5, 33), (4, 255), (3, 256), (65, 1000), (7, 1023), (3, 4099), (2, 16384), (3, 50003), (1, 131072), (2, 150001)]


def _logits(kind, N, V, type_, g):
    z = torch.randn((N, V), generator=g) * 3.0
    if kind == "masked":
        z[torch.rand((N, V), generator=g) < 0.5] = NEG
        z[0] = NEG
        if N > 1:
            z[1] = NEG
            z[1, V // 2] = -3.0
        if N > 2:
            z[2, : V - V // 8] = NEG
    elif kind == "lowest":
        z[torch.rand((N, V), generator=g) < 0.9] = torch.finfo(type_).min
        z[0] = torch.finfo(type_).min
    elif kind == "equal":
        z[:] = torch.arange(N)[:, None].float() - 1.0
    elif kind == "few":                          # a handful of values: ties everywhere
        z = torch.round(z)
    elif kind == "rising":
        z = torch.linspace(-8, 8, V).expand(N, V).clone()
    elif kind == "falling":
        z = torch.linspace(8, -8, V).expand(N, V).clone()
    elif kind == "zeros":
        z = torch.where(torch.rand((N, V), generator=g) < 0.5, 0.0, -0.0)
    elif kind == "blocks":                       # the largest lie side by side
        z[:, V // 3: V // 3 + 200] += 30.0
    return z.to(type_)


def _check_logp(z_dev, z, tok, scale, top):
    r = lm().token_logp(z_dev, tok.cuda(), scale=scale, top=top)
    logp, lse, ent, ids, tl = ref.token_logp(z, tok, scale, top)
    V = z.shape[1]
    s = sum_tol(V)
    size = torch.where(torch.isfinite(lse), lse.abs(), torch.zeros(()).double())
    near(r.lse, lse, s + 4 * EPS * size)
    near(r.logp, logp, s + 8 * EPS * torch.where(torch.isfinite(logp), logp.abs(), torch.zeros(()).double()))
    near(r.entropy, ent, s * (4 + 2 * math.log(V + 1)))
    if top:
        assert torch.equal(r.top_ids.cpu().long(), ids) and r.top_ids.dtype == tok.dtype
        near(r.top_logp, tl, s + 8 * EPS * torch.where(torch.isfinite(tl), tl.abs(), torch.zeros(()).double()))
    return r


@pytest.mark.parametrize("type_,ids", [(F32, torch.int64), (BF16, torch.int32), (F16, torch.int64)])
@pytest.mark.parametrize("N,V", ROWS)
def test_token_logp(N, V, type_, ids):
    g = gen(N * 7 + V)
    z = _logits("plain", N, V, type_, g)
    tok = torch.randint(-1, V, (N,), generator=g).to(ids)
    _check_logp(z.cuda(), z, tok, 0.8, min(V, 11))


@pytest.mark.parametrize("top", [0, 1, 2, 31, 33, 64, 100, 128])
@pytest.mark.parametrize("N,V,type_", [(3, 1000, BF16), (2, 20011, F32), (2, 70001, BF16)])
def test_numbers_of_alternatives(N, V, type_, top):
    g = gen(top)
    z = _logits("plain", N, V, type_, g)
    _check_logp(z.cuda(), z, torch.randint(0, V, (N,), generator=g), 1.0, top)


@pytest.mark.parametrize("kind", ["masked", "lowest", "equal", "few", "rising", "falling", "zeros", "blocks"])
@pytest.mark.parametrize("N,V,type_,top", [(4, 40, F32, 17), (3, 1000, BF16, 64), (3, 5003, F16, 128), (4, 33000, BF16, 20), (2, 140001, F32, 64)])
def test_masks_and_ties(kind, N, V, type_, top):
    g = gen(V)
    z = _logits(kind, N, V, type_, g)
    tok = torch.randint(0, V, (N,), generator=g)
    tok[0] = int(ref.order(z[-1])[0])
    _check_logp(z.cuda(), z, tok, 1.0, min(top, V))


@pytest.mark.parametrize("V", [5, 1000, 40009])
@pytest.mark.parametrize("type_", [F32, BF16, F16])
def test_nan_and_infinity(V, type_):
    z = _logits("plain", 6, V, type_, gen(V))
    z[1, V // 2] = NAN
    z[2, V - 1] = float("inf")
    z[3] = NAN
    z[4] = NEG
    z[4, 0] = NAN
    tok = torch.full((6,), V // 3)
    r = _check_logp(z.cuda(), z, tok, 1.0, 4)
    assert torch.isnan(r.lse.cpu()).tolist() == [False, True, True, True, True, False]


@pytest.mark.parametrize("offset", [0, 1, 3, 8])
@pytest.mark.parametrize("pad", [0, 1, 5, 8])
@pytest.mark.parametrize("type_", [F32, BF16])
def test_rows_of_any_stride(offset, pad, type_):
    N, V = 5, 2051
    g = gen(offset + 10 * pad)
    z = _logits("plain", N, V, type_, g)
    zd, _ = view(z, pad, offset)
    tok = torch.randint(0, V, (N,), generator=g)
    r = _check_logp(zd, z, tok, 1.0, 9)
    gr = torch.randn(N, generator=g)
    out, buf = view(torch.zeros(N, V, dtype=type_), 3 - min(pad, 3), offset // 2)
    lm().token_logp_grad(zd, tok.cuda(), r.lse, gr.cuda(), entropy=r.entropy, grad_entropy=gr.cuda(), out=out)
    _near_logp_grad(out, z, tok, 1.0, gr, gr)
    rest = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(rest, out.shape, out.stride(), out.storage_offset()).fill_(False)
    assert bool((buf[rest] == 77.0).all())
    ids, u = torch.randint(0, V, (N, 4), generator=g), torch.randn((N, 4), generator=g)
    out, buf = view(torch.zeros(N, V, dtype=type_), pad, (offset * 5) % 7)
    got = lm().distill(zd, ids.cuda(), u.cuda(), weight=gr.cuda(), out=out)
    _near_distill(got, z, ids, u, 1.0, 1.0, False, gr)
    rest = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(rest, out.shape, out.stride(), out.storage_offset()).fill_(False)
    assert bool((buf[rest] == 77.0).all())


def test_one_token_of_many_rows_beyond_32_bits():
    """Rows whose offsets pass 2^32 bytes and 2^31 elements."""
    V = 65536
    N = (1 << 31) // V + 3
    z = torch.zeros((N, V), dtype=BF16, device="cuda")
    z[-1, 5] = 9.0
    z[-2, V - 1] = 4.0
    tok = torch.zeros(N, dtype=torch.int64, device="cuda")
    tok[-1] = 5
    r = lm().token_logp(z, tok, top=1)
    assert r.top_ids[-2:, 0].tolist() == [V - 1, 5] and int(r.top_ids[:-2].max()) == 0
    want = 9.0 - math.log(V - 1 + math.exp(9.0))
    assert abs(float(r.logp[-1]) - want) < 1e-5 and abs(float(r.logp[0]) + math.log(V)) < 1e-5
    lm().token_logp_grad(z, tok, r.lse, 1.0, out=z)
    p = math.exp(want)
    assert abs(float(z[-1, 5]) - (1 - p)) < 4e-3 and abs(float(z[0, 0]) - 1.0) < 4e-3 and abs(float(z[0, 1]) * V + 1.0) < 4e-3


# ------------------------------------------------------------------ their gradient
def _near_logp_grad(got, z, tok, scale, g, h):
    want = ref.token_logp_grad(z, tok, scale, g, h)
    lp, lse = ref.log_softmax(z, scale)
    p = lp.exp()
    l0 = torch.where(p > 0, lp.abs(), torch.zeros_like(lp))
    ent = (p * l0).sum(1, keepdim=True)
    size = torch.where(torch.isfinite(lse), lse.abs(), torch.zeros(()).double())[:, None]
    rel = sum_tol(z.shape[1]) + 8 * EPS * (l0 + size + 1)
    terms = scale * p * (g.double().abs()[:, None] + h.double().abs()[:, None] * (l0 + ent + 1))
    hot = torch.zeros_like(p)
    for i, t in enumerate(tok.tolist()):
        if t >= 0:
            hot[i, t] = abs(float(g[i])) * scale
    near(got, want, rel * terms * 4 + 4 * EPS * hot + HALF[z.dtype] * want.abs() + TINY[z.dtype] + 1e-30)


@pytest.mark.parametrize("type_,ids", [(F32, torch.int64), (BF16, torch.int32), (F16, torch.int64)])
@pytest.mark.parametrize("N,V", ROWS[:-2] + [(2, 140001)])
def test_token_logp_gradient(N, V, type_, ids):
    g = gen(N + V)
    z = _logits("plain", N, V, type_, g)
    tok = torch.randint(-1, V, (N,), generator=g).to(ids)
    gl, ge = torch.randn(N, generator=g), torch.randn(N, generator=g)
    zd = z.cuda()
    r = lm().token_logp(zd, tok.cuda(), scale=1.3)
    got = lm().token_logp_grad(zd, tok.cuda(), r.lse, gl.cuda(), scale=1.3, entropy=r.entropy, grad_entropy=ge.cuda())
    _near_logp_grad(got, z, tok, 1.3, gl, ge)
    got = lm().token_logp_grad(zd, tok.cuda(), r.lse, -0.5, scale=1.3)
    _near_logp_grad(got, z, tok, 1.3, torch.full((N,), -0.5), torch.zeros(N))
    got = lm().token_logp_grad(zd, None, r.lse, 1.0, scale=1.3, entropy=r.entropy, grad_entropy=ge.cuda())
    _near_logp_grad(got, z, torch.full((N,), -1), 1.3, gl, ge)
    same = lm().token_logp_grad(zd, tok.cuda(), r.lse, gl.cuda(), scale=1.3, out=zd)          # in the logits' place
    assert same.data_ptr() == zd.data_ptr()
    _near_logp_grad(same, z, tok, 1.3, gl, torch.zeros(N))


@pytest.mark.parametrize("type_,V", [(F32, 131073), (F32, 262200), (BF16, 262145), (F16, 300007)])
def test_rows_beyond_the_registers_of_a_cluster(type_, V):
    N, K = 2, 40
    g = gen(V)
    z = _logits("plain", N, V, type_, g)
    z[1, V - 3000:] = z[1, 0] + 20.0             # ties that defeat the bound, in the last block
    tok = torch.tensor([V - 1, 0])
    zd = z.cuda()
    _check_logp(zd, z, tok, 1.0, K)
    ids, w = torch.randperm(V, generator=g)[: 2 * K].view(N, K).contiguous(), torch.rand(N, generator=g)
    for tail in (False, True):
        u = torch.log_softmax(torch.randn((N, K), generator=g), 1) - 0.3
        got = lm().distill(zd, ids.cuda(), u.cuda(), tail=tail, weight=w.cuda())
        _near_distill(got, z, ids, u, 1.0, 1.0, tail, w)
        place = zd.clone()
        assert torch.equal(lm().distill(place, ids.cuda(), u.cuda(), tail=tail, weight=w.cuda(), out=place).grad, got.grad)


@pytest.mark.parametrize("kind", ["masked", "equal", "few"])
@pytest.mark.parametrize("type_", [F32, BF16])
def test_token_logp_gradient_under_masks(kind, type_):
    N, V = 4, 3001
    g = gen(5)
    z = _logits(kind, N, V, type_, g)
    tok = torch.randint(0, V, (N,), generator=g)
    gl, ge = torch.randn(N, generator=g), torch.randn(N, generator=g)
    r = lm().token_logp(z.cuda(), tok.cuda())
    got = lm().token_logp_grad(z.cuda(), tok.cuda(), r.lse, gl.cuda(), entropy=r.entropy, grad_entropy=ge.cuda())
    _near_logp_grad(got, z, tok, 1.0, gl, ge)


def test_token_logp_gradient_against_differences():
    N, V, step = 3, 23, 1e-5
    g = gen(9)
    z = torch.randn((N, V), generator=g) * 2
    tok = torch.tensor([3, -1, 22])
    gl, ge = torch.randn(N, generator=g), torch.randn(N, generator=g)
    r = lm().token_logp(z.cuda(), tok.cuda(), scale=0.7)
    got = lm().token_logp_grad(z.cuda(), tok.cuda(), r.lse, gl.cuda(), scale=0.7, entropy=r.entropy, grad_entropy=ge.cuda()).cpu().double()

    def f(zz):
        logp, _, ent, _, _ = ref.token_logp(zz, tok, 0.7, 0)
        return gl.double() * logp + ge.double() * ent

    for v in range(V):
        e = torch.zeros((N, V), dtype=torch.float64)
        e[:, v] = step
        diff = (f(z.double() + e) - f(z.double() - e)) / (2 * step)
        assert float((diff - got[:, v]).abs().max()) < 1e-5        # 2^-21 of terms below 8, and the differences' own 1e-9


# ------------------------------------------------------------------ distillation
def _near_distill(got, z, ids, u, scale, ts, tail, weight):
    loss, lse, log_tail = ref.distill(z, ids, u, scale, ts, tail)
    V = z.shape[1]
    s = sum_tol(V)
    fin = lambda t: torch.where(torch.isfinite(t), t.abs(), torch.zeros(()).double())  # noqa: E731
    near(got.lse, lse, s + 4 * EPS * fin(lse))
    lp, _ = ref.log_softmax(z, scale)
    big = torch.stack([fin(lp[i][ids[i].clamp_min(0).long()]).max() for i in range(z.shape[0])])
    a = fin(u.double() * ts).amax(1)
    # log q, log p to 8 EPS of their sizes; q to 2^-21 and the rounding of its exponent; q_T is 1 - sum q
    extra = (fin(log_tail) + 40.0) * (2 ** -19 + a * 8 * EPS) if tail else 0.0
    near(got.loss, loss, s + (2 ** -20 + 16 * EPS * (1 + a)) * (1 + big + a) + extra)
    if tail:
        near(got.log_tail, log_tail, 2 * s + 8 * EPS * fin(log_tail))
    if weight is not None:
        _near_distill_grad(got.grad, z, ids, u, scale, ts, tail, weight)


def _near_distill_grad(got, z, ids, u, scale, ts, tail, weight):
    want = ref.distill_grad(z, ids, u, scale, ts, tail, weight)
    lp, lse = ref.log_softmax(z, scale)
    p = lp.exp()
    q, rest = ref.teacher(ids, u, ts, tail)
    fin = lambda t: torch.where(torch.isfinite(t), t.abs(), torch.zeros(()).double())  # noqa: E731
    a = fin(u.double() * ts).amax(1)
    rel = sum_tol(z.shape[1]) + 8 * EPS * (fin(lp) + fin(lse)[:, None] + a[:, None] + 4) + 2 ** -20
    wt = weight.double().abs()[:, None] * scale
    qv = torch.zeros_like(p)
    for i in range(z.shape[0]):
        for j in range(ids.shape[1]):
            if ids[i, j] >= 0:
                qv[i, ids[i, j]] += q[i, j]
    terms = p * (1 + q.sum(1)[:, None]) + qv
    if tail:
        for i in range(z.shape[0]):
            out = torch.ones(z.shape[1], dtype=torch.bool)
            out[ids[i][ids[i] >= 0].long()] = False
            if out.any() and torch.isfinite(torch.logsumexp(lp[i][out], 0)):
                share = torch.where(out, (lp[i] - torch.logsumexp(lp[i][out], 0)).exp(), torch.zeros(()).double())
                # q_T is 1 - sum q: its error is absolute
                terms[i] += share * (rest[i] + 1.0)
    near(got, want, wt * rel * terms * 4 + HALF[z.dtype] * want.abs() + TINY[z.dtype] + 1e-30)


def _entries(N, V, K, tail, g, type_=F32):
    """Distinct ids and values; some rows are short, one has none."""
    ids = torch.stack([torch.randperm(V, generator=g)[:K] if V < 5000 else (torch.randint(0, V, (1,), generator=g) + torch.arange(K) * (V // K)) % V for _ in range(N)])
    u = torch.randn((N, ids.shape[1]), generator=g) * 2
    if tail:
        u = torch.log_softmax(u, 1) + math.log(0.9)
    if N > 2:
        ids[1, ids.shape[1] // 2:] = -1
        ids[2] = -1
    return ids, u.to(type_)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("type_,ttype,idt", [(F32, F32, torch.int64), (BF16, BF16, torch.int32), (F16, F32, torch.int64)])
@pytest.mark.parametrize("N,V,K", [(1, 1, 1), (1, 2, 1), (3, 7, 7), (4, 33, 5), (5, 256, 32), (37, 1000, 8), (3, 1023, 128), (4, 4099, 64), (3, 16384, 1),
                                   (3, 50003, 100), (2, 131072, 64), (1, 150001, 33)])
def test_distill(N, V, K, type_, ttype, idt, tail):
    g = gen(V + K)
    z = _logits("plain", N, V, type_, g)
    ids, u = _entries(N, V, K, tail, g, ttype)
    w = torch.randn(N, generator=g)
    ids = ids.to(idt)
    zd = z.cuda()
    got = lm().distill(zd, ids.cuda(), u.cuda(), scale=0.7, teacher_scale=0.9, tail=tail, weight=w.cuda())
    _near_distill(got, z, ids, u, 0.7, 0.9, tail, w)
    only = lm().distill(zd, ids.cuda(), u.cuda(), scale=0.7, teacher_scale=0.9, tail=tail)
    assert only.grad is None and torch.equal(only.loss, got.loss) and torch.equal(only.lse, got.lse)
    back = lm().distill_grad(zd, ids.cuda(), u.cuda(), got.lse, w.cuda(), scale=0.7, teacher_scale=0.9, tail=tail, log_tail=got.log_tail)
    _near_distill_grad(back, z, ids, u, 0.7, 0.9, tail, w)
    _near_distill_grad(lm().distill_grad(zd, ids.cuda(), u.cuda(), got.lse, 0.25, scale=0.7, teacher_scale=0.9, tail=tail, log_tail=got.log_tail),
                       z, ids, u, 0.7, 0.9, tail, torch.full((N,), 0.25))
    place = zd.clone()
    lm().distill_grad(place, ids.cuda(), u.cuda(), got.lse, w.cuda(), scale=0.7, teacher_scale=0.9, tail=tail, log_tail=got.log_tail, out=place)
    assert torch.equal(place, back)
    lm().distill(zd, ids.cuda(), u.cuda(), scale=0.7, teacher_scale=0.9, tail=tail, weight=w.cuda(), out=zd)
    assert torch.equal(zd, got.grad)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("kind", ["masked", "lowest", "equal", "few"])
@pytest.mark.parametrize("V,type_", [(50, F32), (3001, BF16), (40001, BF16), (140001, F32)])
def test_distill_under_masks(kind, V, type_, tail):
    N, K = 4, 9
    g = gen(V)
    z = _logits(kind, N, V, type_, g)
    ids, u = _entries(N, V, K, tail, g)
    w = torch.rand(N, generator=g) + 0.5
    got = lm().distill(z.cuda(), ids.cuda(), u.cuda(), tail=tail, weight=w.cuda())
    _near_distill(got, z, ids, u, 1.0, 1.0, tail, w)
    if kind != "lowest":                         # there lse in 32 bits has lost the log of the count
        back = lm().distill_grad(z.cuda(), ids.cuda(), u.cuda(), got.lse, w.cuda(), tail=tail, log_tail=got.log_tail)
        _near_distill_grad(back, z, ids, u, 1.0, 1.0, tail, w)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_special_entries(tail):
    """An id given twice; teacher's weight zero; ids over the whole vocabulary; a tail that the student all but rules out."""
    V = 12
    z = torch.randn((5, V), generator=gen(1))
    z[4, 8:] = -150.0
    ids = torch.tensor([[3, 3, 5, -1, 0, 1, 2, 4], [0, 1, 2, 3, 4, 5, 6, 7], [7, -1, 7, -1, 7, -1, 7, -1], [11, 10, 9, 8, 7, 6, 5, 4], list(range(8))])
    u = torch.log_softmax(torch.randn((5, 8), generator=gen(2)), 1) + math.log(0.8)
    u[3, 2:] = NEG
    w = torch.ones(5)
    got = lm().distill(z.cuda(), ids.cuda(), u.cuda(), tail=tail, weight=w.cuda())
    _near_distill(got, z, ids, u, 1.0, 1.0, tail, w)
    all_ids, all_u = torch.arange(V).expand(2, V).contiguous(), torch.log_softmax(torch.randn((2, V), generator=gen(4)), 1) + math.log(0.999)
    got = lm().distill(z[:2].cuda(), all_ids.cuda(), all_u.cuda(), tail=tail, weight=1.0)
    loss, _, _ = ref.distill(z[:2], all_ids, all_u, 1.0, 1.0, tail)
    if tail:
        assert bool((got.log_tail == NEG).all()) and bool((got.loss == float("inf")).all()) and bool((loss == float("inf")).all())
        assert bool(torch.isfinite(got.grad).all())
    else:
        _near_distill(got, z[:2], all_ids, all_u, 1.0, 1.0, False, torch.ones(2))


@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradient_against_differences(tail):
    N, V, K, step = 3, 19, 5, 1e-5
    g = gen(11)
    z = torch.randn((N, V), generator=g) * 2
    ids, u = _entries(N, V, K, tail, g)
    w = torch.rand(N, generator=g)
    got = lm().distill(z.cuda(), ids.cuda(), u.cuda(), scale=1.4, tail=tail, weight=w.cuda()).grad.cpu().double()
    for v in range(V):
        e = torch.zeros((N, V), dtype=torch.float64)
        e[:, v] = step
        up, down = (ref.distill(z.double() + s * e, ids, u, 1.4, 1.0, tail)[0] for s in (1, -1))
        diff = w.double() * (up - down) / (2 * step)
        assert float((diff - got[:, v]).abs().max()) < 1e-5


def test_cross_entropy_is_one_entry():
    """One entry per row is the cross entropy of its id: loss = -logp, gradient that of -logp."""
    N, V = 6, 777
    g = gen(2)
    z = torch.randn((N, V), generator=g).cuda()
    tok = torch.randint(0, V, (N,), generator=g).cuda()
    r = lm().token_logp(z, tok)
    d = lm().distill(z, tok[:, None].contiguous(), torch.zeros((N, 1), device="cuda"), weight=1.0)
    near(d.loss, -r.logp.double().cpu(), 1e-5)
    near(d.grad, lm().token_logp_grad(z, tok, r.lse, -1.0).double().cpu(), 1e-6)


def test_streams():
    """Work and results on a stream that is not the current one."""
    side = torch.cuda.Stream()
    z = torch.randn(64, 5000, generator=gen(1))
    zd, tok = z.cuda(), torch.arange(64).cuda()
    torch.cuda.synchronize()
    r = lm().token_logp(zd, tok, top=3, stream=side)
    g = lm().token_logp_grad(zd, tok, r.lse, stream=side)
    e = lm().embed_grad(tok, g, 70, stream=side)
    side.synchronize()
    want = ref.token_logp(z, tok.cpu(), 1.0, 3)
    assert torch.equal(r.top_ids.cpu(), want[3])
    near(r.logp, want[0], 1e-5)
    assert torch.equal(e[:64], g) and bool((e[64:] == 0).all())


def test_calls_are_captured_in_a_graph():
    z, tok = torch.randn(8, 3000).cuda(), torch.arange(8).cuda()
    u = torch.zeros(8, 1, device="cuda")

    def step():
        r = lm().token_logp(z, tok, top=2)
        d = lm().distill(z, tok[:, None], u, weight=1.0)
        return r.logp, r.top_ids, d.loss, lm().embed_grad(tok, d.grad, 9), lm().embed(tok, z)

    eager = step()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(eager, out):
        assert torch.equal(a, b)


# ------------------------------------------------------------------ refusals
def test_refusals():
    m = lm()
    from paper_1906_02367_b200 import binding as B
    z, tok = torch.zeros(4, 10).cuda(), torch.zeros(4, dtype=torch.int64).cuda()
    table = torch.zeros(10, 8).cuda()
    lse, ids, u = torch.zeros(4).cuda(), torch.zeros(4, 2, dtype=torch.int64).cuda(), torch.zeros(4, 2).cuda()
    bad = [
        lambda: m.embed(tok.float(), table), lambda: m.embed(tok, table.double()), lambda: m.embed(tok.cpu(), table), lambda: m.embed(tok, table.cpu()),
        lambda: m.embed(tok, table.t()), lambda: m.embed(tok, table, out=torch.zeros(4, 9).cuda()), lambda: m.embed(tok, torch.zeros(2, 10, 8).cuda()),
        lambda: m.embed(tok[::2], table), lambda: m.embed_grad(tok, torch.zeros(3, 8).cuda(), 10), lambda: m.embed_grad(tok, z, 10, accumulate=True),
        lambda: m.embed_grad(tok, z, 10, out=torch.zeros(9, 10).cuda()), lambda: m.embed_grad(tok, z, 10, out=torch.zeros(10, 10).cuda().half()),
        lambda: m.token_logp(z[0], tok), lambda: m.token_logp(z, tok[:3]), lambda: m.token_logp(z.t(), tok), lambda: m.token_logp(z, tok, top=11),
        lambda: m.token_logp(z, tok, top=-1), lambda: m.token_logp(torch.zeros(4, 200).cuda(), tok, top=129), lambda: m.token_logp(z.double(), tok),
        lambda: m.token_logp(z, tok.short()), lambda: m.token_logp_grad(z, tok, lse[:3]), lambda: m.token_logp_grad(z, tok, lse, grad_entropy=lse),
        lambda: m.token_logp_grad(z, tok, lse, out=z.half()), lambda: m.token_logp_grad(z, tok, lse, lse[:2]), lambda: m.token_logp_grad(z, tok, lse.half()),
        lambda: m.distill(z, ids, u[:, :1]), lambda: m.distill(z, ids[:3], u[:3]), lambda: m.distill(z, ids[:, :0], u[:, :0]),
        lambda: m.distill(z, torch.zeros(4, 129, dtype=torch.int64).cuda(), torch.zeros(4, 129).cuda()), lambda: m.distill(z, ids, u, out=z),
        lambda: m.distill(z, ids, u, weight=lse[:1]), lambda: m.distill_grad(z, ids, u, lse, 1.0, tail=True), lambda: m.distill(z, ids, u.double()),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("case", i)
    buf = torch.zeros(100).cuda()
    refused = [
        lambda: m.token_logp(z, tok, scale=0.0), lambda: m.token_logp(z, tok, scale=-1.0), lambda: m.token_logp(z, tok, scale=NAN),
        lambda: m.token_logp(z, tok, scale=float("inf")), lambda: m.distill(z, ids, u, teacher_scale=NAN),
        lambda: m.token_logp(torch.as_strided(buf, (4, 10), (9, 1)), tok),
        lambda: m.token_logp_grad(torch.as_strided(buf, (4, 10), (10, 1)), tok, lse, out=torch.as_strided(buf, (4, 10), (10, 1), 1)),
        lambda: m.distill(torch.as_strided(buf, (4, 10), (10, 1)), ids, u, weight=1.0, out=torch.as_strided(buf, (4, 10), (12, 1))),
        lambda: m.embed_grad(tok, z, 10, workers=False, out=torch.as_strided(buf, (10, 10), (9, 1))),
        lambda: m.embed_grad(tok.view(2, 2), z.view(2, 2, 10), 5, out=torch.as_strided(buf, (2, 5, 10), (3, 10, 1))),
        lambda: m.embed(torch.zeros((33, 1), dtype=torch.int64).cuda(), torch.zeros(33, 2, 4).cuda()),
    ]
    for call in refused:
        with pytest.raises(B.QsError) as e:
            call()
        assert e.value.code == B.QS_INVALID_ARG
    with pytest.raises(B.QsError) as e:
        m.embed_grad(tok, z, 10, work=torch.zeros(16, dtype=torch.uint8).cuda())
    assert e.value.code == B.QS_CAPACITY
    torch.cuda.synchronize()
    # calls without rows do nothing; a gradient without tokens is zero
    none = torch.zeros(0, dtype=torch.int64).cuda()
    assert m.embed(none, table).shape == (0, 8) and m.token_logp(z[:0], none, top=2).top_ids.shape == (0, 2)
    assert m.distill(z[:0], ids[:0], u[:0], weight=1.0).grad.shape == (0, 10)
    assert float(m.embed_grad(none, torch.zeros(0, 8).cuda(), 10, out=torch.ones(10, 8).cuda()).abs().sum()) == 0.0


def test_limits_of_the_c_calls():
    """Sizes and pointers, on the host alone: nothing is enqueued."""
    from paper_1906_02367_b200 import binding as B
    L = B.lib()
    big = (1 << 30) + 1
    p = torch.zeros(64).cuda().data_ptr()
    assert L.qs_embed(1, 4, big, 8, p, 0, p, 0, 0, 8, 1.0, p, 0, 8, None, None) == B.QS_TOO_LARGE
    assert L.qs_embed(1, 4, 4, 8, p, 0, p, 3, 0, 8, 1.0, p, 0, 8, None, None) == B.QS_INVALID_ARG
    assert L.qs_embed(1, 4, 4, 8, p, 1, p, 0, 0, 8, 1.0, None, 0, 8, None, None) == B.QS_INVALID_ARG
    assert L.qs_embed(1, 4, 4, 8, p + 4, 1, p, 0, 0, 8, 1.0, p, 0, 8, None, None) == B.QS_INVALID_ARG
    assert L.qs_embed_grad_bytes(0, 1, 1, 1) == B.QS_INVALID_ARG and L.qs_embed_grad_bytes(1, 1, big, 1) == B.QS_TOO_LARGE
    assert L.qs_token_logp(1, big, p, 0, big, p, 0, 1.0, 0, p, p, p, None, None, None, None) == B.QS_TOO_LARGE
    assert L.qs_token_logp(1, 8, p, 0, 8, None, 0, 1.0, 0, p, p, p, None, None, None, None) == B.QS_INVALID_ARG
    assert L.qs_token_logp(1, 8, p, 0, 8, p, 0, 1.0, 2, p, p, p, None, None, None, None) == B.QS_INVALID_ARG
    assert L.qs_token_logp(1, 8, p + 2, 0, 8, p, 0, 1.0, 0, p, p, p, None, None, None, None) == B.QS_INVALID_ARG
    assert L.qs_distill_grad(1, 8, 1, p, 0, 8, p, 0, p, 0, 1.0, 1.0, 1, p, None, None, 1.0, p, 8, None, None) == B.QS_INVALID_ARG
