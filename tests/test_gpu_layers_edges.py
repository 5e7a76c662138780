"""The operators of a residual block where they can go wrong: other streams, captured graphs, wide strides, boundaries between
forms, waits that run out, a caller's workspace, and a whole block of them."""
import os
import subprocess
import sys

import pytest
import torch

import layers_reference as ref
from test_gpu_layers import BF16, E, F16, F32, U, near, rand

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.fixture
def L():
    from paper_1906_02367_b200 import layers
    return layers


def everything(L, dtype=BF16, M=300, N=520, K=264, seed=1, **kw):
    """One call of each operator; a list of results."""
    x, w, g, z = rand((M, K), dtype, seed), rand((N, K), F32, seed + 1, K ** -0.5), rand((M, N), dtype, seed + 2, 0.1), rand((M, N), dtype, seed + 3)
    nw, res = rand((K,), F32, seed + 4, 0.1, 1.0), rand((M, K), dtype, seed + 5)
    torch.cuda.synchronize()

    def run():
        n = L.rms_norm(x, nw, res, **kw)
        q = L.rms_norm(x, nw, res, quantize=True, **kw)
        w8 = L.quantize(w, **kw)
        y = L.linear(n.out, w, activation="gelu", save=True, **kw)
        y8 = L.linear(q.out, w8.values, x_scale=q.scale, weight_scale=w8.scale, **kw)
        d = L.dropout(y.out, 0.3, 5, residual=z, **kw)
        few = L.linear(x[:5], w, **kw)
        r = L.linear_grad(g, x, w, z, "silu", bias=True, **kw)
        dn = L.rms_norm_grad(r.x, n.hidden, n.rstd, nw, grad_hidden=res, **kw)
        return [n.out, n.hidden, n.rstd, q.out.float(), q.scale, w8.values.float(), w8.scale, y.out, y.pre, y8.out, d, few.out, r.x, r.weight, r.bias, dn.hidden, dn.weight]
    return run


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_on_another_stream(L, dtype):
    want = everything(L, dtype)()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    run = everything(L, dtype, stream=side)
    got = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(side):
        got = everything(L, dtype)()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_streams_at_once(L):
    """Large and small calls side by side: each has scratch of its own, and the blocks of one wait for no other's."""
    runs = [everything(L, BF16, 2000, 1030, 512, seed=1), everything(L, F32, 700, 300, 264, seed=9)]
    want = [r() for r in runs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, r in zip(streams, runs):
            with torch.cuda.stream(s):
                got.append(r())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_captured_and_replayed(L, dtype):
    """Two graphs of the same calls on other inputs, replayed in turn and together with eager calls."""
    runs = [everything(L, dtype, seed=1), everything(L, dtype, seed=40)]
    want = [[t.clone() for t in r()] for r in runs]
    graphs, got = [], []
    for r in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(r())
        graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for i in order:
            for t in got[i]:
                t.zero_()
            graphs[i].replay()
            runs[1 - i]()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_rows_far_apart(L):
    """Offsets past 2^32 elements."""
    step = (1 << 31) + 64
    buf = torch.empty(2 * step + (1 << 21), device="cuda", dtype=BF16)
    x = buf.as_strided((3, 264), (step, 1))
    x.copy_(rand((3, 264), BF16, 1))
    c, w, nw = x.clone(), rand((40, 264), BF16, 2), rand((264,), F32, 3)
    far = [L.rms_norm(x, nw), L.quantize(x), L.linear(x, w), L.linear_grad(rand((3, 40), BF16, 4), x, w), L.rms_norm_grad(x, x, torch.ones(3, device="cuda"), nw)]
    close = [L.rms_norm(c, nw), L.quantize(c), L.linear(c, w), L.linear_grad(rand((3, 40), BF16, 4), c, w), L.rms_norm_grad(c, c, torch.ones(3, device="cuda"), nw)]
    for a, b in zip(far, close):
        assert all(s is None or torch.equal(s.float(), t.float()) for s, t in zip(a, b))
    assert torch.equal(L.dropout(x, 0.5, 1), L.dropout(c, 0.5, 1))
    y = buf[1 << 20:].as_strided((3, 264), (step, 1))
    L.dropout(c, 0.5, 1, out=y)
    assert torch.equal(y, L.dropout(c, 0.5, 1))
    L.linear(c, rand((264, 264), BF16, 5), out=y)
    near(y, ref.product(c, rand((264, 264), BF16, 5))[0], 272 * E * ref.product(c, rand((264, 264), BF16, 5))[1], BF16)
    # tiles by the matrix unit from and to such rows
    big = torch.empty(40 * (1 << 27) + 4096, device="cuda", dtype=BF16).as_strided((40, 512), (1 << 27, 1))
    big.copy_(rand((40, 512), BF16, 6))
    assert torch.equal(L.linear(big, rand((256, 512), BF16, 7)).out, L.linear(big.clone(), rand((256, 512), BF16, 7)).out)
    L.linear(big.clone(), rand((512, 512), BF16, 8), out=big)
    assert bool(torch.isfinite(big).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M", [1, 7, 8, 9, 16, 17, 31, 32, 33, 127, 128, 129])
@pytest.mark.parametrize("N,K", [(48, 640), (300, 1027)])
def test_boundaries_between_forms(L, dtype, M, N, K):
    x, w, b = rand((M, K), dtype, 1), rand((N, K), F32, 2, K ** -0.5), rand((N,), F32, 3)
    z, size = ref.product(x, w.to(dtype))
    near(L.linear(x, w, b).out, z + b.double(), ((K + 8) * E * 1.05 + 6 * E) * (size + b.double().abs()), dtype)


@pytest.mark.parametrize("M,N,K", [(64, 80, 5000), (40, 64, 16384), (64, 256, 9000), (3000, 64, 2100), (256, 2304, 2176)])
def test_long_sums_keep_32_bits(L, M, N, K):
    """Results in fp32 of long sums that have one sign: what is cut at every addition adds up.  1024 elements, the least
    that are summed by the matrix unit in one go, cut off 1024 / 16 steps of at most 2^-23 each; in the mean half of that."""
    x, w = rand((M, K), BF16, 1).abs(), rand((N, K), BF16, 2).abs()
    z, _ = ref.product(x, w)
    off = ((L.linear(x, w, dtype=F32).out.double() - z) / z).abs()
    assert float(off.max()) < 64 * E + (K / 1024 + 2) * E, float(off.max())
    g = L.linear_grad(rand((K, N), BF16, 3).abs(), rand((K, M), BF16, 4).abs(), rand((N, M), BF16, 5), need_x=False).weight
    z, _ = ref.product(rand((K, N), BF16, 3).abs().t(), rand((K, M), BF16, 4).abs().t())
    assert float(((g.double() - z) / z).abs().max()) < 64 * E + (K / 1024 + 2) * E
    f, v = rand((M, K), F32, 6).abs(), rand((N, K), F32, 7).abs()
    z, _ = ref.product(f, v)
    # (and of three parts, at most 2^-21 left out)
    assert float(((L.linear(f, v).out.double() - z) / z).abs().max()) < 64 * E + (K / 1024 + 2) * E + 2.0 ** -21


@pytest.mark.parametrize("M,N,K", [(2000, 520, 3000), (150, 264, 2500), (2000, 519, 1100)])
def test_fp32_results_in_several_sums_with_all_that_follows(L, M, N, K):
    x, w, b, res = rand((M, K), BF16, 1), rand((N, K), BF16, 2, K ** -0.5), rand((N,), F32, 3), rand((M, N), F32, 4)
    r = L.linear(x, w, b, activation="gelu", residual=res, save=True, dtype=F32)
    z, size = ref.product(x, w)
    z, slack = z + b.double(), (K + 8) * E * size + 2 * E * b.double().abs()
    near(r.pre, z, slack, F32)
    near(r.out, ref.activate(z, "gelu") + res.double(), 1.13 * slack + 8 * E * (z.abs() + 1) + 2 * E * res.double().abs(), F32)
    L.linear(x, w, b, activation="gelu", residual=res, out=res)
    near(res, r.out, 2 * (1.13 * slack + 8 * E * (z.abs() + 1) + 2 * E * r.out.double().abs()), F32)


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("M,N,K", [(3000, 264, 520), (100, 1300, 1096), (300, 65, 130), (40, 8, 8)])
def test_weight_gradients_added_to_what_is_there(L, dtype, out, M, N, K):
    g, x, held = rand((M, N), dtype, 1, 0.1), rand((M, K), dtype, 2), rand((N, K), out, 3)
    w = torch.zeros((N, K), device="cuda", dtype=dtype)
    want, size = ref.product(g.t(), x.t())
    got = held.clone()
    L.linear_grad(g, x, w, need_x=False, out_weight=got, accumulate=True)
    near(got, want + held.double(), ((M + 8) * E * 1.05 + 4 * E) * size + 2 * E * held.double().abs(), out)


def test_a_callers_workspace(L):
    from paper_1906_02367_b200.binding import QS_CAPACITY, QsError
    x, w = rand((300, 257), F32, 1), rand((200, 257), F32, 2)
    need = 1 << 23
    work = torch.zeros(need, dtype=torch.uint8, device="cuda")
    assert torch.equal(L.linear(x, w, work=work).out, L.linear(x, w).out)
    with pytest.raises(QsError) as e:
        L.linear(x, w, work=work[:4096])
    assert e.value.code == QS_CAPACITY
    with pytest.raises(QsError):
        L.linear(x, w, work=work[8:])
    guard = torch.full((need + 512,), 7, dtype=torch.uint8, device="cuda")
    from paper_1906_02367_b200.binding import QS_F32, lib
    n = lib().qs_linear_bytes(1, 300, 200, 257, x.data_ptr(), QS_F32, 257, w.data_ptr(), QS_F32, 0, 257)
    L.linear(x, w, work=guard[256:256 + n])
    assert bool((guard[:256] == 7).all()) and bool((guard[256 + n:] == 7).all())
    h, r, nw = rand((300, 257), F32, 3), torch.ones(300, device="cuda"), rand((257,), F32, 4)
    n = lib().qs_rms_norm_grad_bytes(1, 300, 257)
    guard.fill_(7)
    guard = torch.full((n + 512,), 7, dtype=torch.uint8, device="cuda")
    a = L.rms_norm_grad(h, h, r, nw, work=guard[256:256 + n])
    assert torch.equal(a.weight, L.rms_norm_grad(h, h, r, nw).weight) and bool((guard[:256] == 7).all()) and bool((guard[256 + n:] == 7).all())
    with pytest.raises(QsError):
        L.rms_norm_grad(h, h, r, nw, work=guard[256:256 + n - 4])


def test_results_stay_inside(L):
    """Nothing around a result is written: odd sizes in the middle of a buffer, every form."""
    for M, N, K, out_type in ((1, 33, 64, BF16), (40, 65, 130, BF16), (200, 129, 200, F32), (130, 264, 192, F16), (5, 257, 129, F32), (300, 300, 2200, F32)):
        dtype = out_type if out_type != F32 or M == 5 else BF16
        x, w = rand((M, K), dtype, 1), rand((N, K), dtype, 2)
        for pad in (0, 8, 5):
            buf = torch.full((64 + M * (N + pad) + 64,), 7.0, device="cuda", dtype=out_type)
            out = buf[64:64 + M * (N + pad)].view(M, N + pad)[:, :N]
            assert torch.equal(L.linear(x, w, out=out).out, L.linear(x, w, dtype=out_type).out)
            rest = buf.clone()
            rest[64:64 + M * (N + pad)].view(M, N + pad)[:, :N] = 7.0
            assert bool((rest == 7).all())


WAITS = """
import torch, sys
sys.path.insert(0, {root!r})
from paper_1906_02367_b200 import layers as L
x, w = torch.randn(2000, 256, device="cuda").bfloat16(), torch.randn(1100, 256, device="cuda").bfloat16()
status = torch.zeros(1, dtype=torch.int32, device="cuda")
y = L.linear(x, w, status=status).out
g = L.linear_grad(y, x, w, status=status)
f = L.linear(x[:200].float(), w.float(), status=status).out
torch.cuda.synchronize()
print("status", int(status), "nan", bool(torch.isnan(y).all()), bool(torch.isnan(g.weight).all()), bool(torch.isnan(f).all()),
      "fine", bool(torch.isfinite(y).all() and torch.isfinite(g.weight).all() and torch.isfinite(f).all()))
"""


@pytest.mark.parametrize("limit,words", [("0", "status -7 nan True True True fine False"), ("1000000000", "status 0 nan False False False fine True")])
def test_waits_that_run_out_leave_nan(limit, words):
    p = subprocess.run([sys.executable, "-c", WAITS.format(root=ROOT)], env={**os.environ, "QSPARSE_WAIT_LIMIT_NS": limit}, capture_output=True, text=True, timeout=120)
    assert p.returncode == 0 and words in p.stdout, (p.stdout, p.stderr[-2000:])


@pytest.mark.parametrize("vocab,width,blocks", [(300, 64, 2), (77, 5, 1)])
def test_gradient_of_blocks_in_the_example(vocab, width, blocks):
    """The example's whole step with residual blocks, dropout included, against automatic differentiation in 64 bits."""
    import distill_language_model as ex
    R, N, K, key = 3, 40, 6, (11, (1 << 32) + 5)
    student = ex.Student(vocab, width, blocks, drop=0.3)
    flat = rand((R, student.d), F32, 1, 0.1)
    grad = torch.full_like(flat, 7.0)
    g = torch.Generator(device="cuda").manual_seed(3)
    tokens = torch.randint(0, vocab, (R, N), generator=g, device="cuda")
    ids, logp = ex.teacher_entries(rand((vocab, vocab), F32, 2, 2.0), tokens, K)
    loss = student.gradient(flat, grad, tokens, ids, logp, key)
    w = flat.double().cpu().requires_grad_()
    table, bias = student.views(w)
    keep = [torch.stack([torch.from_numpy(ref.words(N * width, r, key[0], key[1], i) >= int(0.3 * 2 ** 32)) for r in range(R)]).view(R, N, width)
            for i in range(blocks)]
    total, rows = 0.0, []
    for r in range(R):
        h = table[r][tokens[r].cpu()] * student.scale
        for i in range(blocks):
            norm, w1, b1, w2, b2 = (t[r] for t in student.block(w, i))
            n = h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * norm
            u = ref.activate(n @ w1.t() + b1, "gelu") @ w2.t() + b2
            h = h + torch.where(keep[i][r], u / 0.7, torch.zeros_like(u))
        lp = torch.log_softmax(h @ table[r].t() + bias[r], 1)
        i, q = ids.view(R, N, K)[r].cpu(), logp.view(R, N, K)[r].double().cpu().exp()
        rest = 1 - q.sum(1)
        out = torch.ones(N, vocab, dtype=torch.bool).scatter_(1, i, False)
        row = (q * (q.log() - lp.gather(1, i))).sum(1) + rest * (rest.log() - torch.logsumexp(lp.masked_fill(~out, float("-inf")), 1))
        rows.append(row)
        total = total + row.mean()
    total.backward()
    # fp32 sums of up to 300 terms through three products a block: 1e-4 of the largest entry is a wide bound
    scale = float(w.grad.abs().max())
    assert float((grad.double().cpu() - w.grad).abs().max()) <= 1e-4 * scale
    assert float((loss.double().cpu() - torch.cat(rows).detach()).abs().max()) <= 1e-4


def test_the_example_runs_with_blocks():
    import distill_language_model as ex
    got = ex.run(steps=4, blocks=2, eta=2.0)
    assert len(got["losses"]) == 4 and all(v == v and abs(v) < 1e4 for v in got["losses"])
    assert ex.run(steps=2, blocks=2, eta=2.0)["losses"][0] == got["losses"][0]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_a_block_and_its_gradient(L, dtype):
    """Norm, product with activation, product with the residual, dropout, and back, for three workers: every operator on what the
    one before it left, compared with the same step in 64 bits on the same operands."""
    R, M, D, H = 3, 150, 72, 200
    flat = rand((R, D + H * D + H + D * H + D), F32, 1, 0.1)
    at = [0]

    def cut(*shape):
        n = int(torch.tensor(shape).prod())
        at[0] += n
        return flat[:, at[0] - n:at[0]].view(R, *shape)
    norm, w1, b1, w2, b2 = cut(D), cut(H, D), cut(H), cut(D, H), cut(D)
    h, dh = rand((R, M, D), dtype, 2), rand((R, M, D), dtype, 3, 0.1)
    n = L.rms_norm(h, norm)
    a = L.linear(n.out, w1, b1, activation="silu", save=True)
    u = L.linear(a.out, w2, b2, residual=h)
    out = L.dropout(u.out, 0.2, 9, layer=3, workers=True, residual=h)
    y, _, rstd = ref.rms_norm(h, norm, None, 1e-6)
    near(n.out, y, (D / 2 + 9) * E * y.abs(), dtype)
    z, size = ref.product(n.out, w1.to(dtype))
    z, slack = z + b1.double()[:, None], ((D + 8) * E * 1.05 + 6 * E) * (size + b1.double().abs()[:, None])
    near(a.pre, z, slack, dtype)
    near(a.out, ref.activate(z, "silu"), 1.13 * slack + 8 * E * (z.abs() + 1), dtype)
    z, size = ref.product(a.out, w2.to(dtype))
    near(u.out, z + b2.double()[:, None] + h.double(), ((H + 8) * E * 1.05 + 8 * E) * (size + b2.double().abs()[:, None] + h.double().abs()), dtype)
    near(out, ref.dropout(u.out, 0.2, 9, 0, 3, 0, h, True), 3 * E * (u.out.double().abs() * 1.25 + h.double().abs()), dtype)
    du = L.dropout(dh, 0.2, 9, layer=3, workers=True)
    near(du, ref.dropout(dh, 0.2, 9, 0, 3, 0, None, True), 3 * E * dh.double().abs(), dtype)
    g2 = L.linear_grad(du, a.out, w2, bias=True)
    dz, size = ref.product(du, w2.to(dtype).transpose(1, 2))
    near(g2.x, dz, ((D + 8) * E * 1.05 + 4 * E) * size, dtype)
    g1 = L.linear_grad(g2.x, n.out, w1, a.pre, "silu", bias=True)
    want = g2.x.double() * ref.slope(a.pre.double(), "silu")
    near(g1.pre, want, 8 * E * g2.x.double().abs() * (1 + a.pre.double().abs()), dtype)
    dw, size = ref.product(g1.pre.transpose(1, 2), n.out.transpose(1, 2))
    near(g1.weight, dw, ((M + 8) * E * 1.05 + 4 * E) * size, F32)
    r = L.rms_norm_grad(g1.x, n.hidden, n.rstd, norm, grad_hidden=dh)
    d, _, _ = ref.rms_norm_grad(g1.x, h, n.rstd, norm, dh)
    wg = (g1.x.double() * norm.double()[:, None]).abs()
    nn = (h.double() * n.rstd.double()[..., None]).abs()
    near(r.hidden, d, n.rstd.double()[..., None] * (6 * E * wg + nn * (D + 8) * E * (wg * nn).mean(-1, keepdim=True)) + 4 * E * (d.abs() + dh.double().abs()), dtype)


def test_half_steps_are_what_the_bounds_count():
    for t, u in U.items():
        assert u == torch.finfo(t).eps / 2
