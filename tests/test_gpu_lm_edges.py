"""Language-model operators at the edges of their types and sizes: rows whose lse has lost its fractions, or passes the
largest number; NaN and infinities; paths that only long lists and long rows take; calls from several threads.
Tolerances as in test_gpu_lm.py: EPS is half a unit in the last place of fp32, an exponential is off by 2^-21, a sum of n
terms by n EPS of their magnitudes."""
import math
import os
import subprocess
import sys
import threading

import pytest
import torch

from tests import lm_reference as ref
from tests.test_gpu_lm import BF16, EPS, F16, F32, HALF, NAN, NEG, TINY, _near_distill, _near_logp_grad, gen, near, sum_tol, view

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INF = float("inf")
SAVED = 256.0                                    # an lse up to here is taken as it is: off by EPS of it


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def lm():
    from paper_1906_02367_b200 import lm as module
    return module


def clip(t, most):
    return torch.where(torch.isfinite(t), t.abs().clamp_max(most), torch.zeros((), dtype=t.dtype))


# ------------------------------------------------------------------ an lse beyond the largest number
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V,type_", [(50, F32), (3001, BF16), (40001, BF16), (140001, F32)])
def test_rows_at_the_lowest_value_with_a_scale_above_one(V, type_, tail):
    """scale * lowest is no finite fp32 number, but the row has live columns: every one of them has the share 1 / V."""
    N, K, scale = 3, 5, 1.25
    g = gen(V)
    z = torch.randn((N, V), generator=g)
    z[0] = torch.finfo(type_).min
    z[1] = NEG
    z = z.to(type_)
    tok = torch.tensor([V // 2, 0, 1])
    r = lm().token_logp(z.cuda(), tok.cuda(), scale=scale, top=2)
    assert float(r.lse[0]) == -torch.finfo(F32).max and float(r.lse[1]) == NEG
    s = sum_tol(V) + 8 * EPS * math.log(V)
    assert abs(float(r.logp[0]) + math.log(V)) <= s and abs(float(r.entropy[0]) - math.log(V)) <= 4 * s
    assert r.top_ids[:2].tolist() == [[0, 1], [-1, -1]]
    ids = torch.arange(K).expand(N, K).contiguous() * (V // K)
    u = torch.log_softmax(torch.randn((N, K), generator=g), 1) - 0.3
    got = lm().distill(z.cuda(), ids.cuda(), u.cuda(), scale=scale, tail=tail, weight=2.0)
    assert float(got.lse[0]) == -torch.finfo(F32).max
    q, rest = ref.teacher(ids, u, 1.0, tail)
    want = float((q[0] * (q[0].log() + math.log(V))).sum())
    if tail:
        want += float(rest[0] * (rest[0].log() - math.log((V - K) / V)))
    assert abs(float(got.loss[0]) - want) <= 2 * s + 2 ** -17
    want, tol = far_distill_grad(z, ids, u, scale, tail, torch.full((N,), 2.0))
    near(got.grad, want, tol)
    assert float(got.loss[1]) == INF and bool((got.grad[1] == 0).all())


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V,type_", [(50, F32), (3001, BF16), (40001, BF16), (140001, F32)])
def test_backward_calls_at_the_lowest_value_with_a_scale_above_one(V, type_, tail):
    N, K, scale = 3, 5, 1.25
    g = gen(V)
    z = torch.randn((N, V), generator=g)
    z[0] = torch.finfo(type_).min
    z[1] = NEG
    z = z.to(type_)
    tok = torch.tensor([V // 2, 0, 1])
    ids = torch.arange(K).expand(N, K).contiguous() * (V // K)
    u = torch.log_softmax(torch.randn((N, K), generator=g), 1) - 0.3
    want, tol = far_distill_grad(z, ids, u, scale, tail, torch.full((N,), 2.0))
    got = lm().distill(z.cuda(), ids.cuda(), u.cuda(), scale=scale, tail=tail)
    near(lm().distill_grad(z.cuda(), ids.cuda(), u.cuda(), got.lse, 2.0, scale=scale, tail=tail, log_tail=got.log_tail), want, tol)
    r, gl = lm().token_logp(z.cuda(), tok.cuda(), scale=scale), torch.ones(N)
    want, tol = far_logp_grad(z, tok, scale, gl, gl)
    near(lm().token_logp_grad(z.cuda(), tok.cuda(), r.lse, 1.0, scale=scale, entropy=r.entropy, grad_entropy=gl.cuda()), want, tol)


@pytest.mark.parametrize("type_", [F32, BF16])
@pytest.mark.parametrize("V", [40, 5001])
def test_losses_at_columns_of_the_lowest_value(V, type_):
    """log p = scale * lowest is no fp32 number, its product with a small share is; a loss that is none is the largest one,
    and only a column at -inf makes it infinite."""
    low, most, scale = torch.finfo(type_).min, torch.finfo(F32).max, 1.25
    z = torch.full((3, V), low).to(type_)
    z[:, 0] = 0.0
    z[2, 7] = NEG
    ids = torch.tensor([[0, 5], [5, -1], [0, 7]])
    u = torch.tensor([[0.9, 0.1], [1.0, 1.0], [0.9, 0.1]]).log()
    got = lm().distill(z.cuda(), ids.cuda(), u.cuda(), scale=scale, weight=1.0)
    want = -0.1 * scale * low
    assert abs(float(got.loss[0]) - want) <= 2 ** -20 * want and got.loss[1:].tolist() == [most, INF]
    assert got.lse.tolist() == [0.0] * 3
    # the rest of the teacher's mass on columns at the lowest value
    got = lm().distill(z.cuda(), ids[:, :1].contiguous().cuda(), torch.tensor([[0.9], [1.0], [0.9]]).log().cuda(), scale=scale, tail=True, weight=1.0)
    assert abs(float(got.loss[0]) - want) <= 2 ** -20 * want and float(got.log_tail[0]) == -most
    assert float(got.loss[1]) == most and abs(float(got.loss[2]) - want) <= 2 ** -20 * want


@pytest.mark.parametrize("type_,value", [(F32, -1e9), (F32, torch.finfo(F32).min), (F32, -300.0), (BF16, -1e9), (F16, -60000.0)])
@pytest.mark.parametrize("V", [40, 5001, 300007])
@pytest.mark.parametrize("scale", [1.0, 1.25])
def test_gradient_outside_ids_that_are_all_live(V, type_, value, scale):
    """The student's mass outside the ids is next to nothing, at columns masked with a finite value: the teacher's rest of the
    mass pulls at each of them by its share of that nothing."""
    z = torch.full((2, V), value).to(type_)
    z[:, 0] = 0.0
    z[1, V // 2:] = NEG
    ids, u = torch.zeros((2, 1), dtype=torch.int64), torch.full((2, 1), math.log(0.9))
    got = lm().distill(z.cuda(), ids.cuda(), u.cuda(), scale=scale, tail=True, weight=1.0)
    rest = 1.0 - float(u[0, 0].double().exp())
    for i, live in enumerate((V - 1, V // 2 - 1)):
        grad = torch.zeros(V, dtype=torch.float64)
        grad[1:live + 1] = -rest * scale / live
        grad[0] = rest * scale
        # q_T is 1 - q, q off by 2^-21 of it
        near(got.grad[i], grad, (2 ** -21 / rest + sum_tol(V) + 2 ** -20 + 2 * HALF[type_]) * grad.abs() + TINY[type_])


# ------------------------------------------------------------------ backward calls where lse has lost its fractions
FAR = ["masked", "lowest", "high", "low", "flat", "plain", "empty", "one", "thin"]


def far_rows(V, type_, g):
    """A row of each kind; `where` masks are finite: -1e9 (fp16: its lowest value)."""
    mask = torch.finfo(type_).min if type_ == F16 else -1e9
    z = torch.randn((len(FAR), V), generator=g) * 2
    z[0] = mask                                  # everything masked: uniform
    z[1] = torch.finfo(type_).min
    z[2] += 9000.0
    z[3] -= 9000.0
    z[4] = 3000.0
    z[6] = NEG
    z[7] = mask
    z[7, V // 3] = -5.0                          # one live column
    z[8] = mask                                  # the first four live
    z[8, :4] = torch.tensor([1.0, 2.0, 0.5, 0.0])
    return z.to(type_)


def far_logp_grad(z, tok, scale, gl, ge):
    want = ref.token_logp_grad(z, tok, scale, gl, ge)
    lp, lse = ref.log_softmax(z, scale)
    p = lp.exp()
    l0 = torch.where(p > 0, clip(lp, 1e4), torch.zeros(()).double())
    ent = (p * l0).sum(1, keepdim=True)
    rel = sum_tol(z.shape[1]) + 8 * EPS * (l0 + clip(lse, SAVED)[:, None] + 1)
    terms = scale * p * (gl.double().abs()[:, None] + ge.double().abs()[:, None] * (l0 + ent + 1))
    hot = torch.zeros_like(p)
    for i, t in enumerate(tok.tolist()):
        if t >= 0:
            hot[i, t] = abs(float(gl[i])) * scale
    return want, rel * terms * 4 + 4 * EPS * hot + HALF[z.dtype] * want.abs() + TINY[z.dtype] + 1e-30


FAR_SIZES = [(37, F32), (3001, BF16), (5003, F16), (50003, BF16), (140001, F32), (300007, BF16), (270011, F32)]


@pytest.mark.parametrize("V,type_", FAR_SIZES)
@pytest.mark.parametrize("entropy", [False, True])
def test_token_logp_gradient_where_lse_is_large(V, type_, entropy):
    g = gen(V)
    z = far_rows(V, type_, g)
    N, scale = z.shape[0], 1.0
    tok = torch.randint(0, V, (N,), generator=g)
    tok[7] = V // 3
    gl, ge = torch.randn(N, generator=g), torch.randn(N, generator=g) if entropy else torch.zeros(N)
    zd, _ = view(z, 3, 1)
    r = lm().token_logp(zd, tok.cuda(), scale=scale)
    extra = dict(entropy=r.entropy, grad_entropy=ge.cuda()) if entropy else {}
    want, tol = far_logp_grad(z, tok, scale, gl, ge)
    got = lm().token_logp_grad(zd, tok.cuda(), r.lse, gl.cuda(), scale=scale, **extra)
    near(got, want, tol)
    near(lm().token_logp_grad(zd, tok.cuda(), r.lse, gl.cuda(), scale=scale, out=zd, **extra), want, tol)     # in place
    # one row at a time: as many blocks as a row takes
    for i in (0, 8):
        zi = z[i:i + 1].cuda()
        one = lm().token_logp_grad(zi, tok[i:i + 1].cuda(), r.lse[i:i + 1], gl[i:i + 1].cuda(), scale=scale, out=zi,
                                   **({k: v[i:i + 1] for k, v in extra.items()}))
        near(one, want[i:i + 1], tol[i:i + 1])


def far_distill_grad(z, ids, u, scale, tail, weight):
    """The gradient with the share outside the ids taken from the largest logit there: nothing is lost at any size."""
    lp, lse = ref.log_softmax(z, scale)
    p = lp.exp()
    q, rest = ref.teacher(ids, u, 1.0, tail)
    want, terms = torch.zeros_like(p), torch.zeros_like(p)
    for i in range(z.shape[0]):
        if lse[i] == NEG:
            continue
        qv, inside = torch.zeros(z.shape[1], dtype=torch.float64), torch.zeros(z.shape[1], dtype=torch.bool)
        for j in range(ids.shape[1]):
            if ids[i, j] >= 0:
                qv[ids[i, j]] += q[i, j]
                inside[ids[i, j]] = True
        d, mag = p[i] * q[i].sum() - qv, p[i] * (1 + q[i].sum()) + qv
        if tail and float(rest[i]) > 0:
            y = torch.where(inside, torch.full((), NEG, dtype=torch.float64), z[i].double() * scale)
            share = torch.zeros_like(y)
            if float(y.max()) > NEG:
                e = (y - y.max()).exp()
                share = e / e.sum()
            d = d + rest[i] * (p[i] - share)
            mag = mag + share * (rest[i] + 1)
        want[i], terms[i] = weight[i].double() * scale * d, mag
    rel = sum_tol(z.shape[1]) + 8 * EPS * (clip(lp, 200.0) + clip(lse, SAVED)[:, None] + clip(u.double(), 200.0).amax(1)[:, None] + 4) + 2 ** -20
    return want, weight.double().abs()[:, None] * scale * rel * terms * 4 + HALF[z.dtype] * want.abs() + TINY[z.dtype] + 1e-30


@pytest.mark.parametrize("V,type_", FAR_SIZES)
@pytest.mark.parametrize("tail", [False, True])
def test_distillation_gradient_where_lse_is_large(V, type_, tail):
    g = gen(V)
    z = far_rows(V, type_, g)
    N, K = z.shape[0], 6
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(N)])
    ids[8] = torch.arange(K)                     # all live columns are named: the student's mass outside is exp(-1e9)
    ids[5, K - 1] = ids[5, 0]
    u = torch.log_softmax(torch.randn((N, K), generator=g), 1) - 0.3
    w = torch.rand(N, generator=g) + 0.5
    want, tol = far_distill_grad(z, ids, u, 1.0, tail, w)
    zd, _ = view(z, 3, 1)
    got = lm().distill(zd, ids.cuda(), u.cuda(), tail=tail, weight=w.cuda())
    near(got.grad, want, tol)
    back = lm().distill_grad(zd, ids.cuda(), u.cuda(), got.lse, w.cuda(), tail=tail, log_tail=got.log_tail)
    near(back, want, tol)
    near(lm().distill_grad(zd, ids.cuda(), u.cuda(), got.lse, w.cuda(), tail=tail, log_tail=got.log_tail, out=zd), want, tol)
    for i in (0, 8):
        zi = z[i:i + 1].cuda()
        one = lm().distill_grad(zi, ids[i:i + 1].cuda(), u[i:i + 1].cuda(), got.lse[i:i + 1], w[i:i + 1].cuda(), tail=tail,
                                log_tail=got.log_tail[i:i + 1] if tail else None, out=zi)
        near(one, want[i:i + 1], tol[i:i + 1])


@pytest.mark.parametrize("V", [12, 128])
@pytest.mark.parametrize("type_", [F32, BF16])
def test_backward_call_where_every_column_is_named(V, type_):
    """No column is left outside the ids: log p_T is -inf, and the rest of the teacher's mass pulls at none."""
    N = 3
    z = torch.randn((N, V), generator=gen(V)).to(type_)
    z[2, V // 2:] = NEG
    ids = torch.stack([torch.randperm(V, generator=gen(i)) for i in range(N)])
    u, w = torch.log_softmax(torch.randn((N, V), generator=gen(4)), 1) + math.log(0.9), torch.ones(N)
    got = lm().distill(z.cuda(), ids.cuda(), u.cuda(), tail=True, weight=1.0)
    assert bool((got.log_tail == NEG).all()) and bool((got.loss == INF).all())
    want, tol = far_distill_grad(z, ids, u, 1.0, True, w)
    near(got.grad, want, tol)
    near(lm().distill_grad(z.cuda(), ids.cuda(), u.cuda(), got.lse, 1.0, tail=True, log_tail=got.log_tail), want, tol)


# ------------------------------------------------------------------ statistics on both sides of the range of one multiply-add
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("rising", [False, True])
@pytest.mark.parametrize("N,V", [(2, 5000), (3, 40009), (1, 130001), (900, 3000)])
def test_rows_on_both_sides_of_the_exponents_range(N, V, rising, sign):
    """Logits around 65536 ln 2: some blocks', threads' or batches' exponents are relative to a rounded product, others' to
    the difference."""
    z = torch.linspace(-1.0, 1.0, V).expand(N, V) + 0.05 * torch.rand((N, V), generator=gen(V))
    z = (45426.0 + (z if rising else -z)) * sign
    tok = torch.randint(0, V, (N,), generator=gen(1))
    logp, lse, ent, ids, tl = ref.token_logp(z, tok, 1.0, 4)
    r = lm().token_logp(z.cuda(), tok.cuda(), top=4)
    s = sum_tol(V) + 8 * EPS * math.log(V)
    near(r.logp, logp, s)
    near(r.entropy, ent, s * (4 + 2 * math.log(V)))
    near(r.top_logp, tl, s)
    d = lm().distill(z.cuda(), tok[:, None].cuda(), torch.zeros(N, 1).cuda(), weight=1.0)
    near(d.loss, -logp, s + 2 ** -19)


# ------------------------------------------------------------------ gradients beside the logits
def test_gradients_in_other_columns_of_the_logits_buffer():
    """Logits and gradient in two halves of the same rows share no element."""
    N, V, K = 5, 203, 3
    z = torch.randn((N, V), generator=gen(1))
    buf = torch.full((N, 2 * V + 2), 77.0, device="cuda")
    for at, out_at in ((0, V + 1), (V + 2, 1)):
        zd, out = buf[:, at:at + V], buf[:, out_at:out_at + V]
        zd.copy_(z)
        tok = torch.arange(N)
        r = lm().token_logp(zd, tok.cuda())
        lm().token_logp_grad(zd, tok.cuda(), r.lse, 1.0, out=out)
        _near_logp_grad(out, z, tok, 1.0, torch.ones(N), torch.zeros(N))
        assert torch.equal(zd.cpu(), z)
        ids, u = torch.randint(0, V, (N, K), generator=gen(2)), torch.randn((N, K), generator=gen(3))
        got = lm().distill(zd, ids.cuda(), u.cuda(), weight=1.0, out=out)
        _near_distill(got, z, ids, u, 1.0, 1.0, False, torch.ones(N))
        assert torch.equal(zd.cpu(), z)
    from paper_1906_02367_b200 import binding as B
    for at in (1, V - 1, V + 3):                 # one element at least is shared, within a row or with the next
        with pytest.raises(B.QsError):
            lm().token_logp_grad(buf[:N - 1, :V], tok[:N - 1].cuda(), r.lse[:N - 1], 1.0, out=torch.as_strided(buf, (N - 1, V), (2 * V + 2, 1), at))


# ------------------------------------------------------------------ calls beside other calls
def test_calls_from_several_threads():
    """Threads distil at vocabularies whose shares of shared memory differ: no call may see another's size."""
    from paper_1906_02367_b200 import binding as B
    L, N, K, calls, codes, work = B.lib(), 890, 4, 2000, [], []
    for V in (18000, 40000, 90000, 33000):
        z = torch.randn((N, V), generator=gen(V)).to(BF16).cuda()
        ids, u = torch.randint(0, V, (N, K), generator=gen(1)).cuda(), torch.zeros(N, K).cuda()
        loss, grad = torch.empty(N, device="cuda"), torch.empty_like(z)
        work.append((z, ids, u, loss, grad, lm().distill(z, ids, u, weight=1.0), torch.cuda.Stream()))
    torch.cuda.synchronize()
    start = threading.Barrier(len(work))

    def run(z, ids, u, loss, grad, _, stream):
        args = (N, z.shape[1], K, z.data_ptr(), B.QS_BF16, z.shape[1], ids.data_ptr(), B.QS_I64, u.data_ptr(), B.QS_F32, 1.0, 1.0, 0, loss.data_ptr(),
                None, None, None, 1.0, grad.data_ptr(), z.shape[1], None, stream.cuda_stream)
        start.wait()
        codes.extend(L.qs_distill(*args) for _ in range(calls))

    threads = [threading.Thread(target=run, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert len(codes) == calls * len(work) and not any(codes)
    for _, _, _, loss, grad, want, _ in work:
        assert torch.equal(loss, want.loss) and torch.equal(grad, want.grad)


def child(code, **env):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env={**os.environ, **env}, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    return r.stdout


def test_an_error_that_another_call_left_is_not_reported():
    """A call that fails on the host (waiting for a stream that is being captured) leaves its error with the runtime; the
    operators' calls after it do their work and say so."""
    child("""
import torch
from paper_1906_02367_b200 import binding as B, lm
side = torch.cuda.Stream()
ctx = B.Context(1, 64, 4, 1, stream=side)
table, tok = torch.randn(10, 8, device="cuda"), torch.arange(5, device="cuda")
z = torch.randn(5, 10, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
try:
    with torch.cuda.stream(side):
        graph.capture_begin()
        code = ctx.sync_status()
        graph.capture_end()
except RuntimeError:
    pass
assert code == B.QS_CUDA
assert torch.equal(lm.embed(tok, table), table[:5])
grad = lm.embed_grad(tok, torch.ones(5, 8, device="cuda"), 10)
assert grad.sum().item() == 40.0
assert lm.embed_grad(tok[:0], torch.ones(0, 8, device="cuda"), 10).sum().item() == 0.0
assert torch.isfinite(lm.token_logp(z, tok).logp).all()
""")


def test_a_wait_that_runs_out_leaves_nan():
    """With no time to wait at all, every row that needs a copy or another block's sums is NaN, with a status or without; the
    memory of the copies is not given up before they have come."""
    child("""
import torch
from paper_1906_02367_b200 import binding as B, lm
for N, V, type_ in ((3, 1000, torch.float32), (2, 50003, torch.bfloat16), (900, 40000, torch.bfloat16), (2, 600000, torch.float32)):
    z = torch.randn(N, V, device="cuda").to(type_)
    ids, u = torch.randint(0, V, (N, 4), device="cuda"), torch.full((N, 4), -2.0, device="cuda")
    ids[1] = torch.tensor([-1, -1, -1, V])                    # an id past the end does not hide it
    for tail in (False, True):
        for weight in (None, 1.0):
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            lm.distill(z, ids, u, tail=tail, weight=weight)
            d = lm.distill(z, ids, u, tail=tail, weight=weight, status=status)
            assert int(status) == B.QS_TIMEOUT
            for t in (d.loss, d.lse, d.log_tail, d.grad):
                assert t is None or bool(torch.isnan(t).all())
    r = lm.token_logp(z, ids[:, 0].contiguous(), top=2)       # the calls that wait for nothing go on
    assert bool(torch.isfinite(r.lse).all())
""", QSPARSE_WAIT_LIMIT_NS="0")
    child("""
import torch
from paper_1906_02367_b200 import lm
z = torch.randn(2, 50003, device="cuda")
d = lm.distill(z, torch.zeros(2, 1, dtype=torch.int64, device="cuda"), torch.zeros(2, 1, device="cuda"), tail=True, weight=1.0)
assert bool(torch.isfinite(d.loss).all()) and bool(torch.isfinite(d.grad).all())
""", QSPARSE_WAIT_LIMIT_NS="1000000000")


# ------------------------------------------------------------------ long lists of tokens
def sums_by_token(tok, go, V, scale):
    out = torch.zeros((V + 1, go.shape[1]), dtype=torch.float64)
    mag, cnt = torch.zeros_like(out), torch.zeros(V + 1, dtype=torch.int64)
    at = torch.where(tok < 0, V, tok).long()
    out.index_add_(0, at, scale * go.double())
    mag.index_add_(0, at, abs(scale) * go.double().abs())
    cnt.index_add_(0, at, torch.ones_like(at))
    return out[:V], mag[:V], cnt[:V]


LONG = [(1, 20000, 700, 2048, "zipf"), (1, 20000, 700, 2048, "runs"), (1, 20001, 90, 2049, "uniform"), (2, 40000, 50, 1030, "runs"), (1, 65537, 1000, 3, "uniform"),
        (1, 140001, 30000, 5, "zipf"), (1, 140001, 300, 4, "runs"), (1, 600011, 70001, 1, "uniform"), (8, 40000, 5000, 8, "zipf"), (3, 131073, 513, 2, "runs")]


@pytest.mark.parametrize("R,N,V,D,kind", LONG)
@pytest.mark.parametrize("type_", [F32, BF16])
def test_embed_gradient_of_long_lists(R, N, V, D, kind, type_):
    """Chunks of 64 places, tiles of several places per thread, more tiles than blocks fit: sizes that short lists do not
    reach."""
    g = gen(N + D)
    if kind == "runs":                           # of lengths that end at every place of a chunk
        tok = torch.stack([(torch.cumsum((torch.rand(N, generator=g) < 0.03).long(), 0) * 7) % V for _ in range(R)])
    elif kind == "zipf":
        tok = torch.clamp((torch.rand((R, N), generator=g) * math.log(V + 1)).exp().long() - 1, 0, V - 1)
    else:
        tok = torch.randint(-1, V, (R, N), generator=g)
    go = torch.randn((R, N, D), generator=g).to(type_)
    td, gd = tok.cuda(), go.cuda()
    got = lm().embed_grad(td, gd, V, scale=0.75)
    assert torch.equal(got, lm().embed_grad(td, gd, V, scale=0.75))
    base = torch.randn((R, V, D), generator=g)
    acc = lm().embed_grad(td, gd, V, scale=0.75, accumulate=True, out=base.cuda())
    for r in range(R):
        want, mag, cnt = sums_by_token(tok[r], go[r], V, 0.75)
        tol = (cnt[:, None] + 2) * EPS * mag
        near(got[r], want, tol)
        near(acc[r], want + base[r].double(), tol + 2 * EPS * (mag + base[r].abs()))
        assert torch.equal(acc[r].cpu()[cnt == 0], base[r][cnt == 0])


def test_embed_gradient_of_seventeen_million_tokens():
    N, V = 17_000_001, 1000
    tok = torch.randint(0, V, (N,), generator=gen(1), dtype=torch.int32)
    go = torch.randn((N, 1), generator=gen(2))
    got = lm().embed_grad(tok.cuda(), go.cuda(), V)
    want, mag, cnt = sums_by_token(tok, go, V, 1.0)
    near(got, want, (cnt[:, None] + 2) * EPS * mag)


def test_embed_gradient_with_a_workspace_of_the_callers():
    N, V, D = 3000, 500, 40
    tok, go = torch.randint(0, V, (N,), generator=gen(1)), torch.randn((N, D), generator=gen(2))
    want = lm().embed_grad(tok.cuda(), go.cuda(), V)
    work = lm().embed_grad_work(1, N, V, D)
    work.fill_(255)
    more = torch.full((work.numel() // 4 + 100,), -1, dtype=torch.int32, device="cuda")
    for w in (work, work, more):
        out = torch.full((V, D), 7.0, device="cuda")
        assert lm().embed_grad(tok.cuda(), go.cuda(), V, out=out, work=w) is out and torch.equal(out, want)
    assert bool((more[work.numel() // 4:] == -1).all())          # nothing past what is asked for


def test_embed_gradient_of_several_tiles_in_a_graph():
    N, V, D = 5000, 800, 24
    tok, go = torch.randint(0, V, (N,), generator=gen(1)).cuda(), torch.randn((N, D), generator=gen(2)).cuda()
    out = torch.empty((V, D), device="cuda")
    want = lm().embed_grad(tok, go, V)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lm().embed_grad(tok, go, V, out=out)
    for _ in range(3):
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    tok.fill_(3)                                 # other tokens, the same launches
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, lm().embed_grad(tok, go, V)) and float(out[4:].abs().sum()) == 0.0


# ------------------------------------------------------------------ long rows by one block
@pytest.mark.parametrize("N,V,type_,top", [(900, 256001, F32, 64), (900, 256000, F32, 8), (1100, 256003, BF16, 128), (900, 150001, F16, 20), (890, 140000, BF16, 1)])
def test_alternatives_of_long_rows_by_one_block(N, V, type_, top):
    """Rows of more batches than there are stretches, so that a stretch is several batches."""
    z = torch.empty((N, V), device="cuda").normal_(0.0, 3.0, generator=torch.Generator(device="cuda").manual_seed(V))
    z[1] = torch.round(z[1])                     # ties everywhere
    z[2] = torch.linspace(-8, 8, V, device="cuda")
    z[3] = torch.linspace(8, -8, V, device="cuda")
    z[4, :] = torch.finfo(type_).min
    z[4, V - 5:] = 1.0
    z[5, V // 2: V // 2 + 300] += 40.0           # the largest side by side
    z[6] = 0.5
    z = z.to(type_)
    tok = torch.randint(0, V, (N,), generator=gen(3))
    r = lm().token_logp(z, tok.cuda(), top=top)
    rows = torch.tensor([0, 1, 2, 3, 4, 5, 6, N // 2, N - 1])
    zr = z[rows.cuda()].cpu()
    logp, lse, ent, ids, tl = ref.token_logp(zr, tok[rows], 1.0, top)
    s = sum_tol(V)
    pick = lambda t: t[rows.cuda()]  # noqa: E731
    assert torch.equal(pick(r.top_ids).cpu(), ids)
    near(pick(r.top_logp), tl, s + 8 * EPS * clip(tl, INF))
    near(pick(r.logp), logp, s + 8 * EPS * clip(logp, INF))
    near(pick(r.lse), lse, s + 4 * EPS * lse.abs())
    near(pick(r.entropy), ent, s * (4 + 2 * math.log(V + 1)))


# ------------------------------------------------------------------ NaN and infinities
@pytest.mark.parametrize("V", [5, 1000, 40009, 140001])
@pytest.mark.parametrize("type_", [F32, BF16, F16])
@pytest.mark.parametrize("tail", [False, True])
def test_nan_and_infinity_in_the_logits(V, type_, tail):
    """A NaN or +inf anywhere in a row makes its results NaN and leaves the other rows' alone."""
    N, K = 5, 3
    z = (torch.randn((N, V), generator=gen(V)) * 2).to(type_)
    z[1, V // 2] = NAN
    z[2, V - 1] = INF
    z[3] = NEG
    z[3, 0] = NAN
    bad = torch.tensor([False, True, True, True, False])
    ids, u = torch.stack([torch.randperm(V, generator=gen(i))[:K] for i in range(N)]), torch.log_softmax(torch.randn((N, K), generator=gen(2)), 1) - 0.2
    tok, w = torch.randint(0, V, (N,), generator=gen(3)), torch.ones(N)
    r = lm().token_logp(z.cuda(), tok.cuda())
    assert torch.equal(torch.isnan(r.lse.cpu()), bad)
    for extra in ({}, dict(entropy=r.entropy, grad_entropy=w.cuda())):
        got = lm().token_logp_grad(z.cuda(), tok.cuda(), r.lse, 1.0, **extra).cpu()
        assert torch.equal(torch.isnan(got).all(1), bad) and torch.equal(torch.isnan(got).any(1), bad)
        _near_logp_grad(got[~bad], z[~bad], tok[~bad], 1.0, w[:2], w[:2] if extra else 0 * w[:2])
    d = lm().distill(z.cuda(), ids.cuda(), u.cuda(), tail=tail, weight=1.0)
    back = lm().distill_grad(z.cuda(), ids.cuda(), u.cuda(), d.lse, 1.0, tail=tail, log_tail=d.log_tail).cpu()
    for t in (d.loss.cpu()[:, None], d.lse.cpu()[:, None], d.grad.cpu(), back):
        assert torch.equal(torch.isnan(t).all(1), bad) and torch.equal(torch.isnan(t).any(1), bad)
    keep = [i for i in range(N) if not bad[i]]
    rows = type(d)(d.loss[keep], d.lse[keep], d.log_tail[keep] if tail else None, d.grad[keep])
    _near_distill(rows, z[keep], ids[keep], u[keep], 1.0, 1.0, tail, w[:2])


@pytest.mark.parametrize("tail", [False, True])
def test_nan_in_the_teachers_values(tail):
    N, V, K = 3, 777, 5
    z, ids = torch.randn((N, V), generator=gen(1)), torch.stack([torch.randperm(V, generator=gen(i))[:K] for i in range(N)])
    u = torch.log_softmax(torch.randn((N, K), generator=gen(2)), 1) - 0.2
    u[1, 2] = NAN
    got = lm().distill(z.cuda(), ids.cuda(), u.cuda(), tail=tail, weight=1.0)
    back = lm().distill_grad(z.cuda(), ids.cuda(), u.cuda(), got.lse, 1.0, tail=tail, log_tail=got.log_tail).cpu()
    for t in (got.loss.cpu()[:, None], got.grad.cpu(), back):
        assert torch.isnan(t).all(1).tolist() == [False, True, False] and torch.isnan(t).any(1).tolist() == [False, True, False]
    ids[1, 2] = -1                               # a place that names nothing: its value is not looked at
    got = lm().distill(z.cuda(), ids.cuda(), u.cuda(), tail=tail, weight=1.0)
    u[1, 2] = 0.0
    _near_distill(got, z, ids, u, 1.0, 1.0, tail, torch.ones(N))


# ------------------------------------------------------------------ types and results
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V,K,type_", [(1000, 8, F32), (33001, 64, BF16)])
def test_a_teacher_in_fp16(V, K, type_, tail):
    N = 4
    z = (torch.randn((N, V), generator=gen(1)) * 2).to(type_)
    ids = torch.stack([torch.randperm(V, generator=gen(i))[:K] for i in range(N)])
    u = (torch.log_softmax(torch.randn((N, K), generator=gen(2)), 1) - 0.2).to(F16)
    got = lm().distill(z.cuda(), ids.cuda(), u.cuda(), tail=tail, weight=1.0)
    _near_distill(got, z, ids, u, 1.0, 1.0, tail, torch.ones(N))
    back = lm().distill_grad(z.cuda(), ids.cuda(), u.cuda(), got.lse, 1.0, tail=tail, log_tail=got.log_tail)
    near(back, got.grad.double().cpu(), 1e-5 + 2 * HALF[type_] * got.grad.double().cpu().abs())


def test_results_that_are_not_asked_for():
    """NULL for any of logp, lse, entropy, loss, log_tail in the C calls: the others are the same."""
    from paper_1906_02367_b200 import binding as B
    L, N, V, K = B.lib(), 4, 3001, 3
    st = torch.cuda.current_stream().cuda_stream
    z, tok = torch.randn((N, V), generator=gen(1)).cuda(), torch.arange(N).cuda()
    full = lm().token_logp(z, tok, top=K)
    for skip in range(3):
        for top in (0, K):
            out = [torch.full((N,), 7.0, device="cuda") for _ in range(3)]
            ids, tl = torch.full((N, K), 7, dtype=torch.int64, device="cuda"), torch.full((N, K), 7.0, device="cuda")
            ptr = [None if i == skip else t.data_ptr() for i, t in enumerate(out)]
            assert L.qs_token_logp(N, V, z.data_ptr(), B.QS_F32, V, tok.data_ptr() if skip else None, B.QS_I64, 1.0, top, *ptr,
                                   ids.data_ptr() if top else None, tl.data_ptr() if top else None, None, st) == 0
            for i, t in enumerate(out):
                assert bool((t == 7.0).all()) if i == skip else torch.equal(t, full[i])
            assert torch.equal(ids, full.top_ids) if top else bool((ids == 7).all())
    ids, u = torch.randint(0, V, (N, K), generator=gen(2)).cuda(), torch.full((N, K), -2.0).cuda()
    want = lm().distill(z, ids, u, tail=True, weight=0.5)
    for skip in range(3):
        out, grad = [torch.full((N,), 7.0, device="cuda") for _ in range(3)], torch.empty_like(z)
        ptr = [None if i == skip else t.data_ptr() for i, t in enumerate(out)]
        assert L.qs_distill(N, V, K, z.data_ptr(), B.QS_F32, V, ids.data_ptr(), B.QS_I64, u.data_ptr(), B.QS_F32, 1.0, 1.0, 1, *ptr, None, 0.5,
                            grad.data_ptr(), V, None, st) == 0
        for i, t in enumerate(out):
            assert bool((t == 7.0).all()) if i == skip else torch.equal(t, want[i])
        assert torch.equal(grad, want.grad)
