"""Roundings of the residual block's operators, held to what include/qsparse.h says of them: 8 bits to the last bit, activations
in fp32 over their whole range, fp32 operands in parts."""
import pytest
import torch

import layers_reference as ref
from test_gpu_layers import BF16, E, F16, F32, near, rand

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.fixture
def L():
    from paper_1906_02367_b200 import layers
    return layers


# ------------------------------------------------------------------ 8 bits
def check_bits(q, scale, y):
    """s = max(max |y| / 448, 2^-126), q = y / s rounded: each one operation in fp32, on the host's own divisions."""
    q, scale, y = q.float().cpu(), scale.cpu(), y.cpu()
    s = (y.abs().amax(-1) / torch.tensor(448.0)).clamp_min(2.0 ** -126)
    assert torch.equal(scale, s)
    want = (y / s[..., None]).clamp(-448.0, 448.0).to(E4M3).float()
    assert torch.equal(q, want), (int((q != want).sum()), q.numel())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,width", [(5, 64), (700, 257), (2000, 1024), (512, 4096), (300, 4100), (40, 20000)])
def test_norm_in_8_bits_to_the_last_bit(L, dtype, rows, width):
    x, res, w = rand((rows, width), dtype, 1, 3.0), rand((rows, width), dtype, 2), rand((width,), dtype, 3, 0.2, 1.0)
    r = L.rms_norm(x, w, res, quantize=True)
    check_bits(r.out, r.scale, r.hidden.cpu().float() * r.rstd.cpu()[:, None] * w.cpu().float())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_quantized_rows_to_the_last_bit(L, dtype):
    for rows, width in ((3, 16), (500, 1001), (300, 4096), (20, 30000)):
        x = rand((rows, width), dtype, 4, 0.02)
        q = L.quantize(x)
        check_bits(q.values, q.scale, x.float())
    # every value that 16 bits hold, by rows whose largest is any of them: quotients next to all middles
    x = torch.arange(1, 0x7c00, device="cuda", dtype=torch.int32).to(torch.int16).view(F16)
    x = x[: 31 * 1000].view(31, 1000).t().contiguous().to(dtype)
    q = L.quantize(x)
    check_bits(q.values, q.scale, x.float())
    # and scales from the smallest to the largest
    x = rand((256, 512), F32, 5) * torch.pow(2.0, torch.arange(-140, 116, device="cuda").float())[:, None]
    q = L.quantize(x)
    check_bits(q.values, q.scale, x)


# ------------------------------------------------------------------ activations
def by_bias(L, z, M, K, activation, dtype, out):
    """act(z) through a product whose sums are zero: z is the bias, the same for every row."""
    x, w = torch.zeros((M, K), device="cuda", dtype=dtype), rand((z.numel(), K), dtype, 2)
    return L.linear(x, w, z, activation=activation, dtype=out, save=True)


# few rows, small products, one tile in a row and several, 64 and 256 columns, in splits (with K), off the boundary
FORMS = [(1, 1024, 64), (20, 1024, 64), (40, 40, 16), (300, 1024, 64), (130, 64, 4096), (3000, 1280, 64), (140, 1023, 100)]


@pytest.mark.parametrize("M,N,K", FORMS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gelu_in_32_bits_over_its_range(L, M, N, K, dtype):
    """Relative to the value, where the normal distribution's tail makes it small too: z^2, log2(e) / 2 and their product, each
    rounded, are 0.6 z^2 2^-23 in the exponential, which is good to 2 steps of 2^-23; the reciprocal, the polynomial, the
    products of the two and of z to 4."""
    z = torch.linspace(-12.5, 6.0, N, device="cuda")
    r = by_bias(L, z, M, K, "gelu", dtype, F32)
    assert torch.equal(r.pre, z.expand(M, N))
    y = ref.activate(z.double(), "gelu").expand(M, N)
    near(r.out, y, (6 + 0.6 * z.double() ** 2) * E * y.abs(), F32)


@pytest.mark.parametrize("M,N,K", FORMS)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_gelu_in_16_bits_over_its_range(L, M, N, K, dtype):
    """Half a step of the type and what fp32 leaves: z^2 rounded in an exponent, about ten more roundings."""
    z = torch.linspace(-12.5, 6.0, N, device="cuda")
    r = by_bias(L, z, M, K, "gelu", dtype, dtype)
    y = ref.activate(z.double(), "gelu")
    near(r.out, y.expand(M, N), ((10 + 2 * z.double() ** 2) * E * y.abs()).expand(M, N), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_slope_of_gelu_over_its_range(L, dtype):
    """slope = Phi + z phi: in fp32 6 + 0.6 z^2 steps of either, in 16 bits about ten and more in the exponent."""
    z = torch.linspace(-12.5, 6.0, 4096, device="cuda").to(dtype).repeat(9, 1)
    z64 = z.double()
    phi = torch.exp(-z64 * z64 / 2) * 0.3989422804014327
    cdf = 0.5 * torch.special.erfc(-z64 * 0.7071067811865476)
    steps = 6 + 0.6 * z64 ** 2 if dtype == F32 else 10 + 2 * z64 ** 2
    got = L.activation_grad(torch.ones_like(z), z, "gelu", bias=True)
    slack = steps * E * (cdf + (z64 * phi).abs())
    near(got[0], cdf + z64 * phi, slack, dtype)
    near(got[1], 9 * (cdf + z64 * phi)[0], 9 * (slack[0] + 9 * E * (cdf + z64 * phi).abs()[0]), F32)


# ------------------------------------------------------------------ fp32 operands in parts
@pytest.mark.parametrize("M,N,K", [(16, 2048, 16), (1024, 1024, 16), (600, 1029, 32)])
def test_parts_of_fp32_leave_little_out(L, M, N, K):
    """Operands just below 1 + 2^-7, whose bits behind the first eight are all ones: cut off instead of rounded, the products
    of their last parts are 2^-21 of the whole.  Rounded parts leave out 2^-25 at most; the matrix unit's sums of 16 terms cut
    off 2^-23 twice at most (in the last two of six products, the others are below 2^-8)."""
    one = 1 + 2.0 ** -7 - 2.0 ** -23
    x, w = rand((M, K), F32, 1).mul_(2.0 ** -16).abs_().neg_().add_(one), torch.full((N, K), one, device="cuda")
    z, _ = ref.product(x, w)
    off = ((L.linear(x, w).out.double() - z) / z).abs().max()
    assert float(off) < (K / 16) * 2 * E + 2.0 ** -25, float(off)


def test_parts_of_the_largest_numbers(L):
    """Numbers that round past the largest bf16 are cut off; NaN and infinities make their rows NaN, and no others."""
    x, w = torch.zeros((600, 64), device="cuda"), torch.zeros((1100, 64), device="cuda")
    x[:, 3], w[:, 3] = torch.finfo(F32).max, 0.5
    x[5, 3], x[6, 3], x[7, 3] = -torch.finfo(F32).max, float("nan"), float("inf")
    y = L.linear(x, w).out
    want = torch.full((600, 1100), torch.finfo(F32).max / 2, device="cuda")
    want[5] *= -1
    keep = [i for i in range(600) if i not in (6, 7)]
    near(y[keep], want[keep].double(), 4 * E * want[keep].double().abs(), F32)
    assert bool(torch.isnan(y[6:8]).all())
    # up to 32 rows by the small instruction, parts on the way
    assert bool(torch.isnan(L.linear(x[:16], w).out[6:8]).all()) and torch.equal(L.linear(x[:16], w).out[:6], y[:6])


# ------------------------------------------------------------------ sums over rows
@pytest.mark.parametrize("R,M,N", [(1, 509, 257), (1, 5000, 1024), (2, 3000, 333), (1, 64, 4096)])
def test_sums_over_rows_round_like_trees(L, R, M, N):
    """A rounding is 0.41 2^-24 of its sum in the mean of squares.  In a tree over rows of mixed signs every level leaves as much: 13
    levels, or stretches of as many rows, and two products' roundings come to 1.6 2^-24 of the result; a chain of 32 partial sums
    alone is worth 16 levels."""
    h, g, w = rand((R, M, N), F32, 1, 2.0), rand((R, M, N), F32, 2, 0.01), rand((R, N), F32, 3, 0.1, 1.0)
    rstd = ref.rms_norm(h, w, None, 1e-6)[2].float()
    _, dw, _ = ref.rms_norm_grad(g, h, rstd, w, None)
    off = L.rms_norm_grad(g, h, rstd, w).weight.double() - dw
    assert float(off.norm() / dw.norm()) < 2 * 2.0 ** -24, float(off.norm() / dw.norm())
    db = L.activation_grad(g, bias=True, workers=True)[1].double() - g.double().sum(1)
    assert float(db.norm() / g.double().sum(1).norm()) < 2 * 2.0 ** -24
