"""Long sums of the products: what the matrix unit cuts off at every addition does not add up, whatever the result's type and
wherever the sums may lie."""
import pytest
import torch

import layers_reference as ref
from test_gpu_layers import BF16, E, F16, F32, U, near, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.fixture
def L():
    from paper_1906_02367_b200 import layers
    return layers


@pytest.mark.parametrize("activation", [None, "gelu"])
@pytest.mark.parametrize("R,M,N,K", [(1, 4000, 1280, 6000), (1, 4000, 1277, 2500), (2, 700, 264, 9000), (1, 140, 64, 8192), (1, 20, 256, 4096), (3, 1500, 1030, 1100)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_residual_in_the_results_place(L, activation, R, M, N, K, dtype):
    """The call with the residual in the result's place gives what the call into another tensor gives, to the last bit, in
    sums of one sign too."""
    x, w, b, res = rand((R, M, K), dtype, 1).abs(), rand((R, N, K), dtype, 2, K ** -0.5).abs(), rand((R, N), F32, 3), rand((R, M, N), F32, 4)
    want = L.linear(x, w, b, activation=activation, residual=res, dtype=F32, save=True)
    place = res.clone()
    assert torch.equal(L.linear(x, w, b, activation=activation, residual=place, out=place).out, want.out)
    place = res.clone()
    got = L.linear(x, w, b, activation=activation, residual=place, out=place, save=True)
    assert torch.equal(got.out, want.out) and torch.equal(got.pre, want.pre) and got.out is place
    z, _ = ref.product(x, w)
    off = ((want.pre.double() - b.double()[:, None] - z) / z).abs()
    assert float(off.max()) < 64 * E + (K / 1024 + 4) * E + 2.0 ** -21, float(off.max())


def test_residual_in_the_results_place_in_a_graph_and_a_callers_workspace(L):
    from paper_1906_02367_b200.binding import QS_BF16, QS_CAPACITY, QsError, lib
    M, N, K = 4000, 1280, 3000
    x, w, res = rand((M, K), BF16, 1), rand((N, K), BF16, 2, K ** -0.5), rand((M, N), F32, 3)
    want = L.linear(x, w, activation="silu", residual=res, dtype=F32).out
    n = lib().qs_linear_bytes(1, M, N, K, x.data_ptr(), QS_BF16, K, w.data_ptr(), QS_BF16, 0, K)
    guard = torch.full((n + 512,), 7, dtype=torch.uint8, device="cuda")
    place = res.clone()
    assert torch.equal(L.linear(x, w, activation="silu", residual=place, out=place, work=guard[256:256 + n]).out, want)
    assert bool((guard[:256] == 7).all()) and bool((guard[256 + n:] == 7).all())
    place = res.clone()
    with pytest.raises(QsError) as e:
        L.linear(x, w, activation="silu", residual=place, out=place, work=guard[256:512])
    assert e.value.code == QS_CAPACITY and torch.equal(place, res)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.linear(x, w, activation="silu", residual=place, out=place)
    for _ in range(2):
        place.copy_(res)
        g.replay()
        assert torch.equal(place, want)


# The matrix unit cuts off less than 2^-23 of the sum so far for every 8 elements of 16 bits, or 16 of 8.  Results in bf16 come from sums
# of 16384 elements at most: 2048 such steps, of sums that grow evenly 1024 2^-23; in fp16 from half as many.  Over
# millions of results the roundings to 16 bits cancel in the mean: each is half a step at most, of which a thousandth is left
CUT = {BF16: 1024 * E, F16: 512 * E}


def check_long(got, a, b, dtype):
    z, _ = ref.product(a, b)
    off = (got.double() - z) / z
    assert abs(float(off.mean())) < CUT[dtype] + 2 * E + U[dtype] / 1000, float(off.mean())
    near(got, z, (CUT[dtype] + 2 * E) * z, dtype)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_long_sums_into_16_bits(L, dtype):
    """More tiles than blocks, so that no sum is split up for its own sake: the result, and both gradients."""
    K, N = 1 << 18, 2560
    x, w = rand((N, K), dtype, 1).abs(), rand((N, K), dtype, 2, 1.0 / K).abs()
    check_long(L.linear(x, w).out, x, w, dtype)
    check_long(L.linear(x, w.float(), rand((N,), F32, 3) * 0).out, x, w.float().to(dtype), dtype)
    g = x.t().contiguous()                            # (K rows of N)
    y = w.t().contiguous()
    one = torch.zeros((N, N), device="cuda", dtype=dtype)
    check_long(L.linear_grad(g, y, one, need_x=False, dtype=dtype).weight, x, w, dtype)
    del g
    check_long(L.linear_grad(x, one, y, need_weight=False).x, x, w, dtype)


def test_long_sums_of_8_bits(L):
    K, N = 1 << 18, 2560
    x, w = L.quantize(rand((N, K), BF16, 1).abs()), L.quantize(rand((N, K), BF16, 2).abs())
    unit = torch.full((N,), 2.0 ** -20, device="cuda")
    got = L.linear(x.values, w.values, x_scale=unit, weight_scale=unit * 0 + 2.0 ** -12, dtype=F16).out
    check_long(got, x.values.float() * 2.0 ** -20, w.values.float() * 2.0 ** -12, F16)
    bias, res = rand((N,), F32, 3), rand((N, N), F16, 4)
    full = L.linear(x.values, w.values, bias, activation="relu", residual=res, x_scale=unit, weight_scale=unit * 0 + 2.0 ** -12, dtype=F16, save=True)
    z, _ = ref.product(x.values.float() * 2.0 ** -20, w.values.float() * 2.0 ** -12)
    near(full.pre, z + bias.double(), (CUT[F16] + 4 * E) * (z + bias.double().abs()), F16)
    near(full.out, (z + bias.double()).clamp_min(0) + res.double(), (CUT[F16] + 6 * E) * (z + bias.double().abs() + res.double().abs()), F16)
    place = res.clone()
    assert torch.equal(L.linear(x.values, w.values, bias, activation="relu", residual=place, x_scale=unit, weight_scale=unit * 0 + 2.0 ** -12, out=place).out, full.out)
