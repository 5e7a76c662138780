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
