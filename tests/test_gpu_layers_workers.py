"""Weights of a worker each in the forms that other tests have for one: 8 bits with scales of every worker's rows, and the most workers
that there may be."""
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


def apart(t, pad):
    """The same values, every worker's `pad` elements further on."""
    R = t.shape[0]
    buf = torch.zeros((R, t[0].numel() + pad), device="cuda", dtype=torch.uint8).view(E4M3)
    v = buf[:, :t[0].numel()].view(torch.uint8)
    v.copy_(t.reshape(R, -1).view(torch.uint8))
    return v.view(E4M3).unflatten(1, t.shape[1:])


# few rows, small products, tiles of each width, splits along k, sizes off the boundary, the most workers
@pytest.mark.parametrize("R,M,N,K", [(3, 1, 64, 64), (2, 40, 24, 8), (3, 300, 264, 192), (8, 20, 520, 256), (32, 5, 130, 65), (32, 70, 96, 128),
                                     (2, 2000, 1100, 264), (4, 9, 33, 129), (2, 140, 256, 4096), (5, 257, 130, 129)])
@pytest.mark.parametrize("out,pad", [(BF16, 0), (F32, 16), (F16, 5)])
def test_8_bit_products_of_a_weight_per_worker(L, R, M, N, K, out, pad):
    scale = torch.pow(2.0, torch.arange(R, device="cuda").float() % 5)[:, None, None]          # workers are told apart by more than chance
    x, w = L.quantize(rand((R, M, K), F32, 1) * scale), L.quantize(rand((R, N, K), F32, 2, K ** -0.5) / scale)
    bias, res = rand((R, N), F32, 3), rand((R, M, N), out, 4)
    values = apart(w.values, pad) if pad else w.values
    r = L.linear(x.values, values, bias, activation="silu", residual=res, x_scale=x.scale, weight_scale=w.scale, dtype=out, save=True)
    z, size = ref.product(x.values.float(), w.values.float())
    s = x.scale.double()[:, :, None] * w.scale.double()[:, None]
    z, slack = z * s + bias.double()[:, None], ((K + 8) * E + 4 * E) * size * s
    slack = slack + 2 * E * (z.abs() + bias.double().abs()[:, None])
    near(r.pre, z, slack, out)
    near(r.out, ref.activate(z, "silu") + res.double(), 1.13 * slack + 8 * E * (z.abs() + 1) + 2 * E * res.double().abs(), out)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,N,K", [(3, 40, 72), (70, 65, 33), (150, 264, 520)])
def test_the_most_workers(L, dtype, M, N, K):
    """32 of them, parameters and their gradients in stretches of a batch's rows."""
    R = 32
    flat, grad = rand((R, K + N * K + N + 3), F32, 1, K ** -0.5), torch.full((R, K + N * K + N + 3), 7.0, device="cuda")
    cut = lambda t: (t[:, 3:3 + K], t[:, 3 + K:3 + K + N * K].view(R, N, K), t[:, 3 + K + N * K:])  # noqa: E731
    (norm, w, b), (dnorm, dw, db) = cut(flat), cut(grad)
    x, g = rand((R, M, K), dtype, 2), rand((R, M, N), dtype, 3, 0.1)
    n = L.rms_norm(x, norm)
    y, _, _ = ref.rms_norm(x, norm, None, 1e-6)
    near(n.out, y, (K / 2 + 9) * E * y.abs(), dtype)
    a = L.linear(n.out, w, b, activation="relu", save=True)
    z, size = ref.product(n.out, w.to(dtype))
    near(a.pre, z + b.double()[:, None], ((K + 8) * E * 1.05 + 6 * E) * (size + b.double().abs()[:, None]), dtype)
    r = L.linear_grad(g, n.out, w, a.pre, "relu", bias=True, out_weight=dw, out_bias=db)
    dz = g.double() * (a.pre > 0)
    want, size = ref.product(dz, w.to(dtype).transpose(1, 2))
    near(r.x, want, ((N + 8) * E * 1.05 + 4 * E) * size, dtype)
    want, size = ref.product(dz.transpose(1, 2), n.out.transpose(1, 2))
    near(dw, want, ((M + 8) * E * 1.05 + 4 * E) * size, F32)
    near(db, dz.sum(1), M * E * dz.abs().sum(1), F32)
    r = L.rms_norm_grad(r.x, n.hidden, n.rstd, norm, out_weight=dnorm)
    _, want, size = ref.rms_norm_grad(L.linear_grad(g, n.out, w, a.pre, "relu", need_weight=False).x, x, n.rstd, norm, None)
    near(dnorm, want, (M + 3) * E * size, F32)
    assert bool((grad[:, :3] == 7).all())
    d = L.dropout(x, 0.4, 3, round=7, layer=1, worker=100, workers=True)
    for i in (0, 17, 31):
        assert torch.equal(d[i], L.dropout(x[i], 0.4, 3, round=7, layer=1, worker=100 + i))
