"""Results in their inputs' places on the GPU: what is still to be read is not written over, and what is written over is not handed
out under its old name."""
import pytest
import torch

from test_gpu_layers import BF16, F32, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.fixture
def L():
    from paper_1906_02367_b200 import layers
    return layers


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R,M,N,K", [(1, 5, 24, 40), (1, 300, 264, 520), (3, 150, 130, 65), (2, 700, 520, 264)])
@pytest.mark.parametrize("activation", [None, "silu"])
def test_gradient_of_x_in_its_place(L, dtype, R, M, N, K, activation):
    x, w, g, z = rand((R, M, K), dtype, 1), rand((R, N, K), F32, 2, K ** -0.5), rand((R, M, N), dtype, 3, 0.1), rand((R, M, N), dtype, 4)
    want = L.linear_grad(g, x, w, z, activation, bias=True)
    place = x.clone()
    got = L.linear_grad(g, place, w, z, activation, bias=True, out=place)
    assert got.x is place and all(torch.equal(a, b) for a, b in zip(got, want))
    # into a batch, added to what is there; and the weights' gradient in the weights' place
    batch = rand((R, N * K + N), F32, 5)
    dw, db = (lambda t: (t[:, :N * K].view(R, N, K), t[:, N * K:]))(batch)
    other = batch.clone()
    dw2, db2 = other[:, :N * K].view(R, N, K), other[:, N * K:]
    L.linear_grad(g, x, w, z, activation, out_weight=dw2, out_bias=db2, accumulate=True)
    place = x.clone()
    L.linear_grad(g, place, w, z, activation, out=place, out_weight=dw, out_bias=db, accumulate=True)
    assert torch.equal(batch, other) and torch.equal(place, want.x)
    over = w.clone()
    got = L.linear_grad(g, x, over, z, activation, out_weight=over)
    assert torch.equal(over, want.weight) and torch.equal(got.x, want.x)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,width", [(3, 64), (9, 257), (2, 20000)])
def test_norm_in_its_inputs_place(L, dtype, rows, width):
    """Without a residual h is x itself: there is no hidden to hand out once the result lies there."""
    x, w = rand((rows, width), dtype, 1, 2.0), rand((width,), F32, 2, 0.2, 1.0)
    want = L.rms_norm(x, w)
    assert want.hidden is x
    place = x.clone()
    r = L.rms_norm(place, w, out=place)
    assert r.out is place and torch.equal(place, want.out) and torch.equal(r.rstd, want.rstd)
    assert r.hidden is None
    place = x.clone()
    assert L.rms_norm(place, w, out=place.view(rows, width)).hidden is None
    with pytest.raises((ValueError, AttributeError)):
        L.rms_norm_grad(x, r.hidden, r.rstd, w)
