"""What the residual block's torch functions hand to the library, checked on the host with a stand-in for it, what they refuse
before anything is enqueued, and what the library itself refuses before it touches a device."""
import ctypes as C

import pytest
import torch

from paper_1906_02367_b200 import binding as B
from paper_1906_02367_b200 import layers as L
from paper_1906_02367_b200 import lm

E4M3 = torch.float8_e4m3fn


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 4096 if name.endswith("_bytes") else 0
        return call


@pytest.fixture
def calls(monkeypatch):
    rec = Recorder()
    monkeypatch.setattr(L, "lib", lambda: rec)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for m in (L, lm):
        monkeypatch.setattr(m, "_allocate", lambda stream, shape, dtype, device: torch.zeros(shape, dtype=dtype))
        monkeypatch.setattr(m, "_handle", lambda stream, device: 0)
    return rec.calls


def last(calls, name):
    return [a for n, a in calls if n == name][-1]


X, W = torch.zeros(4, 6), torch.zeros(5, 6)
H = torch.zeros(4, 6, dtype=torch.bfloat16)
REFUSED = {
    "norm of nothing": lambda: L.rms_norm(torch.zeros(4, 0)),
    "integers": lambda: L.rms_norm(torch.zeros(4, 6, dtype=torch.int32)),
    "weight of another width": lambda: L.rms_norm(X, torch.zeros(5)),
    "weight of another type": lambda: L.rms_norm(H, torch.zeros(6, dtype=torch.float16)),
    "weights of other workers": lambda: L.rms_norm(torch.zeros(3, 4, 6), torch.zeros(2, 6)),
    "residual of another shape": lambda: L.rms_norm(X, residual=torch.zeros(4, 5)),
    "residual of another type": lambda: L.rms_norm(X, residual=H),
    "hidden without a residual": lambda: L.rms_norm(X, hidden=X),
    "eps of zero": lambda: L.rms_norm(X, eps=0.0),
    "scale without 8 bits": lambda: L.rms_norm(X, scale=torch.zeros(4)),
    "short scale": lambda: L.rms_norm(X, quantize=True, scale=torch.zeros(3)),
    "out of another type": lambda: L.rms_norm(X, quantize=True, out=torch.zeros(4, 6)),
    "rows that do not flatten": lambda: L.rms_norm(torch.zeros(4, 3, 6).transpose(0, 1)),
    "columns first": lambda: L.rms_norm(torch.zeros(6, 4).t()),
    "gradient of another shape": lambda: L.rms_norm_grad(torch.zeros(3, 6), X, torch.zeros(4)),
    "short rstd": lambda: L.rms_norm_grad(X, X, torch.zeros(3)),
    "accumulate without a place": lambda: L.rms_norm_grad(X, X, torch.zeros(4), torch.zeros(6), accumulate=True),
    "a place without a weight": lambda: L.rms_norm_grad(X, X, torch.zeros(4), out_weight=torch.zeros(6)),
    "weight gradient in 16 bits": lambda: L.rms_norm_grad(X, X, torch.zeros(4), torch.zeros(6), out_weight=torch.zeros(6, dtype=torch.bfloat16)),
    "p of one": lambda: L.dropout(X, 1.0, 0),
    "negative p": lambda: L.dropout(X, -0.1, 0),
    "p of nan": lambda: L.dropout(X, float("nan"), 0),
    "round too large": lambda: L.dropout(X, 0.1, 0, round=1 << 40),
    "layer too large": lambda: L.dropout(X, 0.1, 0, layer=1 << 16),
    "negative worker": lambda: L.dropout(X, 0.1, 0, worker=-1),
    "dropout residual": lambda: L.dropout(X, 0.1, 0, residual=torch.zeros(4, 5)),
    "workers of a vector": lambda: L.dropout(torch.zeros(6), 0.1, 0, workers=True),
    "inner sizes": lambda: L.linear(X, torch.zeros(5, 7)),
    "weights of other workers in a product": lambda: L.linear(torch.zeros(3, 4, 6), torch.zeros(2, 5, 6)),
    "weight of another type in a product": lambda: L.linear(H, torch.zeros(5, 6, dtype=torch.float16)),
    "16-bit weight of fp32 rows": lambda: L.linear(X, W.bfloat16()),
    "weight across": lambda: L.linear(X, torch.zeros(6, 5).t()),
    "empty weight": lambda: L.linear(X, torch.zeros(0, 6)),
    "bias of another size": lambda: L.linear(X, W, torch.zeros(4)),
    "activation": lambda: L.linear(X, W, activation="tanh"),
    "result type": lambda: L.linear(H, W, dtype=torch.float16),
    "residual of the result's type": lambda: L.linear(H, W, residual=torch.zeros(4, 5)),
    "scales of 16 bits": lambda: L.linear(X, W, x_scale=torch.zeros(4)),
    "8 bits without scales": lambda: L.linear(X.to(E4M3), W.to(E4M3)),
    "8 bits with fp32 weights": lambda: L.linear(X.to(E4M3), W, x_scale=torch.zeros(4), weight_scale=torch.zeros(5)),
    "short scales": lambda: L.linear(X.to(E4M3), W.to(E4M3), x_scale=torch.zeros(3), weight_scale=torch.zeros(5)),
    "one 8-bit weight as many": lambda: L.linear(torch.zeros(3, 4, 6).to(E4M3), W.to(E4M3).expand(3, 5, 6), x_scale=torch.zeros(3, 4), weight_scale=torch.zeros(3, 5)),
    "status": lambda: L.linear(X, W, status=torch.zeros(1, dtype=torch.int64)),
    "workspace in pieces": lambda: L.linear(X, W, work=torch.zeros(8192, dtype=torch.uint8)[::2]),
    "gradient of a product of another shape": lambda: L.linear_grad(torch.zeros(4, 6), X, W),
    "gradient of another type": lambda: L.linear_grad(torch.zeros(4, 5, dtype=torch.bfloat16), X, W),
    "no pre": lambda: L.linear_grad(torch.zeros(4, 5), X, W, activation="silu"),
    "weight gradient type": lambda: L.linear_grad(torch.zeros(4, 5), X, W, dtype=torch.float16),
    "place of another gradient": lambda: L.linear_grad(torch.zeros(4, 5), X, W, need_x=False, out=torch.zeros(4, 6)),
    "accumulate into nothing": lambda: L.linear_grad(torch.zeros(4, 5), X, W, accumulate=True),
    "8-bit gradient": lambda: L.linear_grad(torch.zeros(4, 5).to(E4M3), X.to(E4M3), W.to(E4M3)),
    "out without an activation": lambda: L.activation_grad(X, out=X),
}


@pytest.mark.parametrize("what", list(REFUSED))
def test_refused_before_anything_is_enqueued(calls, what):
    with pytest.raises(ValueError):
        REFUSED[what]()
    assert all(n.endswith("_bytes") for n, _ in calls)


def test_strides_of_views_are_handed_on(calls):
    R, M, N, K, d = 3, 4, 5, 6, 100
    batch, grad = torch.zeros(R, d), torch.zeros(R, d)
    w, b = batch[:, 7:7 + N * K].view(R, N, K), batch[:, 50:50 + N]
    x = torch.zeros(R, M, K + 2)[..., :K]
    L.linear(x, w, b, activation="gelu", save=True)
    a = last(calls, "qs_linear")
    assert a[:4] == (R, M, N, K) and a[6] == K + 2 and a[8] == w.data_ptr() and a[10:12] == (d, K) and a[15] == d and a[16] == B.QS_ACT_GELU
    dw, db = grad[:, 7:7 + N * K].view(R, N, K), grad[:, 50:50 + N]
    r = L.linear_grad(torch.zeros(R, M, N), x, w, bias=True, out_weight=dw, out_bias=db)
    a = last(calls, "qs_linear_grad_weight")
    assert a[9] == dw.data_ptr() and a[11:14] == (d, K, 0) and r.weight is dw and r.bias is db
    assert last(calls, "qs_activation_grad")[11:14] == (db.data_ptr(), d, 0)
    # one scratch for all three
    assert last(calls, "qs_activation_grad")[14] == last(calls, "qs_linear_grad_input")[13] == a[14]
    n = batch[:, 3:3 + K]
    L.rms_norm(x, n)
    assert last(calls, "qs_rms_norm")[5] == K + 2 and last(calls, "qs_rms_norm")[8:11] == (n.data_ptr(), B.QS_F32, d)


def test_one_weight_for_all(calls):
    x = torch.zeros(3, 4, 6)
    L.linear(x, W)
    assert last(calls, "qs_linear")[:4] == (1, 12, 5, 6) and last(calls, "qs_linear")[10:12] == (0, 6)
    L.rms_norm(x, torch.zeros(6))
    assert last(calls, "qs_rms_norm")[:3] == (1, 12, 6)
    L.dropout(x, 0.5, -1, workers=True, worker=2)
    a = last(calls, "qs_dropout")
    assert a[:3] == (3, 4, 6) and a[9] == 2**64 - 1 and a[11] == 2
    assert L.activation_grad(x) == (x, None) and calls[-1][0] == "qs_dropout"


# ------------------------------------------------------------------ the C boundary: refused before any device work
P = 1 << 20                                              # an address that nothing looks at


def norm_args(**kw):
    a = dict(R=1, N=4, D=8, x=P, type=0, xs=8, res=None, rs=0, w=None, wt=0, ws=0, eps=1e-6, hid=None, hs=0, out=P + 4096, ot=0, os=8, scale=None,
             rstd=None, st=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(R=0), -1), (dict(R=33), -1), (dict(N=-1), -1), (dict(D=0), -1), (dict(type=7), -1), (dict(ot=1), -1), (dict(eps=0.0), -1),
    (dict(eps=float("inf")), -1), (dict(xs=7), -1), (dict(os=7), -1), (dict(x=None), -1), (dict(x=P + 2), -1), (dict(out=None), -1),
    (dict(res=P + 8192, rs=8), -1), (dict(hid=P + 8192, hs=8), -1), (dict(ot=3), -1), (dict(ot=3, out=P + 16, scale=P + 8192), -1),
    (dict(out=P + 16), -1), (dict(w=P + 8192, wt=1), -1), (dict(w=P + 8192, ws=-1), -1), (dict(D=1 << 25, xs=1 << 25, os=1 << 25), B.QS_TOO_LARGE),
    (dict(N=1 << 31), B.QS_TOO_LARGE), (dict(rstd=P + 8193), -1),
    (dict(res=P + 8192, rs=8, hid=P + 4096, hs=8), -1)])
def test_norm_refusals(kw, code):
    assert B.lib().qs_rms_norm(*norm_args(**kw)) == code


def test_empty_norm_is_no_error():
    assert B.lib().qs_rms_norm(*norm_args(N=0)) == 0


def linear_args(**kw):
    a = dict(R=1, M=4, N=5, K=8, x=P, xt=0, xs=8, xsc=None, w=P + 4096, wt=0, ww=0, ws=8, wsc=None, bias=None, bt=0, bw=0, act=0, res=None, rs=0,
             pre=None, ps=0, out=P + 8192, ot=0, os=5, work=None, bytes=0, status=None, st=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(R=0), -1), (dict(R=33), -1), (dict(M=-1), -1), (dict(N=0), -1), (dict(K=0), -1), (dict(xt=9), -1), (dict(wt=1), -1), (dict(act=4), -1),
    (dict(ot=1), -1), (dict(xt=3), -1), (dict(xt=3, wt=3), -1), (dict(xsc=P), -1), (dict(x=None), -1), (dict(xs=7), -1), (dict(w=P + 4097), -1),
    (dict(os=4), -1), (dict(out=P + 16), -1), (dict(out=P + 4100), -1), (dict(res=P + 8196, rs=5), -1), (dict(pre=P + 8192, ps=5), -1),
    (dict(pre=P + 8, ps=5), -1), (dict(R=2, ww=20), -1), (dict(bias=P + 1), -1), (dict(bias=P, bt=3), -1), (dict(status=P + 2), -1),
    (dict(M=1 << 29), B.QS_TOO_LARGE), (dict(N=1 << 25), B.QS_TOO_LARGE), (dict(K=1 << 25), B.QS_TOO_LARGE),
    (dict(M=1 << 24, N=1 << 20), B.QS_TOO_LARGE)])
def test_linear_refusals(kw, code):
    assert B.lib().qs_linear(*linear_args(**kw)) == code


def test_other_refusals():
    L_ = B.lib()
    drop = lambda **kw: L_.qs_dropout(*{**dict(R=1, N=4, D=8, x=P, t=0, xs=8, r=None, rs=0, p=0.5, seed=0, round=0, worker=0, layer=0, out=P + 4096, os=8,  # noqa: E731
                                              st=None), **kw}.values())
    for kw in (dict(R=0), dict(p=1.0), dict(p=-0.5), dict(p=float("nan")), dict(round=1 << 40), dict(layer=-1), dict(layer=1 << 16), dict(worker=-1),
               dict(t=3), dict(x=None), dict(out=P + 16), dict(xs=7), dict(x=P + 1), dict(r=P + 4100, rs=8)):
        assert drop(**kw) == -1, kw
    assert drop(N=1 << 20, D=1 << 20) == B.QS_TOO_LARGE and drop(N=0) == 0
    assert L_.qs_quantize_rows(4, 8, P, 0, 8, P + 16, 8, P + 4096, None) == -1
    assert L_.qs_quantize_rows(4, 8, P, 3, 8, P + 4096, 8, P + 8192, None) == -1
    grad = lambda **kw: L_.qs_rms_norm_grad(*{**dict(R=1, N=4, D=8, g=P, t=0, gs=8, h=P + 4096, hs=8, rstd=P + 8192, w=None, wt=0, ww=0, gh=None, ghs=0,  # noqa: E731
                                                    out=P + 12288, os=8, dw=None, dww=0, acc=0, work=None, bytes=0, st=None), **kw}.values())
    for kw in (dict(rstd=None), dict(rstd=P + 2), dict(out=P + 16), dict(gh=P + 12292, ghs=8), dict(dw=P + 16384), dict(dw=P + 16384, work=P + 20488)):
        assert grad(**kw) == -1, kw
    assert grad(dw=P + 16384, work=P + 20480, bytes=31) == B.QS_CAPACITY
    act = lambda **kw: L_.qs_activation_grad(*{**dict(R=1, M=4, N=8, g=P, t=0, gs=8, z=P + 4096, zs=8, act=2, out=P + 8192, os=8, db=None, dbw=0, acc=0,  # noqa: E731
                                                     work=None, bytes=0, st=None), **kw}.values())
    for kw in (dict(out=None), dict(z=None), dict(act=9), dict(out=P + 16), dict(out=P + 4100), dict(db=P + 12288), dict(t=3)):
        assert act(**kw) == -1, kw
    weight = lambda **kw: L_.qs_linear_grad_weight(*{**dict(R=1, M=4, N=5, K=8, dz=P, t=0, dzs=5, x=P + 4096, xs=8, out=P + 8192, ot=0, ow=0, os=8, acc=0,  # noqa: E731
                                                           work=None, bytes=0, status=None, st=None), **kw}.values())
    for kw in (dict(ot=1), dict(t=3), dict(out=P + 8), dict(R=2, ow=20), dict(dz=None), dict(os=7)):
        assert weight(**kw) == -1, kw
    assert weight(M=0, acc=1) == 0
    assert L_.qs_linear_bytes(1, 0, 5, 8, None, 0, 8, None, 0, 0, 8) == 0
    assert L_.qs_linear_bytes(1, 4, 5, 8, P, 1, 8, P, 2, 0, 8) == -1
    assert L_.qs_rms_norm_grad_bytes(1, 0, 8) >= 0 and L_.qs_activation_grad_bytes(0, 1, 1) == -1
    assert C.sizeof(C.c_void_p) == 8
