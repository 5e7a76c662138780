"""Results in their inputs' places, on the host with a stand-in for the library: the order of a call's parts, and refusals that come
before anything is enqueued."""
import pytest
import torch

from paper_1906_02367_b200 import binding as B
from paper_1906_02367_b200 import layers as L
from test_layers_arguments import calls  # noqa: F401


def names(calls):  # noqa: F811
    return [n for n, _ in calls if not n.endswith("_bytes")]


def test_the_weights_gradient_reads_x_before_its_place_is_taken(calls):  # noqa: F811
    x, w, g = torch.zeros(4, 6), torch.zeros(5, 6), torch.zeros(4, 5)
    order = ["qs_linear_grad_weight", "qs_linear_grad_input"]
    r = L.linear_grad(g, x, w, out=x)
    assert names(calls) == order and r.x is x
    calls.clear()
    L.linear_grad(g, x, w, out=x.view(2, 2, 6).view(4, 6), bias=True)
    assert names(calls) == ["qs_activation_grad"] + order
    calls.clear()
    L.linear_grad(g, x, w, out=x, need_weight=False)
    assert names(calls) == order[1:]
    # the weight's place is free once the input's gradient is there
    calls.clear()
    L.linear_grad(g, x, w, out_weight=w)
    L.linear_grad(g, x, w)
    assert names(calls) == order[::-1] * 2
    # other columns of the same rows are no place of x's; one that reaches into them is
    wide = torch.zeros(4, 20)
    calls.clear()
    L.linear_grad(g, wide[:, :6], w, out=wide[:, 6:12])
    assert names(calls) == order[::-1]
    calls.clear()
    L.linear_grad(g, wide[:, :6], w, out=wide[:, 5:11])
    assert names(calls) == order
    long = torch.zeros(60)
    calls.clear()
    L.linear_grad(g, long[:24].view(4, 6), w, out=long[24:48].view(4, 6))
    assert names(calls) == order[::-1]
    calls.clear()
    L.linear_grad(g, long[:24].view(4, 6), w, out=long[18:42].view(4, 6))
    assert names(calls) == order


def test_both_places_at_once_are_refused(calls):  # noqa: F811
    x, w, g = torch.zeros(4, 6), torch.zeros(5, 6), torch.zeros(4, 5)
    with pytest.raises(ValueError):
        L.linear_grad(g, x, w, out=x, out_weight=w, bias=True)
    assert names(calls) == []


def test_a_norm_in_its_inputs_place_hands_out_no_hidden(calls):  # noqa: F811
    x, w = torch.zeros(4, 6), torch.zeros(6)
    assert L.rms_norm(x, w).hidden is x
    assert L.rms_norm(x, w, out=x).hidden is None and L.rms_norm(x, w, out=x.view(4, 6)).hidden is None
    res = torch.zeros(4, 6)
    assert L.rms_norm(x, w, res, hidden=res, out=x).hidden is res and L.rms_norm(x, w, res, out=x).hidden is not None
    wide = torch.zeros(4, 20)
    assert L.rms_norm(wide[:, :6], w, out=wide[:, 6:12]).hidden is not None
    with pytest.raises(ValueError):
        L.rms_norm_grad(x, None, torch.zeros(4), w)


BAD = {
    "status": lambda x, w, g, dw, db: dict(status=torch.zeros(1)),
    "short work": lambda x, w, g, dw, db: dict(work=torch.zeros(4095, dtype=torch.uint8)),
    "work off its boundary": lambda x, w, g, dw, db: dict(work=torch.zeros(8192, dtype=torch.uint8)[1:]),
    "out in grad_out's place": lambda x, w, g, dw, db: dict(out=g),
    "out in weight's place": lambda x, w, g, dw, db: dict(out=w),
    "out_weight in x's place": lambda x, w, g, dw, db: dict(out_weight=x),
    "out_weight in grad_out's place": lambda x, w, g, dw, db: dict(out_weight=g),
    "out_weight that its rows share": lambda x, w, g, dw, db: dict(out_weight=dw[:1].expand(6, 6)),
    "rows of out that overlap": lambda x, w, g, dw, db: dict(out=torch.zeros(36).as_strided((6, 6), (5, 1))),
}


@pytest.mark.parametrize("what", list(BAD))
def test_gradients_are_refused_before_any_is_added_to(calls, what):  # noqa: F811
    x, w, g, dw, db = torch.zeros(6, 6), torch.zeros(6, 6), torch.zeros(6, 6), torch.zeros(6, 6), torch.zeros(6)
    good = dict(out_weight=dw, out_bias=db, accumulate=True)
    L.linear_grad(g, x, w, **good)
    assert len(names(calls)) == 3
    calls.clear()
    with pytest.raises((ValueError, B.QsError)):
        L.linear_grad(g, x, w, **{**good, **BAD[what](x, w, g, dw, db)})
    assert names(calls) == []


@pytest.mark.parametrize("what", ["x", "grad_out", "weight"])
def test_operands_that_share_rows_are_refused_before_any_gradient_is_added_to(calls, what):  # noqa: F811
    t = dict(x=torch.zeros(6, 6), grad_out=torch.zeros(6, 6), weight=torch.zeros(6, 6))
    t[what] = t[what][:1].expand(6, 6)
    with pytest.raises((ValueError, B.QsError)):
        L.linear_grad(t["grad_out"], t["x"], t["weight"], out_weight=torch.zeros(6, 6), out_bias=torch.zeros(6), accumulate=True)
    assert names(calls) == []


def test_the_gradient_behind_an_activation_may_take_grad_outs_place(calls):  # noqa: F811
    x, w, g, z = torch.zeros(6, 6), torch.zeros(6, 6), torch.zeros(6, 6), torch.zeros(6, 6)
    r = L.linear_grad(g, x, w, z, "relu", out=g)
    assert r.x is g and len(names(calls)) == 3


def test_the_workspace_goes_by_the_results_type_and_place(calls):  # noqa: F811
    x, w, r = torch.zeros(4, 6, dtype=torch.bfloat16), torch.zeros(5, 6), torch.zeros(4, 5)
    L.linear(x, w, residual=r, out=r)
    assert [a[-2:] for n, a in calls if n == "qs_linear_call_bytes"] == [(B.QS_F32, 1)]
    calls.clear()
    L.linear(x, w, residual=r, dtype=torch.float32)
    L.linear(x, w)
    assert [a[-2:] for n, a in calls if n == "qs_linear_call_bytes"] == [(B.QS_F32, 0), (B.QS_BF16, 0)]
    calls.clear()
    L.linear_grad(torch.zeros(4, 5, dtype=torch.bfloat16), x, w, dtype=torch.bfloat16)
    L.linear_grad(torch.zeros(4, 5, dtype=torch.bfloat16), x, w)
    assert [a[-1] for n, a in calls if n == "qs_linear_grad_weight_call_bytes"] == [B.QS_BF16, B.QS_F32]


def test_workspace_sizes_are_refused_as_the_calls_are():
    P, lib = 1 << 20, B.lib()
    of = lambda **kw: lib.qs_linear_call_bytes(*{**dict(R=1, M=4, N=5, K=8, x=P, xt=1, xs=8, w=P, wt=0, ww=0, ws=8, ot=0, at=0), **kw}.values())  # noqa: E731
    for kw in (dict(R=0), dict(K=0), dict(ot=3), dict(ot=9), dict(wt=2), dict(M=-1)):
        assert of(**kw) == -1, kw
    assert of(N=1 << 25) == B.QS_TOO_LARGE and of(M=0) == 0
    of = lambda **kw: lib.qs_linear_grad_weight_call_bytes(*{**dict(R=1, M=4, N=5, K=8, dz=P, t=1, dzs=5, x=P, xs=8, ot=0), **kw}.values())  # noqa: E731
    for kw in (dict(R=33), dict(N=0), dict(ot=2), dict(t=3, ot=3), dict(t=0, ot=1)):
        assert of(**kw) == -1, kw
    assert of(M=1 << 29) == B.QS_TOO_LARGE and of(M=0) == 0
