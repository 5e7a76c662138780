"""Operators of a residual block on torch tensors: root-mean-square norm with the residual's addition, dropout from the
counter-based generator, matrix products with bias, activation and residual, and their gradients.

Argument checks and marshalling for the qs_rms_norm, qs_dropout and qs_linear families of include/qsparse.h, which says what
each computes; they stand beside the embedding rows and the losses of lm.py, with the same rules for streams, devices and
status words.  Activations are (.., D); with weights of a worker each, (R, D) or (R, N, K), their first dimension counts the
workers, and weights and gradients may be strided views: stretches of the rows of the R x d batches.
"""
from collections import namedtuple

import torch

from .binding import QS_ACT_GELU, QS_ACT_NONE, QS_ACT_RELU, QS_ACT_SILU, QS_CAPACITY, QS_E4M3, QsError, lib
from .lm import _TYPE, _allocate, _done, _handle, _on, _ptr, _rows, _type, _word

RmsNorm = namedtuple("RmsNorm", "out hidden rstd scale")
RmsNormGrad = namedtuple("RmsNormGrad", "hidden weight")
Quantized = namedtuple("Quantized", "values scale")
Linear = namedtuple("Linear", "out pre")
LinearGrad = namedtuple("LinearGrad", "x weight bias pre")

E4M3 = torch.float8_e4m3fn
_ALL = {**_TYPE, E4M3: QS_E4M3}
_ACT = {None: QS_ACT_NONE, "relu": QS_ACT_RELU, "silu": QS_ACT_SILU, "gelu": QS_ACT_GELU}


def _act(activation):
    if activation not in _ACT:
        raise ValueError(f"activation: {activation!r} is not one of {', '.join(repr(a) for a in _ACT)}")
    return _ACT[activation]


def _like(t, shape, dtype, what):
    """Checks a tensor that goes with another: its shape and type."""
    if t is not None and (t.shape != shape or t.dtype != dtype):
        raise ValueError(f"{what} must be {tuple(shape)} of {dtype}, not {tuple(t.shape)} of {t.dtype}")


def _pitch(t, D, what):
    """Elements between the rows of D of a tensor (None: 0)."""
    if t is None:
        return 0
    if t.is_contiguous():
        return D
    row = _rows(t, what)
    if row < D:
        raise ValueError(f"{what}: rows must not share memory")
    return row


def _counted(t, n, what):
    if t is not None and (t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous()):
        raise ValueError(f"{what} needs {n} contiguous elements of torch.float32")


def _activations(x, workers, what):
    """(R, N, D) of (.., D): with weights of a worker each the first dimension counts the workers."""
    if x.dim() < 1 or x.shape[-1] == 0:
        raise ValueError(f"{what} must be (.., D) with D > 0")
    D = x.shape[-1]
    rows = x.numel() // D
    if not workers:
        return 1, rows, D
    if x.dim() < 2 or x.shape[0] == 0:
        raise ValueError(f"weights of a worker each need {what} (R, .., D)")
    return x.shape[0], rows // x.shape[0], D


def _vector_of(t, R, n, workers, what):
    """Worker stride of a vector of n per worker, (R, n), or of one for all, (n)."""
    if t is None:
        return 0
    if t.shape != ((R, n) if workers else (n,)) or (n > 1 and t.stride(-1) != 1):
        raise ValueError(f"{what} must be {(R, n) if workers else (n,)} with unit stride, not {tuple(t.shape)}")
    return t.stride(0) if workers and R > 1 else (n if workers else 0)


def _matrix_of(t, R, workers, what):
    """(N, K, worker stride, row stride) of an (N, K) or (R, N, K) matrix."""
    if t.dim() != (3 if workers else 2) or (workers and t.shape[0] != R) or 0 in t.shape:
        raise ValueError(f"{what} must be (N, K), or (R, N, K) for R workers, not {tuple(t.shape)}")
    N, K = t.shape[-2], t.shape[-1]
    if t.stride(-1) != 1 and K > 1:
        raise ValueError(f"{what} needs rows with unit stride")
    return N, K, (t.stride(0) if workers and R > 1 else 0), (t.stride(-2) if N > 1 else max(t.stride(-2), K))


def _span(t):
    """The addresses of a tensor's first element and behind its last (None or empty: none)."""
    if t is None or not t.numel():
        return 0, 0
    at = t.data_ptr()
    if t.is_contiguous():
        return at, at + t.nbytes
    return at, at + t.element_size() * (1 + sum((n - 1) * d for n, d in zip(t.shape, t.stride())))


def _cross(a, b):
    return a[0] < b[1] and b[0] < a[1]


def _share(a, b, width):
    """Whether two tensors of rows of one type and width share memory: other columns of the same rows do not."""
    if not _cross(_span(a), _span(b)):
        return False
    row, size = _pitch(a, width, "out"), a.element_size()
    return row != _pitch(b, width, "x") or not width * size <= (b.data_ptr() - a.data_ptr()) % (row * size) <= (row - width) * size


def _work(work, need, what, stream, device):
    """(pointer, bytes) of the scratch: the caller's, or new."""
    _done(need, what)
    if work is None:
        if not need:
            return None, 0, None
        work = _allocate(stream, need, torch.uint8, device)
    elif not work.is_contiguous():
        raise ValueError("work must be contiguous")
    return work.data_ptr(), work.numel() * work.element_size(), work


# ------------------------------------------------------------------ norm
def rms_norm(x, weight=None, residual=None, eps=1e-6, quantize=False, out=None, hidden=None, scale=None, rstd=None, stream=None):
    """h = x + residual, h / sqrt(mean h^2 + eps) * weight (qs_rms_norm).  x (.., D); weight (D), or (R, D) for x (R, .., D), in
    fp32 or x's type.  quantize: the result in 8 bits (torch.float8_e4m3fn) with a scale per row.  Returns RmsNorm(out, hidden,
    rstd, scale): hidden is h, in x's type (x itself without a residual, None where out has taken x's place); scale is None unless
    quantize.  rstd False: not wanted."""
    device = _on(x, weight, residual, out, hidden, scale, rstd if isinstance(rstd, torch.Tensor) else None)
    workers = weight is not None and weight.dim() == 2
    R, N, D = _activations(x, workers, "x")
    w_step = _vector_of(weight, R, D, workers, "weight")
    code = _type(x, "x")
    if weight is not None and weight.dtype not in (x.dtype, torch.float32):
        raise ValueError(f"weight must be of {x.dtype} or torch.float32, not {weight.dtype}")
    if not eps > 0.0:
        raise ValueError("eps must be positive")
    shape = x.shape
    _like(residual, shape, x.dtype, "residual")
    if residual is None:
        if hidden is not None:
            raise ValueError("hidden needs a residual")
    elif hidden is None:
        hidden = _allocate(stream, shape, x.dtype, device)
    else:
        _like(hidden, shape, x.dtype, "hidden")
    out_type, kept = E4M3 if quantize else x.dtype, x if residual is None else hidden
    if out is None:
        out = _allocate(stream, shape, out_type, device)
    else:
        _like(out, shape, out_type, "out")
        if residual is None and not quantize and _share(out, x, D):
            kept = None
    if quantize:
        if scale is None:
            scale = _allocate(stream, shape[:-1], torch.float32, device)
        _counted(scale, R * N, "scale")
    elif scale is not None:
        raise ValueError("scale belongs to quantize")
    if rstd is None:
        rstd = _allocate(stream, shape[:-1], torch.float32, device)
    elif rstd is False:
        rstd = None
    else:
        _counted(rstd, R * N, "rstd")
    _done(lib().qs_rms_norm(R, N, D, x.data_ptr(), code, _pitch(x, D, "x"), _ptr(residual), _pitch(residual, D, "residual"), _ptr(weight),
                            code if weight is None else _TYPE[weight.dtype], w_step, eps, _ptr(hidden), _pitch(hidden, D, "hidden"), out.data_ptr(),
                            _ALL[out_type], _pitch(out, D, "out"), _ptr(scale), _ptr(rstd), _handle(stream, device)), "qs_rms_norm")
    return RmsNorm(out, kept, rstd, scale)


def quantize(x, out=None, scale=None, stream=None):
    """Rows of x (.., D) in 8 bits with a scale per row (qs_quantize_rows): weights laid out once for `linear`, or
    activations that come from elsewhere.  Returns Quantized(values, scale)."""
    device = _on(x, out, scale)
    R, N, D = _activations(x, False, "x")
    code = _type(x, "x")
    if out is None:
        out = _allocate(stream, x.shape, E4M3, device)
    _like(out, x.shape, E4M3, "out")
    if scale is None:
        scale = _allocate(stream, x.shape[:-1], torch.float32, device)
    _counted(scale, N, "scale")
    _done(lib().qs_quantize_rows(N, D, x.data_ptr(), code, _pitch(x, D, "x"), out.data_ptr(), _pitch(out, D, "out"), scale.data_ptr(),
                                 _handle(stream, device)), "qs_quantize_rows")
    return Quantized(out, scale)


def rms_norm_grad(grad_out, hidden, rstd, weight=None, grad_hidden=None, out=None, out_weight=None, accumulate=False, work=None, stream=None):
    """Gradient of rms_norm (qs_rms_norm_grad) from its hidden and rstd: with respect to hidden (so to x and to residual;
    grad_hidden, what arrives by the residual stream, is added), and to the weight, fp32 (out_weight may be a stretch of
    the rows of a gradient batch; accumulate adds to it).  Returns RmsNormGrad(hidden, weight); weight None: none."""
    if hidden is None:
        raise ValueError("hidden is needed: a norm's result that took x's place left none")
    device = _on(hidden, grad_out, rstd, weight, grad_hidden, out, out_weight, work)
    workers = weight is not None and weight.dim() == 2
    R, N, D = _activations(hidden, workers, "hidden")
    w_step = _vector_of(weight, R, D, workers, "weight")
    code = _type(hidden, "hidden")
    if weight is not None and weight.dtype not in (hidden.dtype, torch.float32):
        raise ValueError(f"weight must be of {hidden.dtype} or torch.float32, not {weight.dtype}")
    _like(grad_out, hidden.shape, hidden.dtype, "grad_out")
    _like(grad_hidden, hidden.shape, hidden.dtype, "grad_hidden")
    _counted(rstd, R * N, "rstd")
    if accumulate and out_weight is None:
        raise ValueError("accumulate needs out_weight")
    if out is None:
        out = _allocate(stream, hidden.shape, hidden.dtype, device)
    _like(out, hidden.shape, hidden.dtype, "out")
    dw_step, ptr, size, keep = 0, None, 0, None
    if weight is None:
        if out_weight is not None:
            raise ValueError("out_weight needs weight")
    else:
        if out_weight is None:
            out_weight = _allocate(stream, weight.shape, torch.float32, device)
        _like(out_weight, weight.shape, torch.float32, "out_weight")
        dw_step = _vector_of(out_weight, R, D, workers, "out_weight")
        ptr, size, keep = _work(work, lib().qs_rms_norm_grad_bytes(R, N, D), "qs_rms_norm_grad_bytes", stream, device)
    _done(lib().qs_rms_norm_grad(R, N, D, grad_out.data_ptr(), code, _pitch(grad_out, D, "grad_out"), hidden.data_ptr(), _pitch(hidden, D, "hidden"),
                                 rstd.data_ptr(), _ptr(weight), code if weight is None else _TYPE[weight.dtype], w_step, _ptr(grad_hidden),
                                 _pitch(grad_hidden, D, "grad_hidden"), out.data_ptr(), _pitch(out, D, "out"), _ptr(out_weight), dw_step, int(accumulate), ptr, size, _handle(stream, device)),
          "qs_rms_norm_grad")
    return RmsNormGrad(out, out_weight)


# ------------------------------------------------------------------ dropout
def dropout(x, p, seed, round=0, layer=0, worker=0, workers=False, residual=None, out=None, stream=None):
    """residual + dropout(x) (qs_dropout): an element is dropped with probability p, the others are divided by 1 - p.  Which
    ones depends on seed, round, layer, the worker and the element's number alone, so the gradient is
    dropout(grad, ..) with the same key and no residual.  workers: x is (R, .., D), its first dimension the workers worker,
    worker + 1, ..; otherwise all of x is worker `worker`'s."""
    device = _on(x, residual, out)
    R, N, D = _activations(x, workers, "x")
    code = _type(x, "x")
    _like(residual, x.shape, x.dtype, "residual")
    if not 0.0 <= p < 1.0:
        raise ValueError("p must be at least 0 and below 1")
    if not 0 <= round < 1 << 40 or not 0 <= layer < 1 << 16 or not 0 <= worker < 1 << 31:
        raise ValueError("round must be below 2^40, layer below 2^16, worker below 2^31, none negative")
    if out is None:
        out = _allocate(stream, x.shape, x.dtype, device)
    else:
        _like(out, x.shape, x.dtype, "out")
    _done(lib().qs_dropout(R, N, D, x.data_ptr(), code, _pitch(x, D, "x"), _ptr(residual), _pitch(residual, D, "residual"), p,
                           seed & 0xFFFFFFFFFFFFFFFF, round, worker, layer, out.data_ptr(), _pitch(out, D, "out"), _handle(stream, device)), "qs_dropout")
    return out


# ------------------------------------------------------------------ products
def _operands(x, weight):
    """(workers?, R, M, N, K, worker stride, row stride of the weight)."""
    workers = weight.dim() == 3
    R, M, K = _activations(x, workers, "x")
    N, inner, w_worker, w_row = _matrix_of(weight, R, workers, "weight")
    if inner != K:
        raise ValueError(f"x {tuple(x.shape)} does not go with weight {tuple(weight.shape)}")
    if weight.dtype != x.dtype and (weight.dtype != torch.float32 or x.dtype == E4M3):
        raise ValueError(f"weight must be of {x.dtype}" + ("" if x.dtype == E4M3 else " or torch.float32") + f", not {weight.dtype}")
    return workers, R, M, N, K, w_worker, w_row


def linear(x, weight, bias=None, activation=None, residual=None, x_scale=None, weight_scale=None, save=False, dtype=None, out=None, pre=None,
           work=None, status=None, stream=None):
    """act(x weight^T + bias) + residual (qs_linear).  x (.., K) with weight (N, K), or (R, .., K) with (R, N, K), a weight
    per worker; weight in x's type, or fp32 and rounded to it.  activation: None, "relu", "silu", "gelu".  x and weight in 8
    bits come with x_scale, one per row, and weight_scale, one per row of weight (`rms_norm`, `quantize`).  save: also
    the values in front of the activation, for linear_grad.  Returns Linear(out, pre) in `dtype` (default x's type; bf16
    for 8 bits); residual is of that type too."""
    device = _on(x, weight, bias, residual, x_scale, weight_scale, out, pre, work, status)
    workers, R, M, N, K, w_worker, w_row = _operands(x, weight)
    act, eight = _act(activation), x.dtype == E4M3
    x_code = _type(x, "x", _ALL)
    shape = (*x.shape[:-1], N)
    if dtype is None:
        dtype = out.dtype if out is not None else torch.bfloat16 if eight else x.dtype
    if dtype not in _TYPE or not (eight or dtype in (x.dtype, torch.float32)):
        raise ValueError(f"the result cannot be of {dtype}")
    if eight:
        if x_scale is None or weight_scale is None:
            raise ValueError("8-bit operands need x_scale and weight_scale")
        _counted(x_scale, R * M, "x_scale")
        _counted(weight_scale, (R if workers else 1) * N, "weight_scale")
        if workers and R > 1 and w_worker == 0:
            raise ValueError("8-bit weights that all workers share are (N, K), with one scale per row")
    elif x_scale is not None or weight_scale is not None:
        raise ValueError("scales belong to 8-bit operands")
    bias_step = _vector_of(bias, R, N, workers, "bias")
    bias_type = _type(bias, "bias") if bias is not None else 0
    _like(residual, shape, dtype, "residual")
    if out is None:
        out = _allocate(stream, shape, dtype, device)
    _like(out, shape, dtype, "out")
    if save and pre is None:
        pre = _allocate(stream, shape, dtype, device)
    _like(pre, shape, dtype, "pre")
    L = lib()
    x_row, w_code, in_place = _pitch(x, K, "x"), _ALL[weight.dtype], residual is not None and residual.data_ptr() == out.data_ptr()
    ptr, size, keep = _work(work, L.qs_linear_call_bytes(R, M, N, K, x.data_ptr(), x_code, x_row, weight.data_ptr(), w_code, w_worker, w_row,
                                                         _TYPE[dtype], int(in_place)), "qs_linear_call_bytes", stream, device)
    _done(L.qs_linear(R, M, N, K, x.data_ptr(), x_code, x_row, _ptr(x_scale), weight.data_ptr(), w_code, w_worker, w_row, _ptr(weight_scale),
                      _ptr(bias), bias_type, bias_step, act, _ptr(residual), _pitch(residual, N, "residual"), _ptr(pre), _pitch(pre, N, "pre"),
                      out.data_ptr(), _TYPE[dtype], _pitch(out, N, "out"), ptr, size, _word(status), _handle(stream, device)), "qs_linear")
    return Linear(out, pre)


def activation_grad(grad_out, pre=None, activation=None, out=None, bias=False, out_bias=None, workers=False, accumulate=False, work=None,
                    stream=None):
    """grad_out * act'(pre) and the sum of it over the rows (qs_activation_grad).  Without an activation the first is grad_out
    itself.  bias: the sums too, fp32, (N) or with workers (R, N); out_bias receives them (accumulate adds).
    Returns (gradient, bias gradient or None)."""
    device = _on(grad_out, pre, out, out_bias, work)
    act, code = _act(activation), _type(grad_out, "grad_out")
    R, M, N = _activations(grad_out, workers, "grad_out")
    if act != QS_ACT_NONE:
        if pre is None:
            raise ValueError("the gradient of an activation needs pre")
        _like(pre, grad_out.shape, grad_out.dtype, "pre")
        if out is None:
            out = _allocate(stream, grad_out.shape, grad_out.dtype, device)
        _like(out, grad_out.shape, grad_out.dtype, "out")
    elif out is not None:
        raise ValueError("without an activation there is nothing to write into out")
    bias = bias or out_bias is not None
    if accumulate and out_bias is None:
        raise ValueError("accumulate needs out_bias")
    ptr, size, keep, step = None, 0, None, 0
    if bias:
        if out_bias is None:
            out_bias = _allocate(stream, (R, N) if workers else (N,), torch.float32, device)
        _like(out_bias, (R, N) if workers else (N,), torch.float32, "out_bias")
        step = _vector_of(out_bias, R, N, workers, "out_bias")
        ptr, size, keep = _work(work, lib().qs_activation_grad_bytes(R, M, N), "qs_activation_grad_bytes", stream, device)
    elif out is None:
        return grad_out, None
    _done(lib().qs_activation_grad(R, M, N, grad_out.data_ptr(), code, _pitch(grad_out, N, "grad_out"), _ptr(pre) if act else None,
                                   _pitch(pre, N, "pre") if act else 0, act, _ptr(out), _pitch(out, N, "out"), _ptr(out_bias), step, int(accumulate), ptr, size, _handle(stream, device)), "qs_activation_grad")
    return (grad_out if out is None else out), out_bias


def linear_grad(grad_out, x, weight, pre=None, activation=None, need_x=True, need_weight=True, bias=False, dtype=torch.float32, out=None,
                out_weight=None, out_bias=None, accumulate=False, work=None, status=None, stream=None):
    """Gradients of act(x weight^T + bias) from that of its result (qs_activation_grad, qs_linear_grad_input,
    qs_linear_grad_weight); the residual's is grad_out itself.  pre: what linear saved (not needed without an activation).
    The gradient in front of the activation is rounded to grad_out's type, which is x's.  The weight's gradient is of `dtype`
    (fp32 or x's type), the bias's fp32; out_weight and out_bias may be stretches of a gradient batch, and accumulate adds
    to them.  out may take x's place, or out_weight weight's, not both.  Returns LinearGrad(x, weight, bias, pre): None for what
    was not asked for; pre is the gradient in front of the activation."""
    device = _on(x, weight, grad_out, pre, out, out_weight, out_bias, work, status)
    workers, R, M, N, K, w_worker, w_row = _operands(x, weight)
    code, act = _type(x, "x"), _act(activation)
    _like(grad_out, (*x.shape[:-1], N), x.dtype, "grad_out")
    if not need_x and out is not None or not need_weight and out_weight is not None:
        raise ValueError("out and out_weight belong to gradients that are asked for")
    if accumulate and (need_weight and out_weight is None or bias and out_bias is None):
        raise ValueError("accumulate needs out_weight and out_bias for what it is to be added to")
    place, weight_place = out, out_weight                # (of the caller's: what is made here meets nothing)
    if need_weight:
        if out_weight is None:
            if dtype not in (x.dtype, torch.float32):
                raise ValueError(f"the weight's gradient cannot be of {dtype}")
            out_weight = _allocate(stream, weight.shape, dtype, device)
        elif out_weight.dtype not in (x.dtype, torch.float32) or out_weight.shape != weight.shape:
            raise ValueError(f"out_weight must be {tuple(weight.shape)} of {x.dtype} or torch.float32")
        _, _, g_worker, g_row = _matrix_of(out_weight, R, workers, "out_weight")
        if g_row < K or R > 1 and g_worker < (N - 1) * g_row + K and (g_worker < K or g_row < (R - 1) * g_worker + K):
            raise ValueError("out_weight's rows must not share memory")
    if need_x:
        if out is None:
            out = _allocate(stream, x.shape, x.dtype, device)
        _like(out, x.shape, x.dtype, "out")
    # all that one of the three calls would refuse, before another has added to a gradient; each of the two products reads what the
    # other may be written over, so the weight's comes first where out takes x's place
    weight_first = False
    if place is not None or weight_place is not None:
        to, to_w, of, of_w, read = _span(place), _span(weight_place), _span(x), _span(weight), _span(grad_out if act == QS_ACT_NONE else None)
        if _cross(to, read) or _cross(to, of_w):
            raise ValueError("out must lie apart from grad_out and weight")
        if _cross(to_w, read) or _cross(to_w, of):
            raise ValueError("out_weight must lie apart from grad_out and x")
        weight_first = need_weight and _cross(to, of) and _share(place, x, K)
        if weight_first and _cross(to_w, of_w):
            raise ValueError("out in x's place and out_weight in weight's: each gradient needs what the other would be written over")
    if need_x and w_row < K:
        raise ValueError("weight's rows must not share memory")
    L, bias = lib(), bias or out_bias is not None
    dz = grad_out if act == QS_ACT_NONE else _allocate(stream, grad_out.shape, grad_out.dtype, device)
    dz_row, x_row, out_row = _pitch(dz, N, "grad_out"), _pitch(x, K, "x") if need_weight else K, _pitch(out, K, "out")
    to_x = (R, M, N, K, dz.data_ptr(), code, dz_row, weight.data_ptr(), _TYPE[weight.dtype], w_worker, w_row)
    to_weight = (R, M, N, K, dz.data_ptr(), code, dz_row, x.data_ptr(), x_row)
    # one scratch for the three calls, which follow one another
    need = [L.qs_activation_grad_bytes(R, M, N) if bias else 0, L.qs_linear_grad_input_bytes(*to_x) if need_x else 0,
            L.qs_linear_grad_weight_call_bytes(*to_weight, _TYPE[out_weight.dtype]) if need_weight else 0]
    for n, what in zip(need, ("qs_activation_grad_bytes", "qs_linear_grad_input_bytes", "qs_linear_grad_weight_call_bytes")):
        _done(n, what)
    given = work is not None
    ptr, size, work = _work(work, max(need), "scratch", stream, device)
    if given and size < max(need):
        raise QsError(QS_CAPACITY, f"work holds {size} bytes of {max(need)}")
    if given and ptr % (256 if max(need[1:]) else 16):
        raise ValueError("work must lie on a boundary of 256 bytes")
    word, handle = _word(status), _handle(stream, device)
    db = None
    if bias or act != QS_ACT_NONE:
        _, db = activation_grad(grad_out, pre, activation, out=dz if act != QS_ACT_NONE else None, bias=bias, out_bias=out_bias, workers=workers,
                                accumulate=accumulate and out_bias is not None, work=work if bias else None, stream=stream)
    for product in ("weight", "x") if weight_first else ("x", "weight"):
        if product == "x" and need_x:
            _done(L.qs_linear_grad_input(*to_x, out.data_ptr(), out_row, ptr, size, word, handle), "qs_linear_grad_input")
        if product == "weight" and need_weight:
            _done(L.qs_linear_grad_weight(*to_weight, out_weight.data_ptr(), _TYPE[out_weight.dtype], g_worker, g_row, int(accumulate), ptr, size, word,
                                          handle), "qs_linear_grad_weight")
    return LinearGrad(out, out_weight, db, dz)
