"""Language-model operators on torch tensors: embedding rows and their gradient, log probabilities of
given tokens, distillation from a teacher's top logits.

Argument checks and marshalling for the qs_embed, qs_token_logp and qs_distill families of
include/qsparse.h, which says what each computes; the arithmetic is in the CUDA library.  Everything is
enqueued on `stream` (default: the current stream of the tensors' device, which must be the current
device) and nothing waits for the GPU.  Tensors made on other streams are the caller's to order, as with any
torch call.  `status`, where taken, is an int32 CUDA tensor of one element, zero before the call, that receives
QS_INVALID_ARG if an id lies past the last row or column, and QS_TIMEOUT if a wait on the device ran out (distill; the
rows concerned are NaN with or without it).
"""
from collections import namedtuple

import torch

from .binding import QS_BF16, QS_F16, QS_F32, QS_I32, QS_I64, QS_MAX_TOP, QsError, lib

TokenLogp = namedtuple("TokenLogp", "logp lse entropy top_ids top_logp")
Distill = namedtuple("Distill", "loss lse log_tail grad")

_TYPE = {torch.float32: QS_F32, torch.bfloat16: QS_BF16, torch.float16: QS_F16}
_ID = {torch.int32: QS_I32, torch.int64: QS_I64}
# a serving loop's calls are as short as their marshalling: the stream's handle without a Stream object around it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _type(t, what, table=_TYPE):
    code = table.get(t.dtype)
    if code is None:
        raise ValueError(f"{what}: {t.dtype} is not one of {', '.join(str(d) for d in table)}")
    return code


def _on(first, *rest):
    """The CUDA device of all the tensors, which must be the current one."""
    device = first.get_device()
    if device < 0 or device != torch.cuda.current_device():
        raise ValueError(f"tensors must be on the current CUDA device, not on {first.device}")
    for t in rest:
        if t is not None and t.get_device() != device:
            raise ValueError(f"tensors on different devices: {first.device} and {t.device}")
    return device


_empty = {}


def _allocate(stream, shape, dtype, device):
    """A tensor that belongs to `stream` (None: the current one); shape: a tuple, or a number of elements."""
    like = _empty.get((dtype, device))
    if like is None:                                     # (new_empty takes half of torch.empty's time on the host)
        like = _empty[dtype, device] = torch.empty(0, dtype=dtype, device=device)
    if stream is None:
        return like.new_empty(shape)
    with torch.cuda.stream(stream):
        return like.new_empty(shape)


def _handle(stream, device):
    return _raw_stream(device) if stream is None else stream.cuda_stream


def _ptr(t):
    return None if t is None else t.data_ptr()


def _word(status):
    """Address of the status word: four bytes that the device writes."""
    if status is None:
        return None
    if status.dtype != torch.int32 or status.numel() == 0:
        raise ValueError(f"status must be one element of torch.int32, not {status.numel()} of {status.dtype}")
    return status.data_ptr()


def _done(rc, what):
    if rc < 0:
        raise QsError(rc, what + (": arguments refused" if rc == -1 else " failed"))


def _rows(t, what):
    """Stride between the rows of a tensor whose last dimension is contiguous and whose others flatten into one.
    (Dimensions of one element have no stride; a single row uses none, and gets one that keeps wide accesses.)"""
    shape, stride = t.shape, t.stride()
    D = shape[-1]
    if len(shape) == 2 and stride[1] == 1 and D:
        return stride[0] if shape[0] > 1 else (D + 15) // 16 * 16
    if t.numel() == 0:
        return D
    if stride[-1] != 1 and D > 1:
        raise ValueError(f"{what} needs rows with unit stride")
    row = outer = None                                   # the rows' stride; the one that the next dimension has to have
    for i in range(len(shape) - 2, -1, -1):
        if shape[i] > 1:
            if row is None:
                row = outer = stride[i]
            elif stride[i] != outer:
                raise ValueError(f"{what}: leading dimensions must flatten into rows of one stride")
            outer *= shape[i]
    return (D + 15) // 16 * 16 if row is None else row


def _vector(t, n, what, dtype=torch.float32):
    if t is not None and (t.dtype != dtype or t.numel() != n or not t.is_contiguous()):
        raise ValueError(f"{what} needs {n} contiguous elements of {dtype}")


def _table(t, R, what):
    """(vocabulary, width, worker stride, row stride) of a (V, D) or (R, V, D) table."""
    shape, stride = t.shape, t.stride()
    if len(shape) not in (2, 3) or (len(shape) == 3 and shape[0] != R):
        raise ValueError(f"{what} must be (V, D), or (R, V, D) for R workers' tokens")
    V, D = shape[-2], shape[-1]
    if stride[-1] != 1 and D > 1:
        raise ValueError(f"{what} needs rows with unit stride")
    row = stride[-2] if V > 1 else max(stride[-2], D)
    return V, D, (stride[0] if len(shape) == 3 and R > 1 else 0), row


def _tokens(tokens, workers):
    """(R, N) of tokens: with a table per worker the first dimension counts the workers."""
    if not tokens.is_contiguous():
        raise ValueError("tokens must be contiguous")
    if workers:
        if tokens.dim() < 2:
            raise ValueError("a table per worker needs tokens (R, ..)")
        R = tokens.shape[0]
        return R, tokens.numel() // R if R else 0
    return 1, tokens.numel()


def embed(tokens, table, scale=1.0, dtype=None, out=None, status=None, stream=None):
    """scale * table[tokens] (qs_embed): tokens (.., N) with a (V, D) table, or (R, .., N) with (R, V, D), one table
    per worker.  Negative tokens give zeros.  Returns tokens.shape + (D,) in `dtype` (default the table's)."""
    device = _on(tokens, table, out, status)
    R, N = _tokens(tokens, table.dim() == 3)
    V, D, ws, rs = _table(table, R, "table")
    shape = (*tokens.shape, D)
    if out is None:
        out = _allocate(stream, shape, dtype or table.dtype, device)
        step = D
    else:
        if out.shape != shape or (dtype is not None and out.dtype != dtype):
            raise ValueError(f"out must be {shape}" + (f" of {dtype}" if dtype else ""))
        step = _rows(out, "out") if len(shape) > 1 else D
    _done(lib().qs_embed(R, N, V, D, tokens.data_ptr(), _type(tokens, "tokens", _ID), table.data_ptr(), _type(table, "table"), ws, rs,
                         scale, out.data_ptr(), _type(out, "out"), step, _word(status), _handle(stream, device)), "qs_embed")
    return out


def embed_grad_work(workers, tokens, vocab, width, device=None):
    """Scratch of embed_grad for `tokens` tokens per worker."""
    n = lib().qs_embed_grad_bytes(workers, tokens, vocab, width)
    _done(n, "qs_embed_grad_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device or "cuda")


def embed_grad(tokens, grad_out, vocab, scale=1.0, workers=None, accumulate=False, out=None, work=None, status=None, stream=None):
    """Gradient of embed with respect to the table(s) (qs_embed_grad), fp32.  grad_out: tokens.shape + (D,).
    workers (default: tokens have more than one dimension, or out has three): a table per entry of the tokens' first
    dimension, result (R, vocab, D); otherwise one table, (vocab, D).  `out` may be a strided view, a stretch of
    the rows of a gradient batch; with accumulate it is added to and rows no token names stay untouched."""
    device = _on(tokens, grad_out, out, work, status)
    if workers is None:
        workers = out.dim() == 3 if out is not None else tokens.dim() > 1
    R, N = _tokens(tokens, workers)
    D = grad_out.shape[-1]
    if grad_out.shape[:-1] != tokens.shape:
        raise ValueError(f"grad_out {tuple(grad_out.shape)} does not belong to tokens {tuple(tokens.shape)}")
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    shape = (R, vocab, D) if workers else (vocab, D)
    if out is None:
        out = _allocate(stream, shape, torch.float32, device)
    elif out.shape != shape or out.dtype != torch.float32:
        raise ValueError(f"out must be {shape} of torch.float32")
    L = lib()
    if work is None:
        need = L.qs_embed_grad_bytes(R, N, vocab, D)
        _done(need, "qs_embed_grad_bytes")
        work = _allocate(stream, need, torch.uint8, device)
    elif not work.is_contiguous():
        raise ValueError("work must be contiguous")
    else:
        need = work.numel() * work.element_size()
    _, _, ws, rs = _table(out, R, "out")
    _done(L.qs_embed_grad(R, N, vocab, D, tokens.data_ptr(), _type(tokens, "tokens", _ID), grad_out.data_ptr(),
                          _type(grad_out, "grad_out"), _rows(grad_out, "grad_out"), scale, int(accumulate), out.data_ptr(), ws, rs,
                          work.data_ptr(), need, _word(status), _handle(stream, device)), "qs_embed_grad")
    return out


def _logits(logits):
    if logits.dim() != 2:
        raise ValueError("logits must be (N, V)")
    return logits.shape[0], logits.shape[1], _rows(logits, "logits")


def token_logp(logits, tokens=None, scale=1.0, top=0, status=None, stream=None):
    """Log probabilities of `tokens` (N) under softmax(scale * logits) (qs_token_logp), with the log of the sum, the
    entropy, and the `top` largest logits' columns and log probabilities (equal logits: lower index first).
    tokens None: no logp, and top_ids are int64.  Returns TokenLogp; fields not asked for are None."""
    device = _on(logits, tokens, status)
    N, V, step = _logits(logits)
    if not 0 <= top <= min(QS_MAX_TOP, V):
        raise ValueError(f"top must be between 0 and {min(QS_MAX_TOP, V)}")
    id_type = torch.int64
    if tokens is not None:
        id_type = tokens.dtype
        _type(tokens, "tokens", _ID)
        _vector(tokens, N, "tokens", id_type)
    f32 = torch.float32
    logp = _allocate(stream, N, f32, device) if tokens is not None else None
    lse, entropy = _allocate(stream, N, f32, device), _allocate(stream, N, f32, device)
    ids = top_logp = None
    if top:
        ids = _allocate(stream, (N, top), id_type, device)
        top_logp = _allocate(stream, (N, top), f32, device)
    _done(lib().qs_token_logp(N, V, logits.data_ptr(), _type(logits, "logits"), step, _ptr(tokens), _ID[id_type], scale, top,
                              _ptr(logp), lse.data_ptr(), entropy.data_ptr(), _ptr(ids), _ptr(top_logp), _word(status),
                              _handle(stream, device)), "qs_token_logp")
    return TokenLogp(logp, lse, entropy, ids, top_logp)


def _gradient(logits, out):
    """Stride of the result's rows."""
    if out.shape != logits.shape or out.dtype != logits.dtype:
        raise ValueError("out must have the logits' shape and type")
    return _rows(out, "out")


def _weights(w, n, what):
    """(pointer, number) of a weight per row or one for all."""
    if isinstance(w, torch.Tensor):
        _vector(w, n, what)
        return w.data_ptr(), 0.0
    return None, float(w)


def token_logp_grad(logits, tokens, lse, grad_logp=1.0, scale=1.0, entropy=None, grad_entropy=None, out=None, status=None, stream=None):
    """Gradient of sum(grad_logp * logp + grad_entropy * entropy) with respect to the logits (qs_token_logp_grad).
    grad_logp: (N) or a number; grad_entropy: (N) or None.  out may be the logits themselves."""
    device = _on(logits, tokens, lse, entropy, grad_entropy, out, status)
    N, V, step = _logits(logits)
    if tokens is not None:
        _vector(tokens, N, "tokens", tokens.dtype)
    if grad_entropy is not None and entropy is None:
        raise ValueError("grad_entropy needs the entropy")
    for t, what in ((lse, "lse"), (entropy, "entropy"), (grad_entropy, "grad_entropy")):
        _vector(t, N, what)
    if isinstance(grad_logp, torch.Tensor):
        _on(logits, grad_logp)
    g, g_all = _weights(grad_logp, N, "grad_logp")
    if out is None:
        out = _allocate(stream, (N, V), logits.dtype, device)
    _done(lib().qs_token_logp_grad(N, V, logits.data_ptr(), _type(logits, "logits"), step, _ptr(tokens),
                                   _type(tokens, "tokens", _ID) if tokens is not None else QS_I64, scale, lse.data_ptr(), _ptr(entropy), g, g_all,
                                   _ptr(grad_entropy), out.data_ptr(), _gradient(logits, out), _word(status), _handle(stream, device)),
          "qs_token_logp_grad")
    return out


def _entries(ids, teacher, N):
    """K of the teacher's entries."""
    if ids.dim() != 2 or ids.shape[0] != N or ids.shape != teacher.shape or not ids.is_contiguous() or not teacher.is_contiguous():
        raise ValueError("ids and teacher must be contiguous (N, K)")
    if not 1 <= ids.shape[1] <= QS_MAX_TOP:
        raise ValueError(f"between 1 and {QS_MAX_TOP} entries per row")
    return ids.shape[1]


def distill(logits, ids, teacher, scale=1.0, teacher_scale=1.0, tail=False, weight=None, out=None, status=None, stream=None):
    """Loss of softmax(scale * logits) against a teacher's top entries (qs_distill): ids (N, K) and the teacher's logits
    there, renormalised, or with `tail` its log probabilities and the rest of its mass as one more class.  token_logp's
    top_ids and top_logp are such entries.  weight (N) or a number: the gradient of sum(weight * loss) with
    respect to the logits as well, from the same pass; out receives it and may be the logits themselves."""
    device = _on(logits, ids, teacher, out, status)
    N, V, step = _logits(logits)
    K = _entries(ids, teacher, N)
    w, w_all = None, 0.0
    if weight is not None:
        if isinstance(weight, torch.Tensor):
            _on(logits, weight)
        w, w_all = _weights(weight, N, "weight")
    elif out is not None:
        raise ValueError("a gradient needs weight")
    loss, lse = _allocate(stream, N, torch.float32, device), _allocate(stream, N, torch.float32, device)
    log_tail = _allocate(stream, N, torch.float32, device) if tail else None
    if weight is not None and out is None:
        out = _allocate(stream, (N, V), logits.dtype, device)
    _done(lib().qs_distill(N, V, K, logits.data_ptr(), _type(logits, "logits"), step, ids.data_ptr(), _type(ids, "ids", _ID),
                           teacher.data_ptr(), _type(teacher, "teacher"), scale, teacher_scale, int(tail), loss.data_ptr(), lse.data_ptr(),
                           _ptr(log_tail), w, w_all, _ptr(out), _gradient(logits, out) if out is not None else 0, _word(status),
                           _handle(stream, device)), "qs_distill")
    return Distill(loss, lse, log_tail, out)


def distill_grad(logits, ids, teacher, lse, weight, scale=1.0, teacher_scale=1.0, tail=False, log_tail=None, out=None, status=None,
                 stream=None):
    """Gradient of sum(weight * loss) on its own (qs_distill_grad), from what distill returned."""
    device = _on(logits, ids, teacher, lse, log_tail, out, status)
    N, V, step = _logits(logits)
    K = _entries(ids, teacher, N)
    _vector(lse, N, "lse")
    if tail and log_tail is None:
        raise ValueError("tail needs log_tail")
    _vector(log_tail, N, "log_tail")
    if isinstance(weight, torch.Tensor):
        _on(logits, weight)
    w, w_all = _weights(weight, N, "weight")
    if out is None:
        out = _allocate(stream, (N, V), logits.dtype, device)
    _done(lib().qs_distill_grad(N, V, K, logits.data_ptr(), _type(logits, "logits"), step, ids.data_ptr(), _type(ids, "ids", _ID),
                                teacher.data_ptr(), _type(teacher, "teacher"), scale, teacher_scale, int(tail), lse.data_ptr(), _ptr(log_tail),
                                w, w_all, out.data_ptr(), _gradient(logits, out), _word(status), _handle(stream, device)),
          "qs_distill_grad")
    return out
