"""Binding of the operators between a layer's last activations and the next token
(the third part of lda_draw.h): the rows' norm and its gradient, rows in 8 bits,
their product with 8-bit weights, and the choice of a token by a uniform number.
Argument marshalling only, in the manner of ``_tokens``: rows may lie at any
distance, what a call is given to write into counts as changed in place, and no
call records a gradient (``norm_grad`` is the norm's backward pass; the 8-bit
product is for answering, and has none).
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import _lib
from ._lib import _require
from ._tokens import (_F32, _I32, _MAX_I32, _U8, _UNSUPPORTED, DTYPES, _cut_off, _entry,
                      _mark_written, _rows, _run, _Tensor, _vector)

_I8 = torch.int8
_LDA_I8 = 3
MAX_PRODUCT_K = 131071  # LDA_PROJECT_MAX_K
_empty_like = torch.empty_like
_recording = torch.is_grad_enabled


def bind(lib: ctypes.CDLL) -> None:
    """Argument types of the entry points (called when the library is loaded)."""
    P, I32, I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    F64, SZ = ctypes.c_double, ctypes.c_size_t
    for name, args in (
            ("lda_add_norm", [P, I64, P, I64, P, P, I64, P, I64, P, I64, I32, I32, I32, I32, F64,
                              P]),
            ("lda_norm_grad", [P, I64, P, I64, P, I64, P, P, I64, P, I64, I32, I32, I32, F64, I32,
                               P, SZ, P]),
            ("lda_quantise_rows", [P, I64, P, I64, P, I64, I32, I32, P]),
            ("lda_project_int8", [P, I64, P, P, I64, P, P, P, I64, I64, I32, I32, I32, P]),
            ("lda_sample_logits", [P, I64, I64, I32, I32, P, P, P, P, P, P, P, P])):
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = ctypes.c_int
    lib.lda_norm_grad_workspace_bytes.argtypes = [I64, I32]
    lib.lda_norm_grad_workspace_bytes.restype = SZ


def _matrix(t, name: str):
    """A contiguous tensor as the matrix of its last dimension's rows; a matrix as it
    is."""
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dim() == 2:
        return t
    if t.dim() == 0:
        raise ValueError(f"{name} must have at least 1 dimension")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.view(-1 if t.numel() else 0, t.shape[-1])


def _like(t, name: str, x, dev: int, dtype, shape, out: bool = False) -> tuple[int, int]:
    """(address, elements from row to row) of a tensor of ``x``'s shape."""
    if isinstance(t, _Tensor) and t.dim() == 2 and x.dim() == 2:
        return t.data_ptr(), _rows(t, name, dev, dtype, shape, out)[2]
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.shape != x.shape:
        raise ValueError(f"{name} must have the shape {tuple(x.shape)}, got {tuple(t.shape)}")
    a = t if t.dim() == 2 else _matrix(t, name)
    return a.data_ptr(), _rows(a, name, dev, dtype, shape, out)[2]


def _new(x, dtype=None):
    """A new contiguous tensor of ``x``'s shape."""
    if x.is_contiguous():
        return _empty_like(x, dtype=dtype)
    return x.new_empty(x.shape, dtype=dtype)


def _weight(t, dtype, D: int, dev: int) -> tuple[int, int]:
    """(address, type) of the norm's weight: of the rows' type, or float32."""
    own = isinstance(t, _Tensor) and t.dtype is dtype
    return _vector(t, "weight", dtype if own else _F32, D, dev), DTYPES[dtype] if own else 0


def _scales(t, shape, n: int, dev: int) -> int:
    """The address of the rows' scales, ``out[1]``, to overwrite."""
    if not isinstance(t, _Tensor) or t.shape != shape:
        raise ValueError(f"out[1] must be a tensor of the shape {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError("out[1] must be contiguous")
    return _vector(t.view(-1), "out[1]", _F32, n, dev)


def _norm(x, weight, eps, residual, out, sum_out, bits8):
    if _recording() and (x.requires_grad or (isinstance(weight, _Tensor) and weight.requires_grad)
                         or (isinstance(residual, _Tensor) and residual.requires_grad)):
        _cut_off("x", "weight", "residual")
    dev, dtype = x.get_device(), x.dtype
    a = x if x.dim() == 2 else _matrix(x, "x")
    N, D, ld = _rows(a, "x", dev)
    if D > _MAX_I32:  # the library would take what 32 bits hold of it
        _lib._check(_UNSUPPORTED)
    w, weight_type = _weight(weight, dtype, D, dev)
    r = (None, 0) if residual is None else _like(residual, "residual", x, dev, dtype, (N, D))
    written = []
    if bits8:
        if out is None:
            q, scale = _new(x, _I8), x.new_empty(x.shape[:-1], dtype=_F32)
            to, steps = (q.data_ptr(), D), scale.data_ptr()
        else:
            q, scale = out
            to = _like(q, "out[0]", x, dev, _I8, (N, D), True)
            steps = _scales(scale, x.shape[:-1], N, dev)
            written += out
        result = (q, scale)
    else:
        steps = None
        if out is None:
            out = _new(x)
            to = out.data_ptr(), D
        else:
            to = _like(out, "out", x, dev, dtype, (N, D), True)
            written.append(out)
        result = (out,)
    total = None, 0
    if sum_out is not None:
        total = _like(sum_out, "sum_out", x, dev, dtype, (N, D), True)
        written.append(sum_out)
    elif residual is not None:
        sum_out = _new(x)
        total = sum_out.data_ptr(), D
    if sum_out is not None:
        result = (*result, sum_out)
    if written and any(t.requires_grad for t in written):
        _cut_off("out", "sum_out")
    _run("lda_add_norm", dev, a.data_ptr(), ld, *r, w, *to, *total, steps, N, D, DTYPES[dtype],
         weight_type, _LDA_I8 if bits8 else DTYPES[dtype], eps)
    if written:
        _mark_written(written)
    return result if len(result) > 1 else result[0]


@_entry
def add_norm(x, weight, eps: float = 1e-6, residual=None, out=None, sum_out=None):
    """y = h * weight / sqrt(mean(h^2) + eps) by rows, h = x + residual
    (lda_add_norm).  x: a contiguous tensor of any shape (rows: its last dimension), or a
    matrix of contiguous rows; ``residual``: one of its shape and type; ``weight``
    [D] of its type or float32.  Returns y, or (y, h) where there is a residual or
    ``sum_out``.  ``out``, ``sum_out``: tensors to overwrite with y and h; each may be x or
    the residual.  ``stream``: where it runs (None: the current stream)."""
    return _norm(x, weight, eps, residual, out, sum_out, False)


@_entry
def add_norm_int8(x, weight, eps: float = 1e-6, residual=None, out=None, sum_out=None):
    """``add_norm`` with y in 8 bits: (q int8 of x's shape, scale float32 of x's shape
    without the last dimension), or (q, scale, h); q * scale stands for y, with the
    row's largest magnitude at 127.  ``out``: (q, scale) to overwrite."""
    return _norm(x, weight, eps, residual, out, sum_out, True)


@functools.lru_cache(maxsize=256)
def norm_grad_workspace_bytes(N: int, D: int) -> int:
    """Bytes of device workspace ``norm_grad`` needs (0: none, or unsupported)."""
    if D > _MAX_I32:
        return 0
    return int(_lib.load().lda_norm_grad_workspace_bytes(int(N), int(D)))


@_entry
def norm_grad(grad, h, weight, eps: float = 1e-6, residual_grad=None, out=None, weight_out=None,
              accumulate: bool = False, workspace=None) -> tuple[torch.Tensor, torch.Tensor]:
    """(dx, dweight float32 [D]): the gradients of ``add_norm`` from that of its output
    (lda_norm_grad).  ``h``: its second result, or its x where it had no residual;
    dx is the gradient of x and of the residual alike, ``residual_grad`` (what reaches h
    along the residual stream) added to it.  ``out``: a tensor to overwrite with dx (it may
    be grad, h or residual_grad); ``weight_out``: one for dweight, which ``accumulate`` adds
    to what it holds.  The result does not depend on the order in which the GPU works.
    ``workspace``: a uint8 tensor of at least ``norm_grad_workspace_bytes(N, D)`` bytes,
    or None to allocate one.  ``stream``: where it runs (None: the current stream)."""
    if _recording() and (grad.requires_grad or (isinstance(h, _Tensor) and h.requires_grad)
                         or (isinstance(weight, _Tensor) and weight.requires_grad)
                         or (isinstance(residual_grad, _Tensor) and residual_grad.requires_grad)):
        _cut_off("grad", "h", "weight", "residual_grad")
    dev, dtype = grad.get_device(), grad.dtype
    a = grad if grad.dim() == 2 else _matrix(grad, "grad")
    N, D, ld = _rows(a, "grad", dev)
    if D > _MAX_I32:  # the library would take what 32 bits hold of it
        _lib._check(_UNSUPPORTED)
    x = _like(h, "h", grad, dev, dtype, (N, D))
    w, weight_type = _weight(weight, dtype, D, dev)
    r = ((None, 0) if residual_grad is None
         else _like(residual_grad, "residual_grad", grad, dev, dtype, (N, D)))
    written = []
    if out is None:
        out = _new(grad)
        to = out.data_ptr(), D
    else:
        to = _like(out, "out", grad, dev, dtype, (N, D), True)
        written.append(out)
    if weight_out is None:
        if accumulate:
            raise ValueError("accumulate needs weight_out")
        weight_out = grad.new_empty(D, dtype=_F32)
        dw = weight_out.data_ptr()
    else:
        dw = _vector(weight_out, "weight_out", _F32, D, dev)
        written.append(weight_out)
    if written and any(t.requires_grad for t in written):
        _cut_off("out", "weight_out")
    need = norm_grad_workspace_bytes(N, D)
    if workspace is not None:
        _require(workspace, "workspace", _U8, 1)
        if workspace.get_device() != dev:
            raise ValueError("workspace must be on the tensors' device")
        need = workspace.numel()
    elif need:
        workspace = grad.new_empty(need, dtype=_U8)
    _run("lda_norm_grad", dev, a.data_ptr(), ld, *x, *r, w, *to, dw, N, D, DTYPES[dtype],
         weight_type, eps, 1 if accumulate else 0,
         None if workspace is None else workspace.data_ptr(), need)
    if written:
        _mark_written(written)
    return out, weight_out


@_entry
def quantise_rows(x, out=None) -> tuple[torch.Tensor, torch.Tensor]:
    """(q int8 of x's shape, scale float32 of x's shape without the last dimension): each
    row as whole numbers that stand for themselves times its scale, the row's largest
    magnitude at 127 (lda_quantise_rows).  x: a contiguous tensor of any shape, or a
    matrix of contiguous rows (activations, or a layer's weights [N][K]).  ``out``:
    (q, scale) to overwrite.  ``stream``: where it runs (None: the current stream)."""
    if x.requires_grad:
        _cut_off("x")
    dev = x.get_device()
    a = x if x.dim() == 2 else _matrix(x, "x")
    N, D, ld = _rows(a, "x", dev)
    if D > _MAX_I32:  # the library would take what 32 bits hold of it
        _lib._check(_UNSUPPORTED)
    if out is None:
        q, scale = _new(x, _I8), x.new_empty(x.shape[:-1], dtype=_F32)
        to, steps = (q.data_ptr(), D), scale.data_ptr()
    else:
        q, scale = out
        to = _like(q, "out[0]", x, dev, _I8, (N, D), True)
        steps = _scales(scale, x.shape[:-1], N, dev)
        if scale.requires_grad:
            _cut_off("out")
    _run("lda_quantise_rows", dev, a.data_ptr(), ld, *to, steps, N, D, DTYPES[x.dtype])
    if out is not None:
        _mark_written((q, scale))
    return q, scale


@_entry
def project_int8(q, scale, weight, weight_scale, bias=None, dtype=None,
                 out=None) -> torch.Tensor:
    """out[m][n] = (sum over k of q[m][k] * weight[n][k]) * scale[m] * weight_scale[n]
    + bias[n] (lda_project_int8): rows and weights as ``quantise_rows`` and
    ``add_norm_int8`` give them.  q int8 [M][K] (or a contiguous tensor of any shape) with
    ``scale`` float32 of its shape without the last dimension (a vector is contiguous; of
    more dimensions one that is not is copied); weight int8 [N][K], weight_scale float32 [N],
    bias float32 [N].  ``out``, or a new tensor of type ``dtype`` (None: bfloat16).
    ``stream``: where it runs (None: the current stream)."""
    dev = q.get_device()
    a = q if q.dim() == 2 else _matrix(q, "q")
    M, K, ldq = _rows(a, "q", dev, _I8)
    N, width, ldw = _rows(weight, "weight", dev, _I8)
    if width != K:
        raise ValueError(f"weight must have {K} columns, as q has, got {width}")
    if N > _MAX_I32 or K > MAX_PRODUCT_K:
        _lib._check(_UNSUPPORTED)
    if not isinstance(scale, _Tensor) or scale.shape != q.shape[:-1]:
        raise ValueError(f"scale must be a tensor of the shape {tuple(q.shape[:-1])}")
    # (one of several dimensions may be a copy here, which has to live until the launch)
    steps = scale if scale.dim() == 1 else scale.contiguous().view(-1)
    s = _vector(steps, "scale", _F32, M, dev)
    ws = _vector(weight_scale, "weight_scale", _F32, N, dev)
    b = None if bias is None else _vector(bias, "bias", _F32, N, dev)
    if _recording() and (scale.requires_grad or weight_scale.requires_grad
                         or (bias is not None and bias.requires_grad)):
        _cut_off("scale", "weight_scale", "bias")
    given = out is not None
    if not given:
        dtype = torch.bfloat16 if dtype is None else dtype
        if dtype not in DTYPES:
            raise TypeError("dtype must be float32, bfloat16 or float16")
        out = q.new_empty((*q.shape[:-1], N), dtype=dtype)
        to = out.data_ptr(), N
    else:
        if not isinstance(out, _Tensor) or out.shape != (*q.shape[:-1], N):
            raise ValueError(f"out must be a tensor of the shape {(*q.shape[:-1], N)}")
        if dtype not in (None, out.dtype):
            raise TypeError("dtype must be out's own")
        dtype = out.dtype
        o = out if out.dim() == 2 else _matrix(out, "out")
        to = o.data_ptr(), _rows(o, "out", dev, None, (M, N), True)[2]
        if out.requires_grad:
            _cut_off("out")
    _run("lda_project_int8", dev, a.data_ptr(), ldq, s, weight.data_ptr(), ldw, ws, b, *to, M, N,
         K, DTYPES[dtype])
    if given:
        _mark_written(out)
    return out


@_entry
def sample_logits(logits, u, temperature=None, top_k=None, top_p=None, min_p=None,
                  out=None) -> tuple[torch.Tensor, torch.Tensor]:
    """(z int32 [B], prob float32 [B]): one token of each row of ``logits`` [B][V] by the
    row's uniform number ``u`` float32 [B], and its share of the probability that the
    rules leave (lda_sample_logits).  ``temperature`` float32 [B]: where it is not above 0
    the row takes its largest logit.  Of the tokens in the order of falling logits stay
    the first ``top_k`` int32 [B], of those the fewest that reach the share ``top_p``
    float32 [B], of those the ones of at least ``min_p`` float32 [B] times the likeliest
    token's probability; z is then the first, by number, up to which the shares sum to more
    than u.  Penalties, biases and masks come before (``penalise_logits``).  A row with
    nothing to choose gives z = -1 and prob = 0; neither has a gradient.  ``out``:
    (z, prob) to overwrite.  ``stream``: where it runs (None: the current stream)."""
    dev = logits.get_device()
    B, V, ld = _rows(logits, "logits", dev)
    if V > _MAX_I32:
        _lib._check(_UNSUPPORTED)
    numbers = _vector(u, "u", _F32, B, dev)
    heat = None if temperature is None else _vector(temperature, "temperature", _F32, B, dev)
    k = None if top_k is None else _vector(top_k, "top_k", _I32, B, dev)
    p = None if top_p is None else _vector(top_p, "top_p", _F32, B, dev)
    floor = None if min_p is None else _vector(min_p, "min_p", _F32, B, dev)
    given = out is not None
    if not given:
        z, prob = logits.new_empty(B, dtype=_I32), logits.new_empty(B, dtype=_F32)
        to = z.data_ptr(), prob.data_ptr()
    else:
        z, prob = out
        to = _vector(z, "out[0]", _I32, B, dev), _vector(prob, "out[1]", _F32, B, dev)
        if prob.requires_grad:
            _cut_off("out")
    _run("lda_sample_logits", dev, logits.data_ptr(), ld, B, V, DTYPES[logits.dtype], numbers, heat,
         k, p, floor, *to)
    if given:
        _mark_written((z, prob))
    return z, prob
