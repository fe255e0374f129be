"""Binding of the operators around a language model's tokens (the second half
of lda_draw.h): the embedding and its gradient, dropout, the rules on logits
and the token draw.  Argument marshalling only, as in ``_lib``.

Matrices are 2-D tensors whose rows are contiguous; the rows themselves may lie
at any distance (a slice of a wider buffer, an expanded row).  Tensors that a
call allocates belong to the stream it runs on.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from . import _lib
from ._lib import _handle, _require

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}  # LDA_F32, LDA_BF16, LDA_F16
_I32, _I64, _F32 = torch.int32, torch.int64, torch.float32
_U64, _U32 = 2 ** 64 - 1, 2 ** 32 - 1


class LogitRules(ctypes.Structure):
    """struct lda_logit_rules."""
    _fields_ = [("history", ctypes.c_void_p), ("ld_history", ctypes.c_int64),
                ("capacity", ctypes.c_int64), ("lengths", ctypes.c_void_p),
                ("prompt", ctypes.c_void_p), ("repetition", ctypes.c_void_p),
                ("frequency", ctypes.c_void_p), ("presence", ctypes.c_void_p),
                ("bias", ctypes.c_void_p), ("ld_bias", ctypes.c_int64),
                ("mask", ctypes.c_void_p), ("ld_mask", ctypes.c_int64)]


def bind(lib: ctypes.CDLL) -> None:
    """Argument types of the entry points (called when the library is loaded)."""
    P, I32, I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    F64, U64, U32, SZ = ctypes.c_double, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_size_t
    rules = ctypes.POINTER(LogitRules)
    for name, args in (
            ("lda_embed", [P, I64, P, P, I64, I64, I32, I32, I32, F64, F64, U64, U32, P]),
            ("lda_dropout", [P, I64, P, I64, I64, I64, I32, F64, U64, U32, P]),
            ("lda_embed_grad", [P, I64, P, P, I64, I64, I32, I32, I32, I32, F64, F64, U64, U32,
                                I32, P, SZ, P]),
            ("lda_penalise_logits", [P, I64, P, I64, I64, I32, I32, rules, P]),
            ("lda_draw_logits", [P, I64, I64, I32, I32, rules, P, P, P, P, P, P, P, SZ, P])):
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = ctypes.c_int
    lib.lda_embed_grad_workspace_bytes.argtypes = [I64, I32, I32]
    lib.lda_embed_grad_workspace_bytes.restype = SZ
    lib.lda_draw_logits_workspace_bytes.argtypes = [I64, I32]
    lib.lda_draw_logits_workspace_bytes.restype = SZ


def _ld(t: torch.Tensor) -> int:
    """Elements from row to row (the width where there is one row or none)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _rows(t, name: str, dev=None, dtype=None, shape=None, out: bool = False) -> None:
    """A matrix whose rows are contiguous, of a supported type, on ``dev``."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    if dev is not None and t.device != dev:
        raise ValueError("all tensors must be on one device")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if dtype is None and t.dtype not in DTYPES:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{name} must have 2 dimensions")
    if shape is not None and tuple(t.shape) != shape:
        raise ValueError(f"{name} must have the shape {shape}, got {tuple(t.shape)}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")
    if out and t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        raise ValueError(f"{name}'s rows overlap")


def _vector(t, name: str, dtype, n: int, dev) -> None:
    _require(t, name, dtype, 1)
    if t.shape[0] != n or t.device != dev:
        raise ValueError(f"{name} must hold {n} entries on the tensors' device")


def _probability(p) -> float:
    p = float(p)
    if not 0.0 <= p < 1.0:
        raise ValueError("p must be in [0, 1)")
    return p


def _on(dev, stream):
    """The context in which a call allocates and launches: its device, and the
    stream it was given (so that what it allocates belongs to that stream)."""
    if stream is not None:
        return torch.cuda.stream(stream)
    if dev.index == torch.cuda.current_device():
        return contextlib.nullcontext()
    return torch.cuda.device(dev)


def _run(name: str, dev, stream, *args) -> None:
    st = getattr(_lib.load(), name)(*args, _handle(stream, dev.index))
    if st != 0:
        _lib._check(st)


def embed(table, word_id, scale: float = 1.0, p: float = 0.0, seed: int = 0, step: int = 0,
          out=None, stream=None) -> torch.Tensor:
    """out[n] = table[word_id[n]] * scale, dropped out with probability ``p``
    (lda_embed).  table [V][D] float32, bfloat16 or float16; word_id int32 [N];
    out [N][D] of the table's type.  A word outside [0, V) gives a row of zeros."""
    _rows(table, "table")
    dev = table.device
    _require(word_id, "word_id", _I32, 1)
    if word_id.device != dev:
        raise ValueError("all tensors must be on one device")
    (V, D), N = table.shape, word_id.shape[0]
    p = _probability(p)
    with _on(dev, stream):
        if out is None:
            out = torch.empty((N, D), dtype=table.dtype, device=dev)
        else:
            _rows(out, "out", dev, table.dtype, (N, D), out=True)
        _run("lda_embed", dev, stream, table.data_ptr(), _ld(table), word_id.data_ptr(),
             out.data_ptr(), _ld(out), N, V, D, DTYPES[table.dtype], float(scale), p,
             int(seed) & _U64, int(step) & _U32)
    return out


def embed_grad_workspace_bytes(N: int, V: int, D: int) -> int:
    """Bytes of device workspace ``embed_grad`` needs (0: none, or unsupported)."""
    return int(_lib.load().lda_embed_grad_workspace_bytes(int(N), int(V), int(D)))


def embed_grad(grad, word_id, V: int, scale: float = 1.0, p: float = 0.0, seed: int = 0,
               step: int = 0, out=None, accumulate: bool = False, dtype=None, workspace=None,
               stream=None) -> torch.Tensor:
    """The gradient of ``embed``'s table, [V][D]: the sum over each word's
    tokens of ``grad`` [N][D] (lda_embed_grad), for the same scale, p, seed and
    step.  ``out`` (or a new tensor of type ``dtype``): the gradient's type or
    float32; with ``accumulate`` the sums are added to it and rows without
    tokens are not touched.  The result does not depend on the order in which
    the GPU works.  ``workspace``: a uint8 tensor of at least
    ``embed_grad_workspace_bytes(N, V, D)`` bytes, or None to allocate one."""
    _rows(grad, "grad")
    dev = grad.device
    _require(word_id, "word_id", _I32, 1)
    N, D = grad.shape
    V = int(V)
    if word_id.shape[0] != N:
        raise ValueError("grad and word_id lengths differ")
    if word_id.device != dev:
        raise ValueError("all tensors must be on one device")
    p = _probability(p)
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    with _on(dev, stream):
        if out is None:
            dtype = grad.dtype if dtype is None else dtype
            if dtype not in (_F32, grad.dtype):
                raise TypeError("dtype must be float32 or the gradient's")
            out = torch.empty((V, D), dtype=dtype, device=dev)
        else:
            _rows(out, "out", dev, None, (V, D), out=True)
            if out.dtype not in (_F32, grad.dtype) or dtype not in (None, out.dtype):
                raise TypeError("out must be float32 or the gradient's type, and dtype its own")
        need = embed_grad_workspace_bytes(N, V, D)
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        else:
            _require(workspace, "workspace", torch.uint8, 1)
            if workspace.device != dev:
                raise ValueError("workspace must be on the tensors' device")
        _run("lda_embed_grad", dev, stream, grad.data_ptr(), _ld(grad), word_id.data_ptr(),
             out.data_ptr(), _ld(out), N, V, D, DTYPES[grad.dtype], DTYPES[out.dtype],
             float(scale), p, int(seed) & _U64, int(step) & _U32, int(bool(accumulate)),
             workspace.data_ptr(), workspace.numel())
    return out


def dropout(x, p: float, seed: int, step: int = 0, out=None, stream=None) -> torch.Tensor:
    """``x`` with each element 0 with probability ``p`` and otherwise divided by
    the probability of keeping it (lda_dropout); given the gradient of that,
    the same call gives the gradient of ``x``.  x: a contiguous tensor of any
    shape (rows: its last dimension; a vector is one row), or a matrix of
    contiguous rows.  ``out`` may be ``x``."""
    if not isinstance(x, torch.Tensor):
        raise TypeError("x must be a torch.Tensor")
    if x.dim() == 0:
        raise ValueError("x must have at least 1 dimension")
    p = _probability(p)
    if x.dim() != 2 and not x.is_contiguous():
        raise ValueError("x must be contiguous")
    a = x if x.dim() == 2 else x.view(-1, x.shape[-1]) if x.numel() else x.reshape(0, 1)
    _rows(a, "x")
    dev = x.device
    with _on(dev, stream):
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=dev)
        elif not isinstance(out, torch.Tensor) or out.shape != x.shape:
            raise ValueError("out must be a tensor of x's shape")
        elif out.dim() != 2 and not out.is_contiguous():
            raise ValueError("out must be contiguous")
        b = out if out.dim() == 2 else out.view(a.shape)
        _rows(b, "out", dev, x.dtype, tuple(a.shape), out=True)
        if x.numel():
            _run("lda_dropout", dev, stream, a.data_ptr(), _ld(a), b.data_ptr(), _ld(b),
                 a.shape[0], a.shape[1], DTYPES[x.dtype], p, int(seed) & _U64, int(step) & _U32)
    return out


def _rules(logits, history, lengths, prompt, repetition, frequency, presence, bias, mask):
    """The rules as the library takes them, or None where there are none."""
    B, V = logits.shape
    dev = logits.device
    r = LogitRules()
    if history is not None:
        _rows(history, "history", dev, _I32)
        if history.shape[0] != B:
            raise ValueError("history must have a row for each row of logits")
        if lengths is None:
            raise ValueError("history needs lengths")
        if B > 1 and history.stride(0) < history.shape[1]:
            raise ValueError("history's rows overlap")
        r.history, r.ld_history, r.capacity = history.data_ptr(), _ld(history), history.shape[1]
        _vector(lengths, "lengths", _I32, B, dev)
        r.lengths = lengths.data_ptr()
        for t, name, dtype in ((prompt, "prompt", _I32), (repetition, "repetition", _F32),
                               (frequency, "frequency", _F32), (presence, "presence", _F32)):
            if t is not None:
                _vector(t, name, dtype, B, dev)
                setattr(r, name, t.data_ptr())
    elif not (lengths is prompt is repetition is frequency is presence is None):
        raise ValueError("lengths, prompt and penalties need history")
    for t, name, dtype, width in ((bias, "bias", _F32, V), (mask, "mask", _I32, (V + 31) // 32)):
        if t is None:
            continue
        if isinstance(t, torch.Tensor) and t.dim() == 1:  # one row for all
            _vector(t, name, dtype, width, dev)
            ld = 0
        else:
            _rows(t, name, dev, dtype, (B, width))
            ld = _ld(t)
            if 0 < ld < width:
                raise ValueError(f"{name}'s rows overlap")
        setattr(r, name, t.data_ptr())
        setattr(r, "ld_" + name, ld)
    if history is None and bias is None and mask is None:
        return None
    return ctypes.byref(r)


def penalise_logits(logits, history=None, lengths=None, prompt=None, repetition=None,
                    frequency=None, presence=None, bias=None, mask=None, out=None,
                    stream=None) -> torch.Tensor:
    """logits [B][V] under the rules (lda_penalise_logits): ``history`` int32
    [B][capacity] with ``lengths`` int32 [B], the first ``prompt`` [B] of them
    not generated; ``repetition``, ``frequency``, ``presence`` float32 [B];
    ``bias`` float32 [V] or [B][V]; ``mask`` int32 [V / 32] or [B][V / 32]
    (rounded up), bit 0 where a token is not allowed.  ``out`` may be
    ``logits``."""
    _rows(logits, "logits")
    rules = _rules(logits, history, lengths, prompt, repetition, frequency, presence, bias, mask)
    (B, V), dev = logits.shape, logits.device
    with _on(dev, stream):
        if out is None:
            out = torch.empty((B, V), dtype=logits.dtype, device=dev)
        else:
            _rows(out, "out", dev, logits.dtype, (B, V), out=True)
        _run("lda_penalise_logits", dev, stream, logits.data_ptr(), _ld(logits), out.data_ptr(),
             _ld(out), B, V, DTYPES[logits.dtype], rules)
    return out


def draw_logits_workspace_bytes(B: int, V: int) -> int:
    """Bytes of device workspace ``draw_logits`` needs (0: none, or unsupported)."""
    return int(_lib.load().lda_draw_logits_workspace_bytes(int(B), int(V)))


def draw_logits(logits, seed, position, temperature=None, min_p=None, history=None, lengths=None,
                prompt=None, repetition=None, frequency=None, presence=None, bias=None, mask=None,
                out=None, workspace=None, stream=None) -> tuple[torch.Tensor, torch.Tensor]:
    """(z int32 [B], prob float32 [B]): one token of each row of ``logits``
    [B][V] under ``penalise_logits``' rules, and the probability with which it
    was drawn (lda_draw_logits).  ``seed`` int64 [B] and ``position`` int32 [B]
    fix a row's random numbers, wherever it lies in the batch.  ``temperature``
    float32 [B]: where it is not above 0 the row takes its largest logit.
    ``min_p`` float32 [B]: tokens below that share of the likeliest token's
    probability are not drawn.  A row with nothing to draw gives z = -1 and
    prob = 0.  ``out``: (z, prob) to overwrite."""
    _rows(logits, "logits")
    rules = _rules(logits, history, lengths, prompt, repetition, frequency, presence, bias, mask)
    (B, V), dev = logits.shape, logits.device
    _vector(seed, "seed", _I64, B, dev)
    _vector(position, "position", _I32, B, dev)
    for t, name in ((temperature, "temperature"), (min_p, "min_p")):
        if t is not None:
            _vector(t, name, _F32, B, dev)
    with _on(dev, stream):
        if out is None:
            z = torch.empty(B, dtype=_I32, device=dev)
            prob = torch.empty(B, dtype=_F32, device=dev)
        else:
            z, prob = out
            _vector(z, "out[0]", _I32, B, dev)
            _vector(prob, "out[1]", _F32, B, dev)
        need = draw_logits_workspace_bytes(B, V)
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        else:
            _require(workspace, "workspace", torch.uint8, 1)
            if workspace.device != dev:
                raise ValueError("workspace must be on the tensors' device")
        _run("lda_draw_logits", dev, stream, logits.data_ptr(), _ld(logits), B, V,
             DTYPES[logits.dtype], rules, None if temperature is None else temperature.data_ptr(),
             None if min_p is None else min_p.data_ptr(), seed.data_ptr(), position.data_ptr(),
             z.data_ptr(), prob.data_ptr(), workspace.data_ptr(), workspace.numel())
    return z, prob
