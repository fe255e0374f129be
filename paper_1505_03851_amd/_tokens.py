"""Binding of the operators around a language model's tokens (the second half
of lda_draw.h): the embedding and its gradient, dropout, the rules on logits
and the token draw.  Argument marshalling only, as in ``_lib``.

Matrices are 2-D tensors whose rows are contiguous; the rows themselves may lie
at any distance (a slice of a wider buffer, an expanded row).  Tensors that a
call allocates belong to the stream it runs on.  A tensor that a call is given to
write into counts as changed in place: a backward pass that saved what it held
raises.  No call records a gradient: where gradients are recorded, one whose
result would have one (embed, embed_grad, dropout, penalise_logits) refuses
tensors that require it, and, recorded or not, forward-mode dual tensors.
``embed_grad`` and ``dropout`` are the backward passes, for a
torch.autograd.Function or a training loop to call.
"""
from __future__ import annotations

import ctypes
import functools

import torch
from torch.autograd import forward_ad as _forward

from . import _lib
from ._lib import _require

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}  # LDA_F32, LDA_BF16, LDA_F16
_I32, _I64, _F32, _U8 = torch.int32, torch.int64, torch.float32, torch.uint8
_U64, _U32 = 2 ** 64 - 1, 2 ** 32 - 1
_MAX_I32 = 2 ** 31 - 1
_UNSUPPORTED = _lib.STATUS["LDA_ERR_UNSUPPORTED"]
_Tensor = torch.Tensor
_current_device = _lib._current_device or torch.cuda.current_device
_mark_written = torch.autograd.graph.increment_version


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


# The checks below read each attribute once and in the order in which a call whose
# arguments are all as they should be passes soonest: a small call takes as long
# on the host as on the GPU.  What fails goes on to the checks that say why.


_DRAWN = ("draw_logits", "sample_logits")  # whose results have no gradient


def _no_tangents(fn, args, kw) -> None:
    """Refuses forward-mode dual tensors, whose tangents the result would not have."""
    names = fn.__code__.co_varnames
    for name, value in (*zip(names, args), *kw.items()):
        if fn.__name__ in _DRAWN and name != "out":
            continue
        for t in value if isinstance(value, (tuple, list)) else (value,):
            if isinstance(t, _Tensor) and _forward.unpack_dual(t).tangent is not None:
                raise ValueError(f"{name} has a tangent, which is not recorded here: call this with "
                                 "the tensor that unpack_dual gives")


def _entry(fn):
    """``fn`` in the context of its first tensor's device, and of the stream the
    call is given: what it allocates and launches belongs to that stream."""
    name = fn.__code__.co_varnames[0]

    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        if _forward._current_level >= 0:
            _no_tangents(fn, args, kw)
        first = args[0] if args else kw.get(name)
        if type(first) is _Tensor and stream is None:
            dev = first.get_device()
            if dev >= 0 and dev == _current_device():
                return fn(*args, **kw)
        if not isinstance(first, _Tensor):
            raise TypeError(f"{name} must be a torch.Tensor")
        if not first.is_cuda:
            raise ValueError(f"{name} must be on the GPU")
        if stream is not None and stream.device != first.device:
            raise ValueError("stream must be on the tensors' device")
        with torch.cuda.stream(stream) if stream is not None else torch.cuda.device(first.device):
            return fn(*args, **kw)
    return call


def _run(name: str, dev: int, *args) -> None:
    """One call of the library on the current stream of device ``dev``."""
    raw = _lib._raw_stream
    handle = raw(dev) if raw is not None else torch.cuda.current_stream(dev).cuda_stream
    st = getattr(_lib._lib or _lib.load(), name)(*args, handle)
    if st != 0:
        _lib._check(st)


def _rows(t, name: str, dev: int, dtype=None, shape=None, out: bool = False) -> tuple[int, int, int]:
    """(rows, width, elements from row to row) of a matrix whose rows are
    contiguous, of type ``dtype`` (None: a supported one), on device ``dev``."""
    if isinstance(t, _Tensor) and t.dim() == 2 and t.get_device() == dev and (
            t.dtype is dtype or (dtype is None and t.dtype in DTYPES)):
        n, width = t.shape
        apart, one = t.stride()
        if n <= 1:
            apart = width
        if ((one == 1 or width <= 1) and (shape is None or shape == (n, width))
                and (not out or apart >= width)):
            return n, width, apart
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    if t.get_device() != dev:
        raise ValueError("all tensors must be on one device")
    if t.dtype != dtype if dtype is not None else t.dtype not in DTYPES:
        raise TypeError(f"{name} must be {dtype or 'float32, bfloat16 or float16'}, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{name} must have 2 dimensions")
    if shape is not None and tuple(t.shape) != shape:
        raise ValueError(f"{name} must have the shape {shape}, got {tuple(t.shape)}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")
    raise ValueError(f"{name}'s rows overlap")


def _vector(t, name: str, dtype, n: int, dev: int) -> int:
    """The address of a dense vector of ``n`` entries on device ``dev``."""
    if not (isinstance(t, _Tensor) and t.dtype is dtype and t.dim() == 1 and t.numel() == n
            and t.get_device() == dev and t.is_contiguous()):
        _require(t, name, dtype, 1)
        raise ValueError(f"{name} must hold {n} entries on the tensors' device")
    return t.data_ptr()


def _cut_off(*names: str) -> None:
    """Refuses tensors that require a gradient (some of ``names``), where those are
    recorded."""
    if torch.is_grad_enabled():
        raise ValueError(f"{' or '.join(names)} requires a gradient, which is not recorded here: "
                         "call this under torch.no_grad(), or with a detached tensor")


def _probability(p) -> float:
    p = float(p)
    if not 0.0 <= p < 1.0:
        raise ValueError("p must be in [0, 1)")
    return p


@_entry
def embed(table, word_id, scale: float = 1.0, p: float = 0.0, seed: int = 0, step: int = 0,
          out=None) -> torch.Tensor:
    """out[n] = table[word_id[n]] * scale, dropped out with probability ``p``
    (lda_embed).  table [V][D] float32, bfloat16 or float16; word_id int32 [N];
    out [N][D] of the table's type.  A word outside [0, V) gives a row of zeros.
    ``stream``: where it runs (None: the current stream)."""
    if table.requires_grad:
        _cut_off("table")
    dev = table.get_device()
    V, D, ld = _rows(table, "table", dev)
    if V > _MAX_I32 or D > _MAX_I32:  # the library would take what 32 bits hold of it
        _lib._check(_UNSUPPORTED)
    N = word_id.numel() if isinstance(word_id, _Tensor) else -1
    ids = _vector(word_id, "word_id", _I32, N, dev)
    dtype = table.dtype
    given = out is not None
    if not given:
        out, ldo = table.new_empty((N, D)), D
    else:
        ldo = _rows(out, "out", dev, dtype, (N, D), True)[2]
        if out.requires_grad:
            _cut_off("out")
    _run("lda_embed", dev, table.data_ptr(), ld, ids, out.data_ptr(), ldo, N, V, D, DTYPES[dtype],
         scale, _probability(p), int(seed) & _U64, int(step) & _U32)
    if given:
        _mark_written(out)
    return out


@functools.lru_cache(maxsize=256)
def embed_grad_workspace_bytes(N: int, V: int, D: int) -> int:
    """Bytes of device workspace ``embed_grad`` needs (0: none, or unsupported)."""
    if max(V, D) > _MAX_I32:
        return 0
    return int(_lib.load().lda_embed_grad_workspace_bytes(int(N), int(V), int(D)))


@_entry
def embed_grad(grad, word_id, V: int, scale: float = 1.0, p: float = 0.0, seed: int = 0,
               step: int = 0, out=None, accumulate: bool = False, dtype=None,
               workspace=None) -> torch.Tensor:
    """The gradient of ``embed``'s table, [V][D]: the sum over each word's
    tokens of ``grad`` [N][D] (lda_embed_grad), for the same scale, p, seed and
    step.  ``out`` (or a new tensor of type ``dtype``): the gradient's type or
    float32; with ``accumulate`` the sums are added to it and rows without
    tokens are not touched.  The result does not depend on the order in which
    the GPU works.  ``workspace``: a uint8 tensor of at least
    ``embed_grad_workspace_bytes(N, V, D)`` bytes, or None to allocate one.
    ``stream``: where it runs (None: the current stream)."""
    if grad.requires_grad:
        _cut_off("grad")
    dev = grad.get_device()
    N, D, ld = _rows(grad, "grad", dev)
    ids = _vector(word_id, "word_id", _I32, N, dev)
    V, own = int(V), grad.dtype
    if V > _MAX_I32 or D > _MAX_I32:  # the library would take what 32 bits hold of it
        _lib._check(_UNSUPPORTED)
    given = out is not None
    if not given:
        if accumulate:
            raise ValueError("accumulate needs out")
        if dtype is not None and dtype not in (_F32, own):
            raise TypeError("dtype must be float32 or the gradient's")
        out, ldo = grad.new_empty((V, D), dtype=dtype or own), D
    else:
        ldo = _rows(out, "out", dev, None, (V, D), True)[2]
        if out.requires_grad:
            _cut_off("out")
        if out.dtype not in (_F32, own) or dtype not in (None, out.dtype):
            raise TypeError("out must be float32 or the gradient's type, and dtype its own")
    need = embed_grad_workspace_bytes(N, V, D)
    if workspace is not None:
        _require(workspace, "workspace", _U8, 1)
        if workspace.get_device() != dev:
            raise ValueError("workspace must be on the tensors' device")
        need = workspace.numel()
    elif need:
        workspace = grad.new_empty(need, dtype=_U8)
    _run("lda_embed_grad", dev, grad.data_ptr(), ld, ids, out.data_ptr(), ldo, N, V, D, DTYPES[own],
         DTYPES[out.dtype], scale, _probability(p), int(seed) & _U64, int(step) & _U32,
         1 if accumulate else 0, None if workspace is None else workspace.data_ptr(), need)
    if given:
        _mark_written(out)
    return out


def _as_rows(t, name: str):
    """A contiguous tensor as the matrix of its last dimension's rows (a vector:
    one row); a matrix as it is."""
    if t.dim() == 2:
        return t
    if t.dim() == 0:
        raise ValueError(f"{name} must have at least 1 dimension")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.view(-1, t.shape[-1]) if t.numel() else t.reshape(0, 1)


@_entry
def dropout(x, p: float, seed: int, step: int = 0, out=None) -> torch.Tensor:
    """``x`` with each element 0 with probability ``p`` and otherwise divided by
    the probability of keeping it (lda_dropout); given the gradient of that,
    the same call gives the gradient of ``x``.  x: a contiguous tensor of any
    shape (rows: its last dimension; a vector is one row), or a matrix of
    contiguous rows.  ``out`` may be ``x``.  ``stream``: where it runs (None: the
    current stream)."""
    if x.requires_grad:
        _cut_off("x")
    dev = x.get_device()
    a = _as_rows(x, "x")
    rows, cols, ld = _rows(a, "x", dev)
    p = _probability(p)
    given = out is not None
    if not given:
        out = x.new_empty(x.shape)
        ldo = cols
    else:
        if not isinstance(out, _Tensor) or out.shape != x.shape:
            raise ValueError("out must be a tensor of x's shape")
        if out.requires_grad:
            _cut_off("out")
        ldo = _rows(_as_rows(out, "out"), "out", dev, x.dtype, (rows, cols), True)[2]
    if rows and cols:
        _run("lda_dropout", dev, x.data_ptr(), ld, out.data_ptr(), ldo, rows, cols, DTYPES[x.dtype],
             p, int(seed) & _U64, int(step) & _U32)
    if given:
        _mark_written(out)
    return out


def _rules(dev, B, V, history, lengths, prompt, repetition, frequency, presence, bias, mask):
    """The rules as the library takes them, or None where there are none."""
    past = (None, 0, 0, None, None, None, None, None)
    if history is not None:
        n, capacity, apart = _rows(history, "history", dev, _I32)
        if n != B:
            raise ValueError("history must have a row for each row of logits")
        if lengths is None:
            raise ValueError("history needs lengths")
        if 0 < apart < capacity:
            raise ValueError("history's rows overlap")
        past = (history.data_ptr(), apart, capacity, _vector(lengths, "lengths", _I32, B, dev),
                None if prompt is None else _vector(prompt, "prompt", _I32, B, dev),
                None if repetition is None else _vector(repetition, "repetition", _F32, B, dev),
                None if frequency is None else _vector(frequency, "frequency", _F32, B, dev),
                None if presence is None else _vector(presence, "presence", _F32, B, dev))
    elif not (lengths is prompt is repetition is frequency is presence is None):
        raise ValueError("lengths, prompt and penalties need history")
    elif bias is None and mask is None:
        return None
    return ctypes.byref(LogitRules(*past, *_row_or_rows(bias, "bias", _F32, B, V, dev),
                                   *_row_or_rows(mask, "mask", _I32, B, (V + 31) // 32, dev)))


def _row_or_rows(t, name, dtype, B, width, dev):
    """(address, elements from row to row), 0 where one row serves all."""
    if t is None:
        return None, 0
    if isinstance(t, _Tensor) and t.dim() == 1:
        return _vector(t, name, dtype, width, dev), 0
    apart = _rows(t, name, dev, dtype, (B, width))[2]
    if 0 < apart < width:
        raise ValueError(f"{name}'s rows overlap")
    return t.data_ptr(), apart


@_entry
def penalise_logits(logits, history=None, lengths=None, prompt=None, repetition=None,
                    frequency=None, presence=None, bias=None, mask=None,
                    out=None) -> torch.Tensor:
    """logits [B][V] under the rules (lda_penalise_logits): ``history`` int32
    [B][capacity] with ``lengths`` int32 [B], the first ``prompt`` [B] of them
    not generated; ``repetition``, ``frequency``, ``presence`` float32 [B];
    ``bias`` float32 [V] or [B][V]; ``mask`` int32 [V / 32] or [B][V / 32]
    (rounded up), bit 0 where a token is not allowed.  ``out`` may be
    ``logits``.  ``stream``: where it runs (None: the current stream)."""
    dev = logits.get_device()
    B, V, ld = _rows(logits, "logits", dev)
    if V > _MAX_I32:
        _lib._check(_UNSUPPORTED)
    rules = _rules(dev, B, V, history, lengths, prompt, repetition, frequency, presence, bias, mask)
    if (logits.requires_grad or (bias is not None and bias.requires_grad)
            or (repetition is not None and repetition.requires_grad)
            or (frequency is not None and frequency.requires_grad)
            or (presence is not None and presence.requires_grad)):
        _cut_off("logits", "a rule")
    given = out is not None
    if not given:
        out, ldo = logits.new_empty((B, V)), V
    else:
        ldo = _rows(out, "out", dev, logits.dtype, (B, V), True)[2]
        if out.requires_grad:
            _cut_off("out")
    _run("lda_penalise_logits", dev, logits.data_ptr(), ld, out.data_ptr(), ldo, B, V,
         DTYPES[logits.dtype], rules)
    if given:
        _mark_written(out)
    return out


@functools.lru_cache(maxsize=256)
def draw_logits_workspace_bytes(B: int, V: int) -> int:
    """Bytes of device workspace ``draw_logits`` needs (0: none, or unsupported)."""
    if V > _MAX_I32:
        return 0
    return int(_lib.load().lda_draw_logits_workspace_bytes(int(B), int(V)))


@_entry
def draw_logits(logits, seed, position, temperature=None, min_p=None, history=None, lengths=None,
                prompt=None, repetition=None, frequency=None, presence=None, bias=None, mask=None,
                out=None, workspace=None) -> tuple[torch.Tensor, torch.Tensor]:
    """(z int32 [B], prob float32 [B]): one token of each row of ``logits``
    [B][V] under ``penalise_logits``' rules, and the probability with which it
    was drawn (lda_draw_logits).  ``seed`` int64 [B] and ``position`` int32 [B]
    fix a row's random numbers, wherever it lies in the batch.  ``temperature``
    float32 [B]: where it is not above 0 the row takes its largest logit.
    ``min_p`` float32 [B]: tokens below that share of the likeliest token's
    probability are not drawn.  A row with nothing to draw gives z = -1 and
    prob = 0; neither has a gradient.  ``out``: (z, prob) to overwrite.
    ``workspace``: a uint8 tensor of at least ``draw_logits_workspace_bytes(B, V)``
    bytes, or None to allocate one.  ``stream``: where it runs (None: the current
    stream)."""
    dev = logits.get_device()
    B, V, ld = _rows(logits, "logits", dev)
    if V > _MAX_I32:
        _lib._check(_UNSUPPORTED)
    rules = _rules(dev, B, V, history, lengths, prompt, repetition, frequency, presence, bias, mask)
    seeds = _vector(seed, "seed", _I64, B, dev)
    places = _vector(position, "position", _I32, B, dev)
    heat = None if temperature is None else _vector(temperature, "temperature", _F32, B, dev)
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
    need = draw_logits_workspace_bytes(B, V)
    if workspace is not None:
        _require(workspace, "workspace", _U8, 1)
        if workspace.get_device() != dev:
            raise ValueError("workspace must be on the tensors' device")
        need = workspace.numel()
    elif need:
        workspace = logits.new_empty(need, dtype=_U8)
    _run("lda_draw_logits", dev, logits.data_ptr(), ld, B, V, DTYPES[logits.dtype], rules, heat,
         floor, seeds, places, *to, None if workspace is None else workspace.data_ptr(), need)
    if given:
        _mark_written((z, prob))
    return z, prob
