"""Thin Python binding of include/deft_ends.h (argument marshalling only): the token embedding,
the head with its softmax cross entropy, and distillation from a teacher's top logits.

Every step runs in the HIP library; PyTorch supplies device memory and streams.  There is no CPU
fallback.  Arguments that the kernels do not take as they are (another type, device or shape,
elements of a row apart) are refused with ValueError; nothing is copied or converted silently.
"""
from __future__ import annotations

import ctypes
import functools
from typing import Iterable, Optional, Sequence

import torch

from . import binding
from .binding import DEFT_OK, DeftError

DEFT_F32, DEFT_F16, DEFT_BF16 = range(3)
DTYPES = {torch.float32: DEFT_F32, torch.float16: DEFT_F16, torch.bfloat16: DEFT_BF16}
OPERATORS = {"embed": 1, "embed_grad": 2, "head_loss": 4, "head_grad": 8, "distill": 16}
EXPORTS = ("deft_ends_create", "deft_ends_destroy", "deft_ends_get_info", "deft_embed", "deft_embed_grad",
           "deft_head_loss", "deft_head_grad", "deft_distill")

_MOST = 2 ** 31 - 1   # of a 32-bit field (ctypes cuts what is larger without a word)

_i32, _i64, _f32, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p


class deft_ends_config_t(ctypes.Structure):
    _fields_ = [("device", _i32), ("dtype", _i32), ("operators", ctypes.c_uint32), ("max_rows", _i32),
                ("max_vocab", _i32), ("max_hidden", _i32), ("max_top_k", _i32)]


class deft_ends_info_t(ctypes.Structure):
    _fields_ = [("scratch_bytes", _i64), ("vocab_piece", _i32), ("compute_units", _i32)]


class deft_embed_t(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("vocab", _i32), ("hidden", _i32), ("scale", _f32), ("tokens", _vp), ("table", _vp),
                ("table_stride", _i64), ("out", _vp), ("out_stride", _i64), ("status", _vp), ("stream", _vp)]


class deft_embed_grad_t(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("vocab", _i32), ("hidden", _i32), ("scale", _f32), ("accumulate", _i32),
                ("tokens", _vp), ("grad_out", _vp), ("grad_out_stride", _i64), ("grad_table", _vp),
                ("grad_table_stride", _i64), ("stream", _vp)]


class deft_head_loss_t(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("vocab", _i32), ("hidden", _i32), ("logit_scale", _f32), ("hidden_states", _vp),
                ("hidden_stride", _i64), ("weight", _vp), ("weight_stride", _i64), ("labels", _vp), ("loss", _vp),
                ("lse", _vp), ("status", _vp), ("stream", _vp)]


class deft_head_grad_t(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("vocab", _i32), ("hidden", _i32), ("logit_scale", _f32), ("accumulate", _i32),
                ("n_piece_events", _i32), ("hidden_states", _vp), ("hidden_stride", _i64), ("weight", _vp),
                ("weight_stride", _i64), ("labels", _vp), ("lse", _vp), ("row_grad", _vp), ("grad_hidden", _vp),
                ("grad_hidden_stride", _i64), ("grad_weight", _vp), ("grad_weight_stride", _i64), ("piece_events", _vp),
                ("stream", _vp)]


class deft_distill_t(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("vocab", _i32), ("top_k", _i32), ("temperature", _f32), ("logits", _vp),
                ("logits_stride", _i64), ("teacher_index", _vp), ("teacher_logit", _vp), ("row_grad", _vp),
                ("loss", _vp), ("grad_logits", _vp), ("grad_stride", _i64), ("status", _vp), ("stream", _vp)]


_declared = False


def load_library() -> ctypes.CDLL:
    global _declared
    lib = binding.load_library()
    if not _declared:
        for name, args in (("deft_ends_create", [ctypes.POINTER(deft_ends_config_t), ctypes.POINTER(_vp)]),
                           ("deft_ends_get_info", [_vp, ctypes.POINTER(deft_ends_info_t)]),
                           ("deft_embed", [_vp, ctypes.POINTER(deft_embed_t)]),
                           ("deft_embed_grad", [_vp, ctypes.POINTER(deft_embed_grad_t)]),
                           ("deft_head_loss", [_vp, ctypes.POINTER(deft_head_loss_t)]),
                           ("deft_head_grad", [_vp, ctypes.POINTER(deft_head_grad_t)]),
                           ("deft_distill", [_vp, ctypes.POINTER(deft_distill_t)])):
            getattr(lib, name).restype = ctypes.c_int
            getattr(lib, name).argtypes = args
        lib.deft_ends_destroy.restype = None
        lib.deft_ends_destroy.argtypes = [_vp]
        _declared = True
    return lib


def _on_stream(method):
    """Adds the `stream` argument: what the call allocates belongs to that stream, and its tensors are recorded there."""
    @functools.wraps(method)
    def call(self, *args, stream: Optional[torch.cuda.Stream] = None, **kwargs):
        if stream is None:
            return method(self, *args, **kwargs)
        if stream.device_index != self._index:   # (its device's current stream would be taken instead)
            raise ValueError(f"stream: one of {self.device} is wanted, got one of device {stream.device_index}")
        with torch.cuda.stream(stream):
            out = method(self, *args, **kwargs)
        _record((*args, *kwargs.values()), stream)
        return out
    return call


def _record(values, stream):
    for t in values:
        if isinstance(t, torch.Tensor):
            t.record_stream(stream)
        elif isinstance(t, tuple):
            _record(t, stream)


class Marshalling:
    """What the owners of handles share: `with`, calls and their errors, checks of tensors."""

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _call(self, name: str, arg) -> None:
        if not self._h:
            raise ValueError("the handle is closed")
        rc = getattr(self._lib, name)(self._h, arg)
        if rc != DEFT_OK:
            raise DeftError(name, rc)

    def _rows(self, name, t, rows, width):
        """Checks a matrix of the handle's type whose rows lie apart as they like; gives its shape."""
        return self._matrix(name, t, self.dtype, rows, width)

    def _matrix(self, name, t, dtype, rows, width):
        if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.dtype != dtype or t.get_device() != self._index:
            raise ValueError(f"{name}: a matrix of {dtype} on {self.device} is wanted")
        n, w = shape = t.shape
        if n > _MOST or w > _MOST:
            raise ValueError(f"{name}: sizes of 32 bits are wanted, got {(n, w)}")
        if (rows is not None and n != rows) or (width is not None and w != width):
            raise ValueError(f"{name}: shape {(n, w)} does not fit {(rows, width)}")
        if not t.is_contiguous() and ((w > 1 and t.stride(1) != 1) or (n > 1 and t.stride(0) < w)):
            raise ValueError(f"{name}: a row's elements have to be next to each other, rows apart")
        return shape

    def _words(self, name, t, dtype, shape):
        if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.get_device() != self._index or not t.is_contiguous():
            raise ValueError(f"{name}: a contiguous tensor of {dtype} on {self.device} is wanted")
        got = t.shape
        if len(got) != len(shape) or any(g > _MOST or (s is not None and s != g) for s, g in zip(shape, got)):
            raise ValueError(f"{name}: shape {tuple(got)} does not fit {shape}")
        return got

    def _stream(self) -> int:
        return torch._C._cuda_getCurrentRawStream(self._index)


class DeftEnds(Marshalling):
    """Owner of one deft_ends_t handle.

    `operators` names what the handle serves (keys of OPERATORS): it holds no scratch memory for
    others.  Outputs are allocated unless given; calls run on `stream` (default: torch's current
    stream) and return without waiting.  Tensors of a call on another stream than their own are
    recorded there.  The scratch memory is one call's at a time: a handle's calls go to one stream, or
    the next stream waits for the one before; work on two streams at once takes two handles.  Tokens,
    labels and indices are int32, -1 for nothing.

    Gradients are the *_grad calls' results.  torch's automatic differentiation does not see any of these
    calls: what they give carries no graph, also of inputs that require a gradient, and what they
    write into (out, grad_table, grad_weight, grad_logits) is not marked as changed.
    """

    def __init__(self, operators: Iterable[str], dtype: torch.dtype, max_rows: int, max_vocab: int, max_hidden: int = 0,
                 max_top_k: int = 0, device: int = 0):
        self._h = _vp()
        self._lib = load_library()
        if dtype not in DTYPES:
            raise ValueError(f"dtype is one of {list(DTYPES)}: got {dtype}")
        for name, value in (("max_rows", max_rows), ("max_vocab", max_vocab), ("max_hidden", max_hidden),
                            ("max_top_k", max_top_k), ("device", device)):
            if not -_MOST <= value <= _MOST:
                raise ValueError(f"{name} does not fit 32 bits: got {value}")
        mask = 0
        for name in ((operators,) if isinstance(operators, str) else operators):
            if name not in OPERATORS:
                raise ValueError(f"operators are {list(OPERATORS)}: got {name!r}")
            mask |= OPERATORS[name]
        self.dtype, self.device, self._index = dtype, torch.device("cuda", device), device
        cfg = deft_ends_config_t(device, DTYPES[dtype], mask, max_rows, max_vocab, max_hidden, max_top_k)
        rc = self._lib.deft_ends_create(ctypes.byref(cfg), ctypes.byref(self._h))
        if rc != DEFT_OK:
            self._h = _vp()
            raise DeftError("deft_ends_create", rc)

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h:
            self._lib.deft_ends_destroy(self._h)
            self._h = None   # (at the interpreter's end the module's names are gone)

    __del__ = close

    def info(self) -> deft_ends_info_t:
        info = deft_ends_info_t()
        self._call("deft_ends_get_info", ctypes.byref(info))
        return info

    # ---- the operators ----------------------------------------------------------------------

    @_on_stream
    def embed(self, tokens: torch.Tensor, table: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
              status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """out[n] = scale * table[tokens[n]]."""
        vocab, hidden = self._rows("table", table, None, None)
        n = self._words("tokens", tokens, torch.int32, (None,))[0]
        if out is None:
            out = torch.empty((n, hidden), dtype=self.dtype, device=self.device)
        self._rows("out", out, n, hidden)
        if status is not None:
            self._words("status", status, torch.int32, (n,))
        self._call("deft_embed", ctypes.byref(deft_embed_t(
            n, vocab, hidden, scale, _p(tokens), _p(table), _ld(table), _p(out), _ld(out), _p(status), self._stream())))
        return out

    @_on_stream
    def embed_grad(self, tokens: torch.Tensor, grad_out: torch.Tensor, vocab: Optional[int] = None, scale: float = 1.0,
                   grad_table: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
        """grad_table[v] (+)= scale * the sum of grad_out over the rows whose token is v.  Either
        `grad_table` or `vocab` says how many rows the table has."""
        n = self._words("tokens", tokens, torch.int32, (None,))[0]
        _, hidden = self._rows("grad_out", grad_out, n, None)
        if grad_table is None and (vocab is None or accumulate):
            raise ValueError("embed_grad needs grad_table, or vocab and nothing to add to")
        if grad_table is None:
            grad_table = torch.empty((vocab, hidden), dtype=self.dtype, device=self.device)
        vocab, _ = self._rows("grad_table", grad_table, vocab, hidden)
        self._call("deft_embed_grad", ctypes.byref(deft_embed_grad_t(
            n, vocab, hidden, scale, int(accumulate), _p(tokens), _p(grad_out), _ld(grad_out), _p(grad_table),
            _ld(grad_table), self._stream())))
        return grad_table

    @_on_stream
    def head_loss(self, hidden: torch.Tensor, weight: torch.Tensor, labels: torch.Tensor, logit_scale: float = 1.0,
                  status: Optional[torch.Tensor] = None):
        """(loss, lse) of every position, float32."""
        n, width = self._rows("hidden", hidden, None, None)
        vocab, _ = self._rows("weight", weight, None, width)
        self._words("labels", labels, torch.int32, (n,))
        both = torch.empty((2, n), dtype=torch.float32, device=self.device)
        if status is not None:
            self._words("status", status, torch.int32, (n,))
        self._call("deft_head_loss", ctypes.byref(deft_head_loss_t(
            n, vocab, width, logit_scale, _p(hidden), _ld(hidden), _p(weight), _ld(weight), _p(labels), _p(both[0]),
            _p(both[1]), _p(status), self._stream())))
        return both[0], both[1]

    @_on_stream
    def head_grad(self, hidden: torch.Tensor, weight: torch.Tensor, labels: torch.Tensor, lse: torch.Tensor,
                  row_grad: torch.Tensor, logit_scale: float = 1.0, grad_hidden: Optional[torch.Tensor] = None,
                  grad_weight: Optional[torch.Tensor] = None, accumulate: bool = False, need_hidden: bool = True,
                  need_weight: bool = True, piece_events: Optional[Sequence[torch.cuda.Event]] = None):
        """(grad_hidden, grad_weight) of sum(row_grad * loss); accumulate adds into grad_weight.  Event i of
        piece_events is recorded once the rows of grad_weight below (i + 1) * info().vocab_piece are final."""
        n, width = self._rows("hidden", hidden, None, None)
        vocab, _ = self._rows("weight", weight, None, width)
        self._words("labels", labels, torch.int32, (n,))
        self._words("lse", lse, torch.float32, (n,))
        self._words("row_grad", row_grad, torch.float32, (n,))
        if accumulate and (grad_weight is None or not need_weight):
            raise ValueError("accumulate needs grad_weight")
        if need_hidden and grad_hidden is None:
            grad_hidden = torch.empty((n, width), dtype=self.dtype, device=self.device)
        if need_weight and grad_weight is None:
            grad_weight = torch.empty((vocab, width), dtype=self.dtype, device=self.device)
        grad_hidden, grad_weight = grad_hidden if need_hidden else None, grad_weight if need_weight else None
        if need_hidden:
            self._rows("grad_hidden", grad_hidden, n, width)
        if need_weight:
            self._rows("grad_weight", grad_weight, vocab, width)
        events = None
        if piece_events:
            on = torch.cuda.current_stream(self.device)
            for e in piece_events:   # (torch makes an event when it is first recorded)
                e.record(on)
            events = (_vp * len(piece_events))(*[e.cuda_event for e in piece_events])
        self._call("deft_head_grad", ctypes.byref(deft_head_grad_t(
            n, vocab, width, logit_scale, int(accumulate), len(piece_events or ()), _p(hidden), _ld(hidden),
            _p(weight), _ld(weight), _p(labels), _p(lse), _p(row_grad), _p(grad_hidden), _ld(grad_hidden),
            _p(grad_weight), _ld(grad_weight), ctypes.cast(events, _vp) if events else None, self._stream())))
        return grad_hidden, grad_weight

    @_on_stream
    def distill(self, logits: torch.Tensor, teacher_index: torch.Tensor, teacher_logit: torch.Tensor,
                temperature: float = 1.0, status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """loss of every row, float32."""
        return self._distill(logits, teacher_index, teacher_logit, None, temperature, None, status)[0]

    @_on_stream
    def distill_grad(self, logits: torch.Tensor, teacher_index: torch.Tensor, teacher_logit: torch.Tensor,
                     row_grad: torch.Tensor, temperature: float = 1.0, grad_logits: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None):
        """(loss, grad_logits) in one pass over the logits; grad_logits may be the logits themselves."""
        return self._distill(logits, teacher_index, teacher_logit, row_grad, temperature, grad_logits, status, True)

    def _distill(self, logits, teacher_index, teacher_logit, row_grad, temperature, grad_logits, status, with_grad=False):
        n, vocab = self._rows("logits", logits, None, None)
        if with_grad:
            self._words("row_grad", row_grad, torch.float32, (n,))
        top_k = self._words("teacher_index", teacher_index, torch.int32, (n, None))[1]
        self._words("teacher_logit", teacher_logit, torch.float32, (n, top_k))
        loss = torch.empty(n, dtype=torch.float32, device=self.device)
        if with_grad:
            if grad_logits is None:
                grad_logits = torch.empty((n, vocab), dtype=self.dtype, device=self.device)
            self._rows("grad_logits", grad_logits, n, vocab)
        if status is not None:
            self._words("status", status, torch.int32, (n,))
        self._call("deft_distill", ctypes.byref(deft_distill_t(
            n, vocab, top_k, temperature, _p(logits), _ld(logits), _p(teacher_index), _p(teacher_logit),
            _p(row_grad), _p(loss), _p(grad_logits), _ld(grad_logits), _p(status), self._stream())))
        return loss, grad_logits


def _p(t):
    return None if t is None else t.data_ptr()


def _ld(t):
    """Elements between a matrix's rows (one row may have any stride: its width then)."""
    if t is None:
        return 0
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]
