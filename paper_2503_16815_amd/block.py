"""Thin Python binding of include/deft_block.h (argument marshalling only): the gated feed-forward block
with its gradient, and activation checkpoints in 8 bits.

Every step runs in the HIP library; PyTorch supplies device memory and streams.  There is no CPU
fallback.  Arguments that the kernels do not take as they are (another type, device or shape,
elements of a row apart) are refused with ValueError; nothing is copied or converted silently.
"""
from __future__ import annotations

import ctypes
from typing import Iterable, NamedTuple, Optional, Sequence, Union

import torch

from . import binding
from .binding import DEFT_OK, DeftError
from .ends import DTYPES, _MOST, Marshalling, _ld, _on_stream, _p

OPERATORS = {"ffn": 1, "ffn_grad": 2, "checkpoint": 4, "restore": 8}
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3}
SAVES = {None: 0, "full": 1, "packed": 2}
GROUP = 32   # elements of a row that share a checkpoint's scale
EXPORTS = ("deft_block_create", "deft_block_destroy", "deft_block_get_info", "deft_checkpoint", "deft_restore", "deft_ffn",
           "deft_ffn_grad")

_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class deft_block_config_t(ctypes.Structure):
    _fields_ = [("device", _i32), ("dtype", _i32), ("operators", ctypes.c_uint32), ("max_rows", _i32), ("max_hidden", _i32),
                ("max_inner", _i32)]


class deft_block_info_t(ctypes.Structure):
    _fields_ = [("scratch_bytes", _i64), ("compute_units", _i32)]


class deft_checkpoint_t(ctypes.Structure):
    _fields_ = [("codes", _vp), ("codes_stride", _i64), ("scales", _vp), ("scales_stride", _i64)]


class deft_checkpoint_call_t(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("width", _i32), ("x", _vp), ("x_stride", _i64), ("out", deft_checkpoint_t), ("stream", _vp)]


class deft_restore_call_t(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("width", _i32), ("from_", deft_checkpoint_t), ("out", _vp), ("out_stride", _i64),
                ("stream", _vp)]


class deft_saved_t(ctypes.Structure):
    _fields_ = [("kind", _i32), ("gate", deft_checkpoint_t), ("up", deft_checkpoint_t)]


_WEIGHTS = [(name + end, kind) for name in ("w_gate", "w_up", "w_down") for end, kind in (("", _vp), ("_stride", _i64))]


class deft_ffn_t(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("hidden", _i32), ("inner", _i32), ("activation", _i32), ("x", _vp), ("x_stride", _i64),
                *_WEIGHTS, ("y", _vp), ("y_stride", _i64), ("save", deft_saved_t), ("stream", _vp)]


class deft_ffn_grad_t(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("hidden", _i32), ("inner", _i32), ("activation", _i32), ("accumulate", _i32),
                ("grad_y", _vp), ("grad_y_stride", _i64), ("x", _vp), ("x_stride", _i64), ("packed_x", deft_checkpoint_t),
                *_WEIGHTS, ("saved", deft_saved_t), ("grad_x", _vp), ("grad_x_stride", _i64), ("grad_gate", _vp),
                ("grad_gate_stride", _i64), ("grad_up", _vp), ("grad_up_stride", _i64), ("grad_down", _vp),
                ("grad_down_stride", _i64), ("events", _vp), ("stream", _vp)]


class Checkpoint(NamedTuple):
    """Rows in 8 bits: what they stand for is codes * scales, a scale for each GROUP codes of a row."""
    codes: torch.Tensor    # int8 [rows][width]
    scales: torch.Tensor   # bfloat16 [rows][ceil(width / GROUP)]


class Saved(NamedTuple):
    """What ffn keeps for ffn_grad of the two projections.  "packed": their checkpoints.  "full": the same with int16
    codes, or, in 32 bits, with the numbers themselves as codes and no scales (None)."""
    gate: Checkpoint
    up: Checkpoint


_declared = False


def load_library() -> ctypes.CDLL:
    global _declared
    lib = binding.load_library()
    if not _declared:
        for name, args in (("deft_block_create", [ctypes.POINTER(deft_block_config_t), ctypes.POINTER(_vp)]),
                           ("deft_block_get_info", [_vp, ctypes.POINTER(deft_block_info_t)]),
                           ("deft_checkpoint", [_vp, ctypes.POINTER(deft_checkpoint_call_t)]),
                           ("deft_restore", [_vp, ctypes.POINTER(deft_restore_call_t)]),
                           ("deft_ffn", [_vp, ctypes.POINTER(deft_ffn_t)]),
                           ("deft_ffn_grad", [_vp, ctypes.POINTER(deft_ffn_grad_t)])):
            getattr(lib, name).restype = ctypes.c_int
            getattr(lib, name).argtypes = args
        lib.deft_block_destroy.restype = None
        lib.deft_block_destroy.argtypes = [_vp]
        _declared = True
    return lib


class DeftBlock(Marshalling):
    """Owner of one deft_block_t handle.

    `operators` names what the handle serves (keys of OPERATORS); ffn and ffn_grad hold scratch memory.  Outputs are
    allocated unless given; calls run on `stream` (default: torch's current stream) and return without waiting.  Tensors
    of a call on another stream than their own are recorded there.  The scratch memory is one call's at a time: a
    handle's calls go to one stream, or the next stream waits for the one before; work on two streams at once takes two
    handles, and a captured graph uses its handle's memory when it is replayed.

    Gradients are ffn_grad's results.  torch's automatic differentiation does not see any of these calls: what they give
    carries no graph, also of inputs that require a gradient, and what they write into is not marked as changed.
    """

    def __init__(self, operators: Iterable[str], dtype: torch.dtype, max_rows: int, max_hidden: int, max_inner: int = 0,
                 device: int = 0):
        self._h = _vp()
        self._lib = load_library()
        if dtype not in DTYPES:
            raise ValueError(f"dtype is one of {list(DTYPES)}: got {dtype}")
        for name, value in (("max_rows", max_rows), ("max_hidden", max_hidden), ("max_inner", max_inner), ("device", device)):
            if not -_MOST <= value <= _MOST:
                raise ValueError(f"{name} does not fit 32 bits: got {value}")
        mask = 0
        for name in ((operators,) if isinstance(operators, str) else operators):
            if name not in OPERATORS:
                raise ValueError(f"operators are {list(OPERATORS)}: got {name!r}")
            mask |= OPERATORS[name]
        self.dtype, self.device, self._index = dtype, torch.device("cuda", device), device
        cfg = deft_block_config_t(device, DTYPES[dtype], mask, max_rows, max_hidden, max_inner)
        rc = self._lib.deft_block_create(ctypes.byref(cfg), ctypes.byref(self._h))
        if rc != DEFT_OK:
            self._h = _vp()
            raise DeftError("deft_block_create", rc)

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h:
            self._lib.deft_block_destroy(self._h)
            self._h = None   # (at the interpreter's end the module's names are gone)

    __del__ = close

    def info(self) -> deft_block_info_t:
        info = deft_block_info_t()
        self._call("deft_block_get_info", ctypes.byref(info))
        return info

    # ---- the operators ----------------------------------------------------------------------

    @_on_stream
    def checkpoint(self, x: torch.Tensor, out: Optional[Checkpoint] = None) -> Checkpoint:
        """x in 8 bits."""
        n, width = self._rows("x", x, None, None)
        if out is None:
            out = self._new_checkpoint(n, width)
        else:
            self._check("out", out, n, width)
        self._call("deft_checkpoint", ctypes.byref(deft_checkpoint_call_t(
            n, width, _p(x), _ld(x), _packed(out), self._stream())))
        return out

    @_on_stream
    def restore(self, kept: Checkpoint, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """What a checkpoint stands for, in the handle's type."""
        n, width = self._check("kept", kept, None, None)
        if out is None:
            out = torch.empty((n, width), dtype=self.dtype, device=self.device)
        else:
            self._rows("out", out, n, width)
        self._call("deft_restore", ctypes.byref(deft_restore_call_t(
            n, width, _packed(kept), _p(out), _ld(out), self._stream())))
        return out

    @_on_stream
    def ffn(self, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, activation: str = "silu",
            save: Optional[str] = None, out: Optional[torch.Tensor] = None):
        """y = (act(x w_gate^T) * (x w_up^T)) w_down^T; with `save` ("full" or "packed") the pair (y, Saved)."""
        n, hidden = self._rows("x", x, None, None)
        inner = self._weights(w_gate, w_up, w_down, hidden)
        kind, saves = self._choice("activation", activation, ACTIVATIONS), self._choice("save", save, SAVES)
        if out is None:
            out = torch.empty((n, hidden), dtype=self.dtype, device=self.device)
        else:
            self._rows("out", out, n, hidden)
        saved = None
        if save is not None:
            codes = torch.int8 if save == "packed" else torch.float32 if self.dtype == torch.float32 else torch.int16
            saved = Saved(self._new_checkpoint(n, inner, codes), self._new_checkpoint(n, inner, codes))
        self._call("deft_ffn", ctypes.byref(deft_ffn_t(
            n, hidden, inner, kind, _p(x), _ld(x), _p(w_gate), _ld(w_gate), _p(w_up), _ld(w_up), _p(w_down), _ld(w_down),
            _p(out), _ld(out), _kept(saved, saves), self._stream())))
        return out if save is None else (out, saved)

    @_on_stream
    def ffn_grad(self, grad_y: torch.Tensor, x: Union[torch.Tensor, Checkpoint], w_gate: torch.Tensor, w_up: torch.Tensor,
                 w_down: torch.Tensor, saved: Optional[Saved] = None, activation: str = "silu",
                 grad_x: Optional[torch.Tensor] = None, grad_gate: Optional[torch.Tensor] = None,
                 grad_up: Optional[torch.Tensor] = None, grad_down: Optional[torch.Tensor] = None, accumulate: bool = False,
                 need_x: bool = True, need_weights: bool = True, events: Optional[Sequence[torch.cuda.Event]] = None):
        """(grad_x, grad_gate, grad_up, grad_down) of sum(grad_y * y), with the projections as `saved` has them (None: computed
        again from x, or from what x's checkpoint stands for); accumulate adds into the matrices' gradients.  The first of the
        two `events` is recorded once grad_down is final, the second once grad_gate and grad_up are."""
        n, hidden = self._rows("grad_y", grad_y, None, None)
        inner = self._weights(w_gate, w_up, w_down, hidden)
        kind = self._choice("activation", activation, ACTIVATIONS)
        packed_x = deft_checkpoint_t()
        if isinstance(x, Checkpoint):
            self._check("x", x, n, hidden)
            packed_x = _packed(x)
        else:
            self._rows("x", x, n, hidden)
        saves = 0
        if saved is not None:
            if not isinstance(saved, Saved):
                raise ValueError("saved: what ffn gave is wanted")
            wide = torch.float32 if self.dtype == torch.float32 else torch.int16
            packed = isinstance(saved.gate, Checkpoint) and saved.gate.codes.dtype == torch.int8
            self._check("saved.gate", saved.gate, n, inner, torch.int8 if packed else wide)
            self._check("saved.up", saved.up, n, inner, torch.int8 if packed else wide)
            saves = SAVES["packed" if packed else "full"]
        if accumulate and (not need_weights or grad_gate is None or grad_up is None or grad_down is None):
            raise ValueError("accumulate needs grad_gate, grad_up and grad_down")
        if not need_x and not need_weights:
            raise ValueError("no gradient is asked for")
        empty = lambda *shape: torch.empty(shape, dtype=self.dtype, device=self.device)  # noqa: E731
        grad_x = None if not need_x else empty(n, hidden) if grad_x is None else grad_x
        grad_gate = None if not need_weights else empty(inner, hidden) if grad_gate is None else grad_gate
        grad_up = None if not need_weights else empty(inner, hidden) if grad_up is None else grad_up
        grad_down = None if not need_weights else empty(hidden, inner) if grad_down is None else grad_down
        if need_x:
            self._rows("grad_x", grad_x, n, hidden)
        if need_weights:
            self._rows("grad_gate", grad_gate, inner, hidden)
            self._rows("grad_up", grad_up, inner, hidden)
            self._rows("grad_down", grad_down, hidden, inner)
        handles = None
        if events:
            if len(events) != 2:
                raise ValueError("events: two are wanted")
            on = torch.cuda.current_stream(self.device)
            for e in events:   # (torch makes an event when it is first recorded)
                e.record(on)
            handles = (_vp * 2)(*[e.cuda_event for e in events])
        of_x = (None, 0) if isinstance(x, Checkpoint) else (_p(x), _ld(x))
        self._call("deft_ffn_grad", ctypes.byref(deft_ffn_grad_t(
            n, hidden, inner, kind, int(accumulate), _p(grad_y), _ld(grad_y), *of_x, packed_x, _p(w_gate), _ld(w_gate),
            _p(w_up), _ld(w_up), _p(w_down), _ld(w_down), _kept(saved, saves), _p(grad_x), _ld(grad_x),
            _p(grad_gate), _ld(grad_gate), _p(grad_up), _ld(grad_up), _p(grad_down), _ld(grad_down),
            ctypes.cast(handles, _vp) if handles else None, self._stream())))
        return grad_x, grad_gate, grad_up, grad_down

    # ---- marshalling ------------------------------------------------------------------------

    @staticmethod
    def _choice(name, value, choices):
        if not isinstance(value, (str, type(None))) or value not in choices:
            raise ValueError(f"{name} is one of {list(choices)}: got {value!r}")
        return choices[value]

    def _weights(self, w_gate, w_up, w_down, hidden):
        inner, _ = self._rows("w_gate", w_gate, None, hidden)
        self._rows("w_up", w_up, inner, hidden)
        self._rows("w_down", w_down, hidden, inner)
        return inner

    def _new_checkpoint(self, n, width, dtype=torch.int8):   # (rows from 16-byte boundaries on)
        codes = torch.empty_strided((n, width), (-(-width // 16) * 16, 1), dtype=dtype, device=self.device)
        if dtype == torch.float32:
            return Checkpoint(codes, None)
        return Checkpoint(codes, torch.empty((n, -(-width // GROUP)), dtype=torch.bfloat16, device=self.device))

    def _check(self, name, kept, n, width, dtype=torch.int8):
        if not isinstance(kept, Checkpoint):
            raise ValueError(f"{name}: a Checkpoint is wanted")
        n, width = self._matrix(name + ".codes", kept.codes, dtype, n, width)
        if dtype != torch.float32:
            self._matrix(name + ".scales", kept.scales, torch.bfloat16, n, -(-width // GROUP))
        return n, width


def _packed(kept):
    return deft_checkpoint_t(_p(kept.codes), _ld(kept.codes), _p(kept.scales), _ld(kept.scales))


def _kept(saved, kind):
    return deft_saved_t(kind, _packed(saved.gate), _packed(saved.up)) if saved is not None else deft_saved_t()
