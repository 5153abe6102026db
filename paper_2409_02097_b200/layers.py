"""ctypes binding over the C ABI in ``include/linfusion_layers.h``: a block's own layers.

``Linear``           a matrix product with bias, activation and residual in its epilogue
``GatedRecurrence``  a gated linear recurrence over the tokens, each channel for itself
``pack8``            activation checkpoints in 8 bits (``Packed8``), which both backward passes read as they are

Argument marshalling only: the arithmetic is in the CUDA library, and there is no CPU fallback.  Objects hold a
configuration and no device memory, so one may serve any streams and threads at once.
"""
from __future__ import annotations

import ctypes
from typing import Dict, Optional, Tuple

from . import block
from .attn import DTYPE_FP16, ERR_INVALID_ARG, LinFusionError, OK, allocating_on
from .block import Rows, _Checked, _Fixed, _call, _check_rc, _check_tensor, _copy, _like, _look, _torch_dtype

GROUP = 32          # channels that share a scale of a checkpoint
STATE_EVERY = 64    # tokens from one kept state of the recurrence to the next

ACTIVATIONS = {"none": 0, None: 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}

EXPORTED = ["linfusion_linear", "linfusion_linear_backward", "linfusion_linear_workspace_bytes", "linfusion_pack8", "linfusion_unpack8",
            "linfusion_recurrence", "linfusion_recurrence_backward", "linfusion_recurrence_workspace_bytes", "linfusion_layers_expired"]

_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class Pack8Desc(ctypes.Structure):
    """Mirror of ``linfusion_pack8_desc_t``."""
    _fields_ = [("B", _i32), ("N", _i32), ("C", _i32), ("flags", ctypes.c_uint32)]


class Packed8Struct(ctypes.Structure):
    """Mirror of ``linfusion_packed8_t``."""
    _fields_ = [("codes", _vp), ("scales", _vp)]


class RecurrenceDesc(ctypes.Structure):
    """Mirror of ``linfusion_recurrence_desc_t``."""
    _fields_ = [("B", _i32), ("N", _i32), ("C", _i32), ("reverse", _i32), ("flags", ctypes.c_uint32)]


class RecurrenceInput(ctypes.Structure):
    """Mirror of ``linfusion_recurrence_input_t``."""
    _fields_ = [("rows", Rows), ("packed", Packed8Struct)]


class RecurrenceGrads(ctypes.Structure):
    """Mirror of ``linfusion_recurrence_grads_t``."""
    _fields_ = [("x", Rows), ("decay", Rows), ("gate", Rows), ("rate", _vp), ("h0", _vp)]


class LinearDesc(ctypes.Structure):
    """Mirror of ``linfusion_linear_desc_t``."""
    _fields_ = [("M", _i32), ("K", _i32), ("N", _i32), ("act", _i32), ("w_transposed", _i32), ("flags", ctypes.c_uint32)]


class Matrix(ctypes.Structure):
    """Mirror of ``linfusion_matrix_t``."""
    _fields_ = [("p", _vp), ("row", _i64)]


class LinearSaved(ctypes.Structure):
    """Mirror of ``linfusion_linear_saved_t``."""
    _fields_ = [("x", Matrix), ("u", Matrix), ("x_packed", Packed8Struct), ("u_packed", Packed8Struct)]


_lib = None


def load_library() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        lib, P, size = block.load_library(), ctypes.POINTER, ctypes.c_size_t
        rows, given, matrix, linear = P(Rows), P(RecurrenceInput), P(Matrix), P(LinearDesc)
        for name, args in {
                "linfusion_linear": [linear, matrix, matrix, _vp, matrix, matrix, matrix, P(Packed8Struct), _vp, size, _vp],
                "linfusion_linear_backward": [linear, matrix, P(LinearSaved), matrix, matrix, matrix, _vp, _vp, size, _vp],
                "linfusion_linear_workspace_bytes": [linear, _i32, _i32, P(size)],
                "linfusion_pack8": [P(Pack8Desc), rows, P(Packed8Struct), _vp],
                "linfusion_unpack8": [P(Pack8Desc), P(Packed8Struct), rows, _vp],
                "linfusion_recurrence": [P(RecurrenceDesc), given, given, given, _vp, _vp, rows, _vp, _vp, _vp, size, _vp],
                "linfusion_recurrence_backward": [P(RecurrenceDesc), given, given, given, _vp, _vp, _vp, rows, _vp, P(RecurrenceGrads), _vp,
                                                  size, _vp],
                "linfusion_recurrence_workspace_bytes": [P(RecurrenceDesc), _i32, P(size)],
                "linfusion_layers_expired": [_i32, P(ctypes.c_uint32), _vp]}.items():
            getattr(lib, name).restype = ctypes.c_int
            getattr(lib, name).argtypes = args
        _lib = lib
    return _lib


def expired(device: int = 0, stream: Optional[int] = None) -> int:
    """How many waits of these layers' kernels expired on `device` since the library was loaded (synchronizes the stream); outputs
    of a call whose wait expired are not to be used."""
    import torch
    n = ctypes.c_uint32(0)
    if stream is None:
        stream = torch.cuda.current_stream(device).cuda_stream
    _check_rc(load_library().linfusion_layers_expired(int(device), ctypes.byref(n), stream), "linfusion_layers_expired")
    return int(n.value)


def _counted(**counts):
    """Refuses what the descriptors' 32 bits do not hold (ctypes would cut it off)."""
    for name, n in counts.items():
        if n > 2 ** 31 - 1:
            raise ValueError(f"{name}: {n} does not fit 32 bits")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _refusal(rc, what, apart=(), **tensors):
    """The error of a call that the library refused; of an invalid argument with the name of the first tensor whose place or strides are the
    reason (the checks above it have seen to shapes and types).  ``apart``: those whose rows may not lie on top of one another."""
    if rc == ERR_INVALID_ARG:
        for name, t in tensors.items():
            if t is None:
                continue
            if isinstance(t, Packed8):
                p, axes = t._at[0], []
            else:
                p, axes = t.data_ptr(), sorted((s, n) for n, s in zip(t.shape, t.stride()) if n > 1 and s != 1)
            reach = 1 if not axes else t.shape[-1] if t.stride(-1) == 1 or t.shape[-1] == 1 else t.shape[-2]
            if p % 16 != 0 or (name == "workspace" and p % 256 != 0):
                return LinFusionError(rc, f"{what}: {name}: not on a boundary of {256 if name == 'workspace' else 16} bytes")
            for s, n in axes:
                if s % 8 != 0:
                    return LinFusionError(rc, f"{what}: {name}: a stride of {s} elements is no multiple of 8")
                if name in apart and s < reach:
                    return LinFusionError(rc, f"{what}: {name}: rows on top of one another ({s} elements apart)")
                reach += (n - 1) * s
    return LinFusionError(rc, what)


# -------------------------------------------------------------------------------------- checkpoints
def _rows3(t, name):
    """A tensor [..., C] as [B, N, C] without a copy: the axes before the last two have to merge."""
    if t.dim() == 0:
        raise ValueError(f"{name}: expected [..., C], got a number")
    if t.dim() == 3:
        return t
    if t.dim() < 3:
        return t.view((1,) * (3 - t.dim()) + tuple(t.shape)) if t.is_contiguous() else t.unsqueeze(0)
    try:
        return t.view(-1, *t.shape[-2:])
    except RuntimeError:
        raise ValueError(f"{name}: the axes before the last two, of strides {t.stride()}, do not merge") from None


def _pack8_desc(t, name, dtype):
    _check_tensor(t, name, _torch_dtype(dtype))
    if t.numel() == 0:
        raise ValueError(f"{name}: no values")
    r = _rows3(t, name)
    B, N, C = r.shape
    _counted(**{f"{name}: batch": B, f"{name}: rows": N, f"{name}: channels": C})
    return Pack8Desc(B, N, C, DTYPE_FP16 if dtype == "fp16" else 0), Rows(None, r.stride(0), r.stride(1))


_packings = _Checked()


def _pack8_rows(t, name, dtype):
    """Descriptor and rows of a tensor, the checks made once for each combination of what they depend on."""
    key = (_look(t), dtype)
    found = _packings.get(key)
    if found is None:
        found = _packings.keep(key, _pack8_desc(t, name, dtype))
    rows = _copy(found[1])
    rows.p = t.data_ptr()
    return found[0], rows


class Packed8:
    """A tensor in 8 bits: ``codes`` int8 of its shape, ``scales`` uint8 [..., ceil(C / 32)], both contiguous CUDA tensors; a value is
    ``codes * 2 ** (scales - 127)``, the scale that of its 32 channels.  ``dtype``: the storage type ("bf16" or "fp16") that it
    was made from, in which those values are exact.  A code of -128 stands for what was not finite and reads as NaN
    (``GatedRecurrence``: as a padded token, where it is decay's)."""

    __slots__ = ("_codes", "_scales", "_buffer", "_at", "shape", "dtype", "device")

    def __init__(self, codes, scales, dtype: str = "bf16"):
        import torch
        _torch_dtype(dtype)
        if codes.dtype != torch.int8 or scales.dtype != torch.uint8:
            raise ValueError(f"expected int8 codes and uint8 scales, got {codes.dtype} and {scales.dtype}")
        if codes.dim() < 1 or tuple(scales.shape) != (*codes.shape[:-1], -(-codes.shape[-1] // GROUP)):
            raise ValueError(f"codes {tuple(codes.shape)} and scales {tuple(scales.shape)} do not belong together")
        if not codes.is_cuda or scales.device != codes.device:
            raise ValueError("expected CUDA tensors on one device")
        if not codes.is_contiguous() or not scales.is_contiguous():
            raise ValueError("codes and scales must be contiguous")
        self._codes, self._scales, self._buffer = codes, scales, None
        self._at = (codes.data_ptr(), scales.data_ptr())
        self.shape, self.dtype, self.device = codes.shape, dtype, codes.device

    @classmethod
    def _new(cls, shape, dtype, device):
        """An uninitialised checkpoint; its two tensors lie in one allocation and are made when they are asked for."""
        import torch
        self = object.__new__(cls)
        rows = 1
        for n in shape[:-1]:
            rows *= n
        room = -(-rows * shape[-1] // 256) * 256
        self._buffer = torch.empty(room + rows * -(-shape[-1] // GROUP), dtype=torch.uint8, device=device)
        p = self._buffer.data_ptr()
        self._codes = self._scales = None
        self._at = (p, p + room)
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, self._buffer.device
        return self

    @property
    def codes(self):
        import torch
        if self._codes is None:
            self._codes = self._buffer[:self.shape.numel()].view(torch.int8).view(self.shape)
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            groups = (*self.shape[:-1], -(-self.shape[-1] // GROUP))
            self._scales = self._buffer[self._at[1] - self._at[0]:].view(groups)
        return self._scales

    def _struct(self):
        return Packed8Struct(*self._at)

    def unpack(self, out=None, stream: Optional[int] = None):
        """The values in the storage type (exact)."""
        import torch
        index = self.device.index
        if stream is not None:
            with allocating_on(stream, index):
                return self.unpack(out)
        if out is None:
            out = torch.empty(self.shape, dtype=_torch_dtype(self.dtype), device=self.device)
        elif out.shape != self.shape or out.device != self.device:
            raise ValueError(f"out: expected {tuple(self.shape)} on {self.device}, got {tuple(out.shape)} on {out.device}")
        desc, rows = _pack8_rows(out, "out", self.dtype)
        rc = _call(index, load_library().linfusion_unpack8, desc, self._struct(), rows)
        if rc != OK:
            raise _refusal(rc, "linfusion_unpack8", ("out",), codes=self, out=out)
        return out


def pack8(x, out: Optional[Packed8] = None, stream: Optional[int] = None) -> Packed8:
    """A bf16 or fp16 CUDA tensor [..., C] in 8 bits (see ``Packed8``): 32 channels share a power of two, values are rounded to 255 steps.
    Axes before the last two must merge; strides are multiples of 8."""
    import torch
    if x.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"x: expected bf16 or fp16, got {x.dtype}")
    dtype = "fp16" if x.dtype == torch.float16 else "bf16"
    if stream is not None and x.is_cuda:
        with allocating_on(stream, x.get_device()):
            return pack8(x, out)
    desc, rows = _pack8_rows(x, "x", dtype)
    if out is None:
        out = Packed8._new(x.shape, dtype, x.device)
    elif out.shape != x.shape or out.dtype != dtype or out.device != x.device:
        raise ValueError(f"out: expected a {dtype} checkpoint of {tuple(x.shape)} on {x.device}")
    rc = _call(x.get_device(), load_library().linfusion_pack8, desc, rows, out._struct())
    if rc != OK:
        raise _refusal(rc, "linfusion_pack8", x=x, out=out)
    return out


# -------------------------------------------------------------------------------------- recurrence
def _look8(t):
    """_look() of a tensor or a checkpoint (whose tensors are contiguous)."""
    return (t.shape, t.dtype, t.device) if isinstance(t, Packed8) else _look(t)


class GatedRecurrence(_Fixed):
    """A gated linear recurrence over the tokens of x [B, N, C], each channel for itself, from the first token to the last or
    with ``reverse`` from the last to the first:

        a_t = exp(-rate * sigmoid(decay_t))        v_t = sigmoid(gate_t) * x_t    (x_t without ``gate``)
        h_t = a_t h_(t-1) + (1 - a_t) v_t

    x, decay, gate: 16-bit CUDA tensors [B, N, C] with any batch and row strides that are multiples of 8 elements (windows of
    one projection are fine); rate: fp32 [C], a negative one counts as NaN, an infinite one as fp32's largest number; h0: fp32
    [B, C], the state before the first token (None: zero).
    A token with decay = -inf leaves the state as it is, whatever its x and gate hold: padding (in a checkpoint of decay, a token whose
    decay was not finite: give a finite one of 17 or more for +inf).  One token at a time, with h0 the state that the call before
    returned, gives what one call over all tokens gives (up to the rounding of fp32).
    """

    def __init__(self, C: int, reverse: bool = False, dtype: str = "bf16"):
        if int(C) <= 0 or int(C) % 8 != 0:
            raise ValueError(f"C: expected a multiple of 8, got {C}")
        _counted(C=int(C))
        self.C, self.reverse, self.dtype = int(C), bool(reverse), dtype
        self._torch_dtype = _torch_dtype(dtype)
        self._flags = DTYPE_FP16 if dtype == "fp16" else 0
        self._lib = load_library()
        self._checked = _Checked()

    def _desc(self, B, N):
        _counted(B=B, N=N)
        return RecurrenceDesc(B, N, self.C, self.reverse, self._flags)

    def workspace_bytes(self, B: int, N: int, backward: bool = False, state: bool = True) -> int:
        """Bytes of workspace that ``forward`` takes for B x N tokens, or ``backward`` with or without the saved states."""
        n = ctypes.c_size_t(0)
        _check_rc(self._lib.linfusion_recurrence_workspace_bytes(ctypes.byref(self._desc(int(B), int(N))), (1 if state else 2) if backward else 0,
                                                                 ctypes.byref(n)), "linfusion_recurrence_workspace_bytes")
        return int(n.value)

    def state_shape(self, B: int, N: int) -> Tuple[int, int, int]:
        """Shape of the saved states, those before every 64th token in the order of the scan."""
        return (B, -(-N // STATE_EVERY), self.C)

    def _rows(self, t, name, shape, device):
        if tuple(t.shape) != shape:
            raise ValueError(f"{name}: expected {shape}, got {tuple(t.shape)}")
        _check_tensor(t, name, self._torch_dtype, device)
        return Rows(None, t.stride(0), t.stride(1))

    def _input(self, t, name, shape, device, packed):
        if isinstance(t, Packed8) != packed:
            raise ValueError("x, decay and gate: either all in 8 bits or none")
        if not packed:
            return RecurrenceInput(self._rows(t, name, shape, device), Packed8Struct())
        if tuple(t.shape) != shape or t.dtype != self.dtype or t.device != device:
            raise ValueError(f"{name}: expected a {self.dtype} checkpoint of {shape} on {device}, got a {t.dtype} one of {tuple(t.shape)} on {t.device}")
        return RecurrenceInput()

    def _floats(self, t, name, shape, device):
        import torch
        if t is None:
            if name == "rate":
                raise ValueError("rate: needed")
            return
        if tuple(t.shape) != shape or t.dtype != torch.float32 or t.device != device or not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous fp32 tensor of {shape} on {device}")

    def _check(self, x, decay, gate, rate, h0, others, floats, backward):
        if len(x.shape) != 3 or x.shape[0] == 0 or x.shape[1] == 0 or x.shape[2] != self.C:
            raise ValueError(f"x: expected [B, N, {self.C}] with at least one token, got {tuple(x.shape)}")
        shape, device, packed = tuple(x.shape), x.device, isinstance(x, Packed8)
        B, N, _ = shape
        ins = [None if t is None else self._input(t, name, shape, device, packed) for name, t in (("x", x), ("decay", decay), ("gate", gate))]
        ends = (B, self.C)
        for name, t, want in (("rate", rate, (self.C,)), ("h0", h0, ends), *((n, t, self.state_shape(B, N) if n == "state" else ends) for n, t in floats)):
            self._floats(t, name, want, device)
        outs = [None if t is None else self._rows(t, name, shape, device) for name, t in others]
        state = any(n == "state" and t is not None for n, t in floats)
        return self._desc(B, N), ins, outs, self.workspace_bytes(B, N, backward, state)

    @staticmethod
    def _inputs(structs, tensors):
        out = []
        for s, t in zip(structs, tensors):
            if s is not None:
                s = _copy(s)
                if isinstance(t, Packed8):
                    s.packed = t._struct()
                else:
                    s.rows.p = t.data_ptr()
            out.append(s)
        return out

    @staticmethod
    def _workspace(workspace, need, device):
        import torch
        if workspace is None:
            return torch.empty(need, dtype=torch.uint8, device=device) if need else None
        if not workspace.is_cuda or workspace.device != device or not workspace.is_contiguous():
            raise ValueError("workspace: expected a contiguous CUDA tensor on the device of the others")
        return workspace

    def forward(self, x, decay, rate, gate=None, h0=None, save: bool = False, h=None, last=None, state=None, workspace=None,
                stream: Optional[int] = None) -> Tuple:
        """(h, last, state): the states of all tokens in the storage type, the last of the scan in fp32 [B, C], and with ``save`` those
        before every 64th token in fp32 (``state_shape``; else None), which ``backward`` recomputes h from.  ``h`` may be given as x,
        decay or gate, ``last`` as h0 (in place).  ``workspace``: a CUDA tensor of at least ``workspace_bytes``, else one is
        allocated."""
        import torch
        if isinstance(x, Packed8) or isinstance(decay, Packed8) or isinstance(gate, Packed8):
            raise ValueError("the forward pass takes 16-bit inputs")
        if decay is None:
            raise ValueError("decay: needed")
        if stream is not None and x.is_cuda:
            with allocating_on(stream, x.get_device()):
                return self.forward(x, decay, rate, gate, h0, save, h, last, state, workspace)
        if state is not None and not save:
            raise ValueError("state is given, but not save")
        key = (x.shape, x.stride(), x.dtype, decay.shape, decay.stride(), decay.dtype, x.get_device(), decay.get_device(), _look(gate), _look(rate), _look(h0),
               _look(h), _look(last), _look(state))
        found = self._checked.get(key)
        if found is None:
            found = self._checked.keep(key, self._check(x, decay, gate, rate, h0, (("h", h),), (("last", last), ("state", state)), False))
        desc, ins, outs, need = found
        B, N, C = x.shape
        device = x.device
        if h is None:
            h, rows = _like(x), Rows(None, N * C, C)
        else:
            rows = _copy(outs[0])
        rows.p = h.data_ptr()
        if last is None:
            last = torch.empty((B, C), dtype=torch.float32, device=device) if h0 is None else torch.empty_like(h0)
        if save and state is None:
            state = torch.empty(self.state_shape(B, N), dtype=torch.float32, device=device)
        ws = self._workspace(workspace, need, device)
        ix, id_, ig = self._inputs(ins, (x, decay, gate))
        rc = _call(x.get_device(), self._lib.linfusion_recurrence, desc, ix, id_, ig, rate.data_ptr(), _ptr(h0), rows, last.data_ptr(), _ptr(state),
                   _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size())
        if rc != OK:
            raise _refusal(rc, "linfusion_recurrence", ("h",), x=x, decay=decay, gate=gate, rate=rate, h0=h0, h=h, last=last, state=state, workspace=ws)
        return h, last, state

    def backward(self, dh, x, decay, rate, gate=None, h0=None, state=None, dlast=None, dx=None, ddecay=None, dgate=None, workspace=None,
                 stream: Optional[int] = None) -> Dict:
        """Gradients by name: ``x``, ``decay``, ``gate`` where there is one, in the storage type, ``rate`` and, with h0, ``h0`` in fp32.

        x, decay, gate as ``forward`` had them, or all as ``Packed8``; ``state`` as ``forward(save=True)`` returned it (None:
        recomputed, from the inputs and h0); ``dlast`` the gradient of the last state.  dx, ddecay and dgate may be given as dh
        or as their 16-bit inputs (in place), or as windows of one tensor."""
        import torch
        if stream is not None and dh.is_cuda:
            with allocating_on(stream, dh.get_device()):
                return self.backward(dh, x, decay, rate, gate, h0, state, dlast, dx, ddecay, dgate, workspace)
        if dgate is not None and gate is None:
            raise ValueError("dgate is given, but no gate")
        if decay is None:
            raise ValueError("decay: needed")
        key = (1, _look(dh), _look8(x), _look8(decay), _look8(gate), _look(rate), _look(h0), _look(state), _look(dlast), _look(dx), _look(ddecay),
               _look(dgate))
        found = self._checked.get(key)
        if found is None:
            others = (("dh", dh), ("dx", dx), ("ddecay", ddecay), ("dgate", dgate))
            found = self._checked.keep(key, self._check(x, decay, gate, rate, h0, others, (("state", state), ("dlast", dlast)), True))
        desc, ins, outs, need = found
        B, N, C = x.shape
        out, rows = {}, []
        for name, t, struct, wanted in (("x", dx, outs[1], True), ("decay", ddecay, outs[2], True), ("gate", dgate, outs[3], gate is not None)):
            if not wanted:
                rows.append(Rows())
                continue
            if t is None:
                t, struct = _like(dh), Rows(None, N * C, C)
            out[name] = t
            rows.append(Rows(t.data_ptr(), struct.batch, struct.row))
        device = dh.device
        out["rate"] = torch.empty(C, dtype=torch.float32, device=device)
        if h0 is not None:
            out["h0"] = torch.empty((B, C), dtype=torch.float32, device=device)
        grads = RecurrenceGrads(*rows, out["rate"].data_ptr(), _ptr(out.get("h0")))
        ws = self._workspace(workspace, need, device)
        ix, id_, ig = self._inputs(ins, (x, decay, gate))
        rdh = Rows(dh.data_ptr(), outs[0].batch, outs[0].row)
        rc = _call(dh.get_device(), self._lib.linfusion_recurrence_backward, desc, ix, id_, ig, rate.data_ptr(), _ptr(h0), _ptr(state), rdh,
                   _ptr(dlast), grads, ws.data_ptr(), ws.numel() * ws.element_size())
        if rc != OK:
            raise _refusal(rc, "linfusion_recurrence_backward", ("dx", "ddecay", "dgate"), dh=dh, x=x, decay=decay, gate=gate, rate=rate, h0=h0, state=state,
                           dlast=dlast, dx=dx, ddecay=ddecay, dgate=dgate, workspace=ws)
        return out


# -------------------------------------------------------------------------------------- matrix product
def _as_matrix(t, name, C):
    """(rows, stride of a row) of a tensor [..., C] whose leading axes are rows evenly spaced."""
    if t.dim() < 1 or t.shape[-1] != C:
        raise ValueError(f"{name}: expected [..., {C}], got {tuple(t.shape)}")
    rows, step = 1, None
    for n, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n == 1:
            continue
        if step is not None and s != rows * step:
            raise ValueError(f"{name}: the rows of strides {t.stride()} are not evenly spaced")
        if step is None:
            step = s
        rows *= n
    return rows, C if step is None else step


class Linear(_Fixed):
    """A matrix product with its epilogue, u = x w + bias, y = act(u) + residual, from ``K`` input to ``N`` output channels (multiples
    of 8).

    x [..., K], residual and y [..., N]: 16-bit CUDA tensors whose leading axes are evenly spaced rows, a multiple of 8
    elements and at least their own length apart (an expanded tensor is made contiguous first); w [K, N] with either axis contiguous (a torch.nn.Linear's weight is given as ``weight.t()``); bias [N].
    ``activation``: "none", "relu", "silu", "gelu" or "gelu_tanh".
    """

    def __init__(self, K: int, N: int, activation: Optional[str] = "none", dtype: str = "bf16"):
        if activation not in ACTIVATIONS:
            raise ValueError("activation must be 'none', 'relu', 'silu', 'gelu' or 'gelu_tanh'")
        for name, n in (("K", K), ("N", N)):
            if int(n) <= 0 or int(n) % 8 != 0:
                raise ValueError(f"{name}: expected a multiple of 8, got {n}")
            _counted(**{name: int(n)})
        self.K, self.N, self.act, self.dtype = int(K), int(N), ACTIVATIONS[activation], dtype
        self._torch_dtype = _torch_dtype(dtype)
        self._flags = DTYPE_FP16 if dtype == "fp16" else 0
        self._lib = load_library()
        self._checked = _Checked()

    def _desc(self, M, transposed=False):
        _counted(rows=M)
        return LinearDesc(M, self.K, self.N, self.act, transposed, self._flags)

    def workspace_bytes(self, rows: int, backward: bool = False, x_packed: bool = False, transposed: bool = False, sm_count: int = 0) -> int:
        """Bytes of workspace that ``forward`` takes for that many rows, or ``backward``, with x in 16 or 8 bits and a weight as [K, N] or, seen
        transposed, as [N, K]."""
        n = ctypes.c_size_t(0)
        _check_rc(self._lib.linfusion_linear_workspace_bytes(ctypes.byref(self._desc(int(rows), bool(transposed))),
                                                             (2 if x_packed else 1) if backward else 0, int(sm_count), ctypes.byref(n)),
                  "linfusion_linear_workspace_bytes")
        return int(n.value)

    def _matrix(self, t, name, C, rows, device):
        if t is None:
            return None
        _check_tensor(t, name, self._torch_dtype, device)
        n, step = _as_matrix(t, name, C)
        if n != rows:
            raise ValueError(f"{name}: expected {rows} rows, got {n}")
        return Matrix(None, step)

    def _weight(self, t, name, device):
        """(structure, transposed)"""
        if tuple(t.shape) != (self.K, self.N) or t.dtype != self._torch_dtype or t.device != device:
            raise ValueError(f"{name}: expected {self._torch_dtype} {(self.K, self.N)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
        if t.stride(1) == 1:
            return Matrix(None, t.stride(0)), False
        if t.stride(0) == 1:
            return Matrix(None, t.stride(1)), True
        raise ValueError(f"{name}: one of its axes must be contiguous, got strides {t.stride()}")

    def _packed(self, t, name, C, rows, device):
        if t.shape[-1] != C or t.shape.numel() != rows * C or t.dtype != self.dtype or t.device != device:
            raise ValueError(f"{name}: expected a {self.dtype} checkpoint of {rows} x {C} on {device}, got a {t.dtype} one of {tuple(t.shape)} on {t.device}")

    @staticmethod
    def _at(struct, t):
        if struct is None or t is None:
            return None
        return Matrix(t.data_ptr(), struct.row)

    def _check_forward(self, x, w, bias, residual, y, u):
        if not x.is_cuda:
            raise ValueError("x: expected a CUDA tensor")
        device = x.device
        rows, _ = _as_matrix(x, "x", self.K)
        if rows == 0 or x.numel() == 0:
            raise ValueError("x: no rows")
        mx = self._matrix(x, "x", self.K, rows, device)
        mw, transposed = self._weight(w, "w", device)
        if bias is not None and (tuple(bias.shape) != (self.N,) or bias.dtype != self._torch_dtype or bias.device != device or not bias.is_contiguous()):
            raise ValueError(f"bias: expected a contiguous {self._torch_dtype} tensor of {(self.N,)} on {device}")
        shape = (*x.shape[:-1], self.N)
        for name, t in (("residual", residual), ("y", y), ("u", u)):
            if t is not None and tuple(t.shape) != shape:
                raise ValueError(f"{name}: expected {shape}, got {tuple(t.shape)}")
        mr, my = self._matrix(residual, "residual", self.N, rows, device), self._matrix(y, "y", self.N, rows, device)
        mu = None
        if isinstance(u, Packed8):
            self._packed(u, "u", self.N, rows, device)
        else:
            mu = self._matrix(u, "u", self.N, rows, device)
        dense = Matrix(None, self.N)
        return (self._desc(rows, transposed), mx, mw, mr, my or dense, mu or dense, shape,
                self.workspace_bytes(rows, transposed=transposed, sm_count=block._sm_count(device.index)))

    def forward(self, x, w, bias=None, residual=None, save: Optional[str] = None, y=None, u=None, workspace=None,
                stream: Optional[int] = None) -> Tuple:
        """(y, u).  ``save``: what is kept of the pre-activation for ``backward``: None (u is None; enough without an activation), "full"
        (in the storage type) or "packed" (a ``Packed8``, made from the fp32 sums).  ``y`` may be given as ``residual`` (in place).
        ``workspace``: a CUDA tensor of at least ``workspace_bytes``, else one is allocated."""
        import torch
        if save not in (None, "full", "packed"):
            raise ValueError("save must be None, 'full' or 'packed'")
        if u is not None and (save is None or (save == "packed") != isinstance(u, Packed8)):
            raise ValueError("u: expected a tensor with save='full', a Packed8 with save='packed'")
        if stream is not None and x.is_cuda:
            with allocating_on(stream, x.get_device()):
                return self.forward(x, w, bias, residual, save, y, u, workspace)
        key = (x.shape, x.stride(), x.dtype, w.shape, w.stride(), w.dtype, x.get_device(), w.get_device(), _look(bias), _look(residual), _look(y), _look8(u))
        found = self._checked.get(key)
        if found is None:
            found = self._checked.keep(key, self._check_forward(x, w, bias, residual, y, u))
        desc, mx, mw, mr, my, mu, shape, need = found
        device = x.device
        if y is None:
            y = torch.empty(shape, dtype=self._torch_dtype, device=device) if residual is None else _like(residual)
        packed = None
        if save == "packed":
            if u is None:
                u = Packed8._new(shape, self.dtype, device)
            packed = u._struct()
        elif save == "full" and u is None:
            u = torch.empty(shape, dtype=self._torch_dtype, device=device)
        ws = GatedRecurrence._workspace(workspace, need, device)
        rc = _call(x.get_device(), self._lib.linfusion_linear, desc, self._at(mx, x), self._at(mw, w), _ptr(bias), self._at(mr, residual),
                   self._at(my, y), self._at(mu, u) if save == "full" else None, packed, _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size())
        if rc != OK:
            raise _refusal(rc, "linfusion_linear", ("x", "w", "residual", "y", "u"), x=x, w=w, bias=bias, residual=residual, y=y, u=u, workspace=ws)
        return y, u

    def _check_backward(self, dy, x, w, u, dx, dw, need):
        if not dy.is_cuda:
            raise ValueError("dy: expected a CUDA tensor")
        device = dy.device
        rows, _ = _as_matrix(dy, "dy", self.N)
        if rows == 0 or dy.numel() == 0:
            raise ValueError("dy: no rows")
        mdy = self._matrix(dy, "dy", self.N, rows, device)
        ms = {}
        for name, t, C, wanted in (("x", x, self.K, "w" in need), ("u", u, self.N, self.act != 0)):
            if not wanted:
                continue
            if t is None:
                raise ValueError(f"{name}: needed for this backward pass")
            if isinstance(t, Packed8):
                self._packed(t, name, C, rows, device)
            else:
                ms[name] = self._matrix(t, name, C, rows, device)
        if w is None and ("x" in need or "w" in need):
            raise ValueError("w: needed for x's gradient, and for the layout of its own")
        mw, transposed = (None, False) if w is None else self._weight(w, "w", device)
        if dx is not None and tuple(dx.shape) != (*dy.shape[:-1], self.K):
            raise ValueError(f"dx: expected {(*dy.shape[:-1], self.K)}, got {tuple(dx.shape)}")
        mdx = self._matrix(dx, "dx", self.K, rows, device) or Matrix(None, self.K)
        mdw = Matrix(None, self.K if transposed else self.N)
        if dw is not None:
            mdw, other = self._weight(dw, "dw", device)
            if other != transposed:
                raise ValueError("dw: expected the contiguous axis of w")
        return (self._desc(rows, transposed), mdy, ms, mw, mdx, mdw, transposed,
                self.workspace_bytes(rows, True, isinstance(x, Packed8) and "w" in need, transposed, block._sm_count(device.index)))

    def backward(self, dy, x, w=None, u=None, need=("x", "w", "bias"), dx=None, dw=None, workspace=None, stream: Optional[int] = None) -> Dict:
        """Gradients by name, those in ``need``: ``x`` and ``w`` in the storage type (w's laid out as w is), ``bias`` in fp32.  The residual's is dy.

        x and, with an activation, u as ``forward`` had and returned them, each in 16 bits or as a ``Packed8``; x may be None without
        w's gradient, w where only the bias' is wanted.  du = dy * act'(u) is rounded to 16 bits before the two products; the
        bias' gradient sums it unrounded."""
        import torch
        need = tuple(need)
        if not need or any(n not in ("x", "w", "bias") for n in need):
            raise ValueError("need: some of 'x', 'w' and 'bias'")
        if (dx is not None and "x" not in need) or (dw is not None and "w" not in need):
            raise ValueError("dx and dw: only where they are needed")
        if stream is not None and dy.is_cuda:
            with allocating_on(stream, dy.get_device()):
                return self.backward(dy, x, w, u, need, dx, dw, workspace)
        key = (1, _look(dy), _look8(x), _look(w), _look8(u), _look(dx), _look(dw), need)
        found = self._checked.get(key)
        if found is None:
            found = self._checked.keep(key, self._check_backward(dy, x, w, u, dx, dw, need))
        desc, mdy, ms, mw, mdx, mdw, transposed, size = found
        device, out = dy.device, {}
        if "x" in need:
            out["x"] = dx if dx is not None else torch.empty((*dy.shape[:-1], self.K), dtype=self._torch_dtype, device=device)
        if "w" in need:
            if dw is None:
                dw = torch.empty((self.N, self.K) if transposed else (self.K, self.N), dtype=self._torch_dtype, device=device)
                dw = dw.t() if transposed else dw
            out["w"] = dw
        if "bias" in need:
            out["bias"] = torch.empty(self.N, dtype=torch.float32, device=device)
        saved = LinearSaved()
        for name, t, wanted in (("x", x, "w" in need), ("u", u, self.act != 0)):
            if wanted and isinstance(t, Packed8):
                setattr(saved, name + "_packed", t._struct())
            elif wanted:
                setattr(saved, name, self._at(ms[name], t))
        ws = GatedRecurrence._workspace(workspace, size, device)
        rc = _call(dy.get_device(), self._lib.linfusion_linear_backward, desc, self._at(mdy, dy), saved, self._at(mw, w), self._at(mdx, out.get("x")),
                   self._at(mdw, out.get("w")), _ptr(out.get("bias")), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size())
        if rc != OK:
            raise _refusal(rc, "linfusion_linear_backward", ("dy", "x", "w", "u", "dx", "dw"), dy=dy, x=x, w=w, u=u, dx=dx, dw=dw, workspace=ws)
        return out
