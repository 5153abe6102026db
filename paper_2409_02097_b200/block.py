"""ctypes binding over the C ABI in ``include/linfusion_block.h``: the operators that stand before and
after the attention inside a transformer block.

``AxialRope``  rotary positions with several axes (time, height, width) on Q and K
``BlockNorm``  the norms before and after a block, fused with modulation, gate and residual scale

Both have a ``backward``.  Argument marshalling only: the arithmetic is in the CUDA library, and there is
no CPU fallback.  Objects hold a configuration and no device memory, so one may serve any streams and
threads at once.
"""
from __future__ import annotations

import ctypes
from typing import Dict, Optional, Sequence, Tuple

from . import attn
from .attn import DTYPE_FP16, LinFusionError, OK, allocating_on

MAX_AXES = 4
NORM_NONE, NORM_LAYER, NORM_RMS = 0, 1, 2
NORMS = {"none": NORM_NONE, "layer": NORM_LAYER, "rms": NORM_RMS, None: NORM_NONE}

EXPORTED = ["linfusion_rope", "linfusion_block_norm", "linfusion_block_norm_backward", "linfusion_block_norm_workspace_bytes"]

_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class RopeDesc(ctypes.Structure):
    """Mirror of ``linfusion_rope_desc_t``."""
    _fields_ = [("B", _i32), ("N", _i32), ("d", _i32), ("n_axes", _i32), ("pairs", _i32 * MAX_AXES), ("interleaved", _i32),
                ("backward", _i32), ("theta", ctypes.c_double), ("flags", ctypes.c_uint32)]


class RopeTensor(ctypes.Structure):
    """Mirror of ``linfusion_rope_tensor_t``."""
    _fields_ = [("in_", _vp), ("out", _vp), ("heads", _i32), ("in_batch", _i64), ("in_token", _i64), ("in_head", _i64),
                ("out_batch", _i64), ("out_token", _i64), ("out_head", _i64)]


class NormDesc(ctypes.Structure):
    """Mirror of ``linfusion_block_norm_desc_t``."""
    _fields_ = [("B", _i32), ("N", _i32), ("C", _i32), ("pre", _i32), ("post", _i32), ("eps", ctypes.c_float),
                ("residual_scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


class Rows(ctypes.Structure):
    """Mirror of ``linfusion_rows_t``."""
    _fields_ = [("p", _vp), ("batch", _i64), ("row", _i64)]


class Channels(ctypes.Structure):
    """Mirror of ``linfusion_channels_t``."""
    _fields_ = [("p", _vp), ("batch", _i64)]


class NormVectors(ctypes.Structure):
    """Mirror of ``linfusion_block_norm_vectors_t``."""
    _fields_ = [("gate", Channels), ("scale", Channels), ("shift", Channels), ("pre_weight", _vp), ("pre_bias", _vp),
                ("post_weight", _vp), ("post_bias", _vp)]


class NormGrads(ctypes.Structure):
    """Mirror of ``linfusion_block_norm_grads_t``."""
    _fields_ = [("gate", _vp), ("scale", _vp), ("shift", _vp), ("pre_weight", _vp), ("pre_bias", _vp), ("post_weight", _vp),
                ("post_bias", _vp), ("per_entry", ctypes.c_uint32)]


PER_ENTRY = {"gate": 1, "scale": 2, "shift": 4}  # bits of NormGrads.per_entry
_lib = None


def load_library() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        lib, P = attn.load_library(), ctypes.POINTER
        lib.linfusion_rope.restype = ctypes.c_int
        lib.linfusion_rope.argtypes = [P(RopeDesc), P(RopeTensor), P(RopeTensor), _vp, _i64, _vp]
        lib.linfusion_block_norm.restype = ctypes.c_int
        lib.linfusion_block_norm.argtypes = [P(NormDesc), P(Rows), P(Rows), P(NormVectors), P(Rows), P(Rows), _vp]
        lib.linfusion_block_norm_backward.restype = ctypes.c_int
        lib.linfusion_block_norm_backward.argtypes = [P(NormDesc), P(Rows), P(Rows), P(NormVectors), P(Rows), P(Rows), P(Rows),
                                                      P(Rows), P(NormGrads), _vp, ctypes.c_size_t, _vp]
        lib.linfusion_block_norm_workspace_bytes.restype = ctypes.c_int
        lib.linfusion_block_norm_workspace_bytes.argtypes = [P(NormDesc), _i32, P(ctypes.c_size_t)]
        _lib = lib
    return _lib


def _check_rc(rc: int, what: str) -> None:
    if rc != OK:
        raise LinFusionError(rc, what)


def _torch_dtype(name: str):
    import torch
    if name not in ("bf16", "fp16"):
        raise ValueError("dtype must be 'bf16' or 'fp16'")
    return torch.float16 if name == "fp16" else torch.bfloat16


def _check_tensor(t, name, dtype, device=None):
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a CUDA tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name}: on {t.device}, the others are on {device}")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the channels of a row must be contiguous")


_sms: Dict[int, int] = {}


def _sm_count(index: int) -> int:
    n = _sms.get(index)
    if n is None:
        import torch
        n = _sms[index] = torch.cuda.get_device_properties(index).multi_processor_count
    return n


def _look(t):
    """What the checks of a tensor depend on; its address is no part of it."""
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device())


class _Checked(dict):
    """Argument checks by what they depend on (shapes, strides, types, devices): made once for each combination, not on
    every call.  Holds descriptors only, no tensor and no address."""

    MOST = 256

    def keep(self, key, value):
        if len(self) >= self.MOST:
            self.clear()
        self[key] = value
        return value


def _like(t):
    """An uninitialised contiguous tensor of t's shape, type and device."""
    import torch
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _copy(struct):
    """A structure of the caller's own (calls of several threads share the checked one)."""
    return type(struct).from_buffer_copy(struct)


def _call(index, function, *args):
    """`function(*args, stream)` on the current stream of the tensors' device, which is made current."""
    import torch
    stream = torch._C._cuda_getCurrentRawStream(index)
    if torch._C._cuda_getDevice() == index:
        return function(*args, stream)
    with torch.cuda.device(index):
        return function(*args, stream)


class _Fixed:
    """A configuration that stays as it was made: calls keep what they checked under it."""

    def __setattr__(self, name, value):
        if "_checked" in self.__dict__:
            raise AttributeError(f"{type(self).__name__}.{name} is fixed: make another object")
        object.__setattr__(self, name, value)


class AxialRope(_Fixed):
    """Rotary positions with several axes for heads of width ``d``.

    ``pairs``: how many pairs of channels each axis turns, e.g. ``(16, 24, 24)`` for time, height and width
    of a head of 128; channels beyond ``2 * sum(pairs)`` pass unchanged.  The i-th of an axis' n pairs turns by
    ``position * theta ** (-i / n)``.  Pairs are channels (2p, 2p + 1) with ``interleaved``, else (p, p + P).

    ``positions``: fp32 CUDA tensor [N, axes], or [B, N, axes] for positions of each batch entry.
    Q and K: [B, H, N, d] (``head_major``) or [B, N, H, d] (``token_major``), with any strides that are
    multiples of 8 elements (views of one packed projection are fine) and head counts of their own; either may be
    None.  Outputs may be the inputs (in place).
    """

    def __init__(self, d: int, pairs: Sequence[int], theta: float = 10000.0, interleaved: bool = True,
                 layout: str = "head_major", dtype: str = "bf16"):
        if layout not in ("head_major", "token_major"):
            raise ValueError("layout must be 'head_major' or 'token_major'")
        pairs = [int(p) for p in pairs]
        if not 1 <= len(pairs) <= MAX_AXES or any(p < 0 for p in pairs) or not 2 <= 2 * sum(pairs) <= int(d):
            raise ValueError(f"pairs: 1 to {MAX_AXES} axes with 1 to d / 2 = {int(d) // 2} pairs in all")
        self.d, self.pairs, self.theta, self.layout, self.dtype = int(d), tuple(pairs), float(theta), layout, dtype
        self.interleaved = bool(interleaved)
        self._torch_dtype = _torch_dtype(dtype)
        self._padded = (_i32 * MAX_AXES)(*pairs)
        self._flags = DTYPE_FP16 if dtype == "fp16" else 0
        self._lib = load_library()
        self._checked = _Checked()

    def _axes(self, t):
        """(batch, tokens, heads) axes' sizes and strides."""
        s, st = t.shape, t.stride()
        return ((s[0], s[2], s[1]), (st[0], st[2], st[1])) if self.layout == "head_major" else ((s[0], s[1], s[2]), st[:3])

    def _tensor(self, t, out, name, B, N, device):
        if t.dim() != 4 or t.shape[-1] != self.d:
            raise ValueError(f"{name}: expected four axes, the last of {self.d} channels, got {tuple(t.shape)}")
        _check_tensor(t, name, self._torch_dtype, device)
        (b, n, h), strides = self._axes(t)
        if (b, n) != (B, N):
            raise ValueError(f"{name}: expected {B} x {N} tokens, got {b} x {n}")
        if out.shape != t.shape:
            raise ValueError(f"{name}: the output's shape is {tuple(out.shape)}, the input's {tuple(t.shape)}")
        _check_tensor(out, name + " output", self._torch_dtype, device)
        return RopeTensor(None, None, h, *strides, *self._axes(out)[1])

    def _check(self, q, k, positions, q_out, k_out, backward):
        import torch
        some = q if q is not None else k
        (B, N, _), _s = self._axes(some)
        axes = len(self.pairs)
        device = some.device
        if positions.dtype != torch.float32 or not positions.is_cuda or not positions.is_contiguous() or positions.device != device:
            raise ValueError("positions: expected a contiguous fp32 CUDA tensor on the device of q and k")
        if tuple(positions.shape) == (N, axes):
            pos_batch = 0
        elif tuple(positions.shape) == (B, N, axes):
            pos_batch = N * axes
        else:
            raise ValueError(f"positions: expected {(N, axes)} or {(B, N, axes)}, got {tuple(positions.shape)}")
        if B == 0 or N == 0:
            raise ValueError("no tokens")
        tq = None if q is None else self._tensor(q, q_out, "q", B, N, device)
        tk = None if k is None else self._tensor(k, k_out, "k", B, N, device)
        return RopeDesc(B, N, self.d, axes, self._padded, self.interleaved, backward, self.theta, self._flags), tq, tk, pos_batch

    def _run(self, q, k, positions, q_out, k_out, backward, stream):
        some = q if q is not None else k
        if some is None:
            raise ValueError("neither q nor k is given")
        if some.dim() != 4:
            raise ValueError(f"expected four axes, got {tuple(some.shape)}")
        if stream is not None and some.is_cuda:
            with allocating_on(stream, some.get_device()):
                return self._run(q, k, positions, q_out, k_out, backward, None)
        look_q = look_k = None  # of outputs that are given: those made here follow from the inputs
        if q is None:
            q_out = None
        elif q_out is None:
            q_out = _like(q)
        else:
            look_q = _look(q_out)
        if k is None:
            k_out = None
        elif k_out is None:
            k_out = _like(k)
        else:
            look_k = _look(k_out)
        key = (_look(q), _look(k), _look(positions), look_q, look_k, backward)
        found = self._checked.get(key)
        if found is None:
            found = self._checked.keep(key, self._check(q, k, positions, q_out, k_out, backward))
        desc, tq, tk, pos_batch = found
        if tq is not None:
            tq = _copy(tq)
            tq.in_, tq.out = q.data_ptr(), q_out.data_ptr()
        if tk is not None:
            tk = _copy(tk)
            tk.in_, tk.out = k.data_ptr(), k_out.data_ptr()
        rc = _call(some.get_device(), self._lib.linfusion_rope, desc, tq, tk, positions.data_ptr(), pos_batch)
        if rc != OK:
            raise LinFusionError(rc, "linfusion_rope")
        return q_out, k_out

    def forward(self, q, k, positions, q_out=None, k_out=None, stream: Optional[int] = None):
        """(rotated q, rotated k), None where none was given."""
        return self._run(q, k, positions, q_out, k_out, 0, stream)

    def backward(self, dq, dk, positions, dq_out=None, dk_out=None, stream: Optional[int] = None):
        """Gradients of q and k from those of the rotated q and k."""
        return self._run(dq, dk, positions, dq_out, dk_out, 1, stream)


class BlockNorm(_Fixed):
    """The norms before and after a block of a residual stream x [B, N, C], ``a`` the block's output:

        y = residual_scale * x + gate * (Post(a) * post_weight + post_bias)       (y = x without ``a``)
        n = (Pre(y) * pre_weight + pre_bias) * (1 + scale) + shift

    ``pre`` / ``post``: "none", "layer" or "rms".  Tensors have any batch and row strides that are multiples of 8
    elements.  gate, scale and shift are [B, C] (views of one projection and expanded vectors are fine) or [C] for all batch
    entries, the weights and biases [C]; all in the storage type, absent where None.  Gradients of vectors are fp32, of the
    vector's shape.
    """

    def __init__(self, C: int, pre: Optional[str] = "layer", post: Optional[str] = "none", eps: float = 1e-6,
                 residual_scale: float = 1.0, dtype: str = "bf16"):
        for n in (pre, post):
            if n not in NORMS:
                raise ValueError("pre and post must be 'none', 'layer' or 'rms'")
        self.C, self.pre, self.post = int(C), NORMS[pre], NORMS[post]
        self.eps, self.residual_scale, self.dtype = float(eps), float(residual_scale), dtype
        self._torch_dtype = _torch_dtype(dtype)
        self._flags = DTYPE_FP16 if dtype == "fp16" else 0
        self._lib = load_library()
        self._checked = _Checked()

    def _desc(self, B, N):
        return NormDesc(B, N, self.C, self.pre, self.post, self.eps, self.residual_scale, self._flags)

    def workspace_bytes(self, B: int, N: int, sm_count: int = 0) -> int:
        """Bytes of workspace that ``backward`` takes for B x N rows."""
        n = ctypes.c_size_t(0)
        _check_rc(self._lib.linfusion_block_norm_workspace_bytes(ctypes.byref(self._desc(int(B), int(N))), int(sm_count),
                                                                 ctypes.byref(n)), "linfusion_block_norm_workspace_bytes")
        return int(n.value)

    def _rows(self, t, name, shape, device):
        if t is None:
            return None
        if tuple(t.shape) != shape:
            raise ValueError(f"{name}: expected {shape}, got {tuple(t.shape)}")
        _check_tensor(t, name, self._torch_dtype, device)
        return Rows(None, t.stride(0), t.stride(1))

    def _vector(self, t, name, B, device, per_entry):
        """Stride of a vector's batch axis."""
        _check_tensor(t, name, self._torch_dtype, device)
        if tuple(t.shape) == (self.C,):
            return 0
        if per_entry and tuple(t.shape) == (B, self.C):
            # an expanded vector has a stride of zero; a batch of one needs none of its own
            return t.stride(0) if B > 1 else self.C
        raise ValueError(f"{name}: expected {(B, self.C)} or {(self.C,)}, got {tuple(t.shape)}" if per_entry else
                         f"{name}: expected {(self.C,)}, got {tuple(t.shape)}")

    def _check(self, rows, vectors, shape, device):
        """Descriptor, row structures and vector strides for tensors whose addresses come with each call."""
        if len(shape) != 3 or shape[0] == 0 or shape[1] == 0:
            raise ValueError(f"expected [B, N, C] with at least one row, got {shape}")
        B = shape[0]
        out = [self._rows(t, name, shape, device) for name, t in rows]
        vec = NormVectors()
        for name, t in vectors:
            if t is not None:
                per_entry = name in ("gate", "scale", "shift")
                stride = self._vector(t, name, B, device, per_entry)
                if per_entry:
                    getattr(vec, name).batch = stride
        return self._desc(B, shape[1]), out, vec

    @staticmethod
    def _addresses(vec, vectors):
        vec = _copy(vec)
        for name, t in vectors:
            if t is not None:
                if name in ("gate", "scale", "shift"):
                    getattr(vec, name).p = t.data_ptr()
                else:
                    setattr(vec, name, t.data_ptr())
        return vec

    @staticmethod
    def _row_addresses(structs, rows):
        out = []
        for struct, (_, t) in zip(structs, rows):
            if struct is not None:
                struct = _copy(struct)
                struct.p = t.data_ptr()
            out.append(struct)
        return out

    def forward(self, x, a=None, gate=None, scale=None, shift=None, pre_weight=None, pre_bias=None, post_weight=None,
                post_bias=None, y=None, n=None, stream: Optional[int] = None) -> Tuple:
        """(y, n): the stream after the block (``x`` itself without ``a``) and the next block's input (None
        without ``pre``).  ``y`` may be given as ``x`` or ``a`` (in place)."""
        if stream is not None and x.is_cuda:
            with allocating_on(stream, x.get_device()):
                return self.forward(x, a, gate, scale, shift, pre_weight, pre_bias, post_weight, post_bias, y, n)
        vectors = (("gate", gate), ("scale", scale), ("shift", shift), ("pre_weight", pre_weight), ("pre_bias", pre_bias),
                   ("post_weight", post_weight), ("post_bias", post_bias))
        # outputs that are made here follow from the inputs
        key = (_look(x), _look(a), _look(y), _look(n), *[_look(t) for _, t in vectors])
        if a is not None and y is None:
            y = _like(x)
        if self.pre != NORM_NONE and n is None:
            n = _like(x)
        rows = (("x", x), ("a", a), ("y", y), ("n", n))
        found = self._checked.get(key)
        if found is None:
            found = self._checked.keep(key, self._check(rows, vectors, tuple(x.shape), x.device))
        desc, structs, vec = found
        rx, ra, ry, rn = self._row_addresses(structs, rows)
        rc = _call(x.get_device(), self._lib.linfusion_block_norm, desc, rx, ra, self._addresses(vec, vectors), ry, rn)
        if rc != OK:
            raise LinFusionError(rc, "linfusion_block_norm")
        return (y if a is not None else x), n

    def backward(self, y, a=None, gate=None, scale=None, shift=None, pre_weight=None, pre_bias=None, post_weight=None,
                 post_bias=None, dy=None, dn=None, dx=None, da=None, need_vectors: bool = True, workspace=None,
                 stream: Optional[int] = None) -> Dict:
        """Gradients by name: ``x``, ``a`` where it was given, and each given vector's in fp32 (``need_vectors``).

        ``y`` is the stream as ``forward`` returned it (not needed without ``pre``), ``dy`` its gradient from
        everything but ``n`` (None: zero), ``dn`` the gradient of ``n``.  ``dx`` may be given as ``dy`` and ``da`` as
        ``a`` (in place).  ``workspace``: a CUDA tensor of at least ``workspace_bytes``, else one is allocated."""
        import torch
        some = dn if dn is not None else dy
        if some is None:
            raise ValueError("neither dy nor dn is given")
        if stream is not None and some.is_cuda:
            with allocating_on(stream, some.get_device()):
                return self.backward(y, a, gate, scale, shift, pre_weight, pre_bias, post_weight, post_bias, dy, dn, dx, da, need_vectors,
                                     workspace)
        device = some.device
        vectors = (("gate", gate), ("scale", scale), ("shift", shift), ("pre_weight", pre_weight), ("pre_bias", pre_bias),
                   ("post_weight", post_weight), ("post_bias", post_bias))
        # outputs that are made here follow from the inputs
        key = (_look(y), _look(a), _look(dy), _look(dn), _look(dx), _look(da), *[_look(t) for _, t in vectors])
        if dx is None:
            dx = _like(some)
        if a is not None and da is None:
            da = _like(some)
        rows = (("y", y), ("a", a), ("dy", dy), ("dn", dn), ("dx", dx), ("da", da))
        found = self._checked.get(key)
        if found is None:
            desc, structs, vec = self._check(rows, vectors, tuple(some.shape), device)
            found = self._checked.keep(key, (desc, structs, vec, self.workspace_bytes(some.shape[0], some.shape[1], _sm_count(device.index))))
        desc, structs, vec, ws_bytes = found
        out, grads, ws = {"x": dx}, None, None
        if a is not None:
            out["a"] = da
        if need_vectors:
            # one allocation for the gradients of [C] vectors, one for those of [B, C]
            grads = NormGrads()
            for dims in (1, 2):
                names = [name for name, t in vectors if t is not None and t.dim() == dims]
                if names:
                    shape = (len(names), self.C) if dims == 1 else (len(names), some.shape[0], self.C)
                    for name, t in zip(names, torch.empty(shape, dtype=torch.float32, device=device).unbind(0)):
                        out[name] = t
                        setattr(grads, name, t.data_ptr())
                    if dims == 2:  # whatever the vectors' strides: an expanded one gets the gradient of each entry too
                        grads.per_entry = sum(PER_ENTRY[name] for name in names)
            if workspace is None:
                workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=device)
            elif not workspace.is_cuda or workspace.device != device or not workspace.is_contiguous():
                raise ValueError("workspace: expected a contiguous CUDA tensor on the device of the others")
            ws, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        ry, ra, rdy, rdn, rdx, rda = self._row_addresses(structs, rows)
        rc = _call(some.get_device(), self._lib.linfusion_block_norm_backward, desc, ry, ra, self._addresses(vec, vectors), rdy,
                   rdn, rdx, rda, grads, ws, ws_bytes if need_vectors else 0)
        if rc != OK:
            raise LinFusionError(rc, "linfusion_block_norm_backward")
        return out
