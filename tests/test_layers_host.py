"""The layers as far as no GPU is needed: formulas against differences and autograd, the 8-bit format, and what the C entry points
refuse before they touch CUDA."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2409_02097_b200 import attn, block, build, layers

import _layers_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A16 = 1 << 24  # an aligned address that is never read: the calls below are refused, or find no device
NO_GPU = not torch.cuda.is_available()


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return layers.load_library()


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "linfusion_layers.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(linfusion_[a-z_0-9]+)\s*\(", text))
    assert set(layers.EXPORTED) == names
    for name in names:
        assert hasattr(lib, name)


# ------------------------------------------------------------------ formulas
@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu", "gelu_tanh"])
def test_slopes_are_those_of_the_activations(kind):
    u = torch.linspace(-6, 6, 121, dtype=torch.float64) + 0.013
    d = (ref.act(u + 1e-5, kind) - ref.act(u - 1e-5, kind)) / 2e-5
    assert (d - ref.act_slope(u, kind)).abs().max() < 1e-9


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("gated", [False, True])
def test_recurrence_gradients_against_autograd_and_differences(gated, reverse):
    g = torch.Generator().manual_seed(3)
    B, N, C = 2, 9, 3
    names = ["x", "decay", "rate", "h0"] + (["gate"] if gated else [])
    t = {n: torch.randn(B, N, C, generator=g, dtype=torch.float64) for n in ("x", "decay", "gate")}
    t["rate"], t["h0"] = torch.rand(C, generator=g, dtype=torch.float64), torch.randn(B, C, generator=g, dtype=torch.float64)
    dh, dlast = torch.randn(B, N, C, generator=g, dtype=torch.float64), torch.randn(B, C, generator=g, dtype=torch.float64)

    def loss(**t):
        f = ref.recurrence(t["x"], t["decay"], t["rate"], t.get("gate"), t["h0"], reverse)
        return (f["h"] * dh).sum() + (f["last"] * dlast).sum()

    t = {n: t[n] for n in names}
    grads, _, _ = ref.recurrence_backward(dh, t["x"], t["decay"], t["rate"], t.get("gate"), t["h0"], dlast, reverse)
    for n in names:
        for i in range(t[n].numel()):
            up, down = t[n].clone(), t[n].clone()
            up.view(-1)[i] += 1e-5
            down.view(-1)[i] -= 1e-5
            d = (loss(**{**t, n: up}) - loss(**{**t, n: down})) / 2e-5
            assert abs(d - grads[n].view(-1)[i]) <= 1e-8 * (1 + abs(d)), (n, i)  # differences: h^2 + 1e-16 / h


def test_a_padded_token_leaves_the_state():
    x = torch.tensor([[[1.0], [math.nan], [2.0]]])
    decay = torch.tensor([[[0.0], [-math.inf], [0.0]]])
    f = ref.recurrence(x, decay, torch.tensor([0.5]))
    assert f["h"][0, 1] == f["h"][0, 0] and torch.isfinite(f["h"]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_8_bit_values_are_numbers_of_the_storage_type(dtype):
    g = torch.Generator().manual_seed(4)
    x = (torch.randn(64, 72, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-20, 12, (64, 1), generator=g).double())).to(dtype)
    x[0], x[1, :3], x[2] = 0, torch.tensor([math.inf, -math.inf, math.nan]).to(dtype), torch.finfo(dtype).max
    x[3] = torch.finfo(dtype).tiny
    codes, scales = ref.pack(x, dtype)
    v = ref.unpack(codes, scales)
    assert torch.equal(torch.isnan(v), ~torch.isfinite(x.double()))
    fine = torch.isfinite(v)
    assert torch.equal(v[fine], v.to(dtype).double()[fine])  # rounds nothing
    most = torch.where(fine, x.double().abs(), torch.zeros_like(v))
    most = torch.cat([most[:, c:c + 32].amax(-1, keepdim=True).expand(-1, min(32, 72 - c)) for c in range(0, 72, 32)], -1)
    # a step is at most 2 most / 127, so half of one most / 127; above 127 steps of the largest kind a value is off by what passes
    # 127 of them, less than one; at the bottom of the range half of the smallest step
    assert ((v - x.double()).abs()[fine] <= most[fine] / 127 + 2.0 ** (ref.EXPONENTS[dtype][0] - 1)).all()


# ------------------------------------------------------------------ refusals: the 8-bit format
def _pack(lib, unpack=False, B=2, N=8, C=64, flags=0, p=A16, batch=512, row=64, codes=4 * A16, scales=8 * A16):
    desc, rows, packed = layers.Pack8Desc(B, N, C, flags), block.Rows(p, batch, row), layers.Packed8Struct(codes, scales)
    if unpack:
        return lib.linfusion_unpack8(ctypes.byref(desc), ctypes.byref(packed), ctypes.byref(rows), None)
    return lib.linfusion_pack8(ctypes.byref(desc), ctypes.byref(rows), ctypes.byref(packed), None)


@pytest.mark.parametrize("unpack", [False, True])
@pytest.mark.parametrize("kw", [dict(B=0), dict(N=-1), dict(C=0), dict(C=60), dict(p=0), dict(p=A16 + 8), dict(codes=0), dict(codes=A16 * 4 + 8), dict(scales=0),
                                dict(row=60), dict(batch=-8), dict(codes=A16 + 16), dict(scales=A16 + 1024), dict(scales=4 * A16 + 1000)])
def test_pack8_refuses_bad_arguments(lib, kw, unpack):
    assert _pack(lib, unpack, **kw) == attn.ERR_INVALID_ARG


def test_pack8_refuses_what_it_does_not_serve(lib):
    assert _pack(lib, flags=1) == attn.ERR_UNSUPPORTED
    assert _pack(lib, B=1 << 20, N=1 << 12) == attn.ERR_UNSUPPORTED          # 2^33 groups
    assert _pack(lib, unpack=True, row=32) == attn.ERR_INVALID_ARG           # rows of the output on top of one another
    if NO_GPU:
        assert _pack(lib, row=0, batch=0) == attn.ERR_CUDA                   # an input may repeat a row
        assert _pack(lib) == attn.ERR_CUDA and _pack(lib, True) == attn.ERR_CUDA


# ------------------------------------------------------------------ refusals: the recurrence
def _rows(p, batch=4096 * 3, row=64):
    return block.Rows(p, batch, row)


def _in(p=None, batch=4096 * 3, row=64, codes=None, scales=None):
    return layers.RecurrenceInput(block.Rows(p, batch, row), layers.Packed8Struct(codes, scales))


def _ref(s):
    return None if s is None else ctypes.byref(s)


def _forward(lib, B=2, N=192, C=64, reverse=0, flags=0, x=None, decay=None, gate=None, rate=20 * A16, h0=None, h=None, last=None, state=None,
             ws=30 * A16, size=None):
    desc = layers.RecurrenceDesc(B, N, C, reverse, flags)
    if size is None:
        n = ctypes.c_size_t(0)
        lib.linfusion_recurrence_workspace_bytes(ctypes.byref(desc), 0, ctypes.byref(n))
        size = n.value
    return lib.linfusion_recurrence(ctypes.byref(desc), _ref(x or _in(A16)), _ref(decay or _in(2 * A16)), _ref(gate), rate, h0, _ref(h or _rows(4 * A16)), last,
                                    state, ws, size, None)


@pytest.mark.parametrize("kw", [
    dict(B=0), dict(N=0), dict(C=0), dict(C=36), dict(reverse=2), dict(x=_in(A16 + 8)), dict(x=_in(A16, row=60)), dict(decay=_in(None)),
    dict(decay=_in(2 * A16, batch=-8)), dict(rate=None), dict(rate=20 * A16 + 4), dict(h0=21 * A16 + 8), dict(last=22 * A16 + 4), dict(state=23 * A16 + 4),
    dict(h=_rows(None)), dict(h=_rows(4 * A16, row=32)), dict(h=_rows(4 * A16, row=0)), dict(h=_rows(A16 + 128)), dict(h=_rows(A16, row=128, batch=4096 * 8)),
    dict(last=20 * A16), dict(last=4 * A16), dict(state=4 * A16 + 256), dict(h0=21 * A16, last=21 * A16 + 256), dict(ws=None), dict(ws=30 * A16 + 128),
    dict(ws=A16), dict(ws=4 * A16), dict(ws=20 * A16 - 256)])
def test_recurrence_refuses_bad_arguments(lib, kw):
    assert _forward(lib, **kw) == attn.ERR_INVALID_ARG


def test_recurrence_refuses_what_it_does_not_serve(lib):
    packed = _in(codes=A16, scales=2 * A16)
    assert _forward(lib, x=packed) == attn.ERR_UNSUPPORTED                       # the forward pass reads 16 bits
    assert _forward(lib, flags=2) == attn.ERR_UNSUPPORTED
    assert _forward(lib, B=65536) == attn.ERR_UNSUPPORTED
    assert _forward(lib, size=256) == attn.ERR_ALLOC
    if NO_GPU:  # refused for want of a device only: in place, side by side, the last state over the first
        side = [dict(batch=192 * 192, row=192) for _ in range(3)]
        x, d = _in(A16, **side[0]), _in(A16 + 128, **side[1])
        assert _forward(lib, x=x, decay=d, h=_rows(A16 + 256, **side[2])) == attn.ERR_CUDA
        assert _forward(lib, x=x, decay=d, h=_rows(A16, **side[2])) == attn.ERR_CUDA
        assert _forward(lib, h0=21 * A16, last=21 * A16) == attn.ERR_CUDA
        assert _forward(lib, N=64, ws=None) == attn.ERR_CUDA                       # one tile takes no workspace


def _backward(lib, B=2, N=192, C=64, x=None, decay=None, gate=None, rate=20 * A16, h0=None, state=22 * A16, dh=None, dlast=None, dx=None, dd=None, dg=None, drate=None,
              dh0=None, ws=30 * A16, size=None, grads=True):
    desc = layers.RecurrenceDesc(B, N, C, 0, 0)
    if size is None:
        n = ctypes.c_size_t(0)
        lib.linfusion_recurrence_workspace_bytes(ctypes.byref(desc), 1 if state else 2, ctypes.byref(n))
        size = n.value
    g = layers.RecurrenceGrads(dx or _rows(6 * A16), dd or _rows(7 * A16), dg or block.Rows(), drate, dh0)
    return lib.linfusion_recurrence_backward(ctypes.byref(desc), _ref(x or _in(A16)), _ref(decay or _in(2 * A16)), _ref(gate), rate, h0, state, _ref(dh or _rows(4 * A16)), dlast,
                                             _ref(g) if grads else None, ws, size, None)


@pytest.mark.parametrize("kw", [
    dict(N=0), dict(C=4), dict(grads=False), dict(x=_in(codes=A16, scales=3 * A16)), dict(x=_in(codes=A16)), dict(dh=_rows(None)), dict(dh=_rows(4 * A16 + 2)),
    dict(dx=_rows(7 * A16)), dict(dx=_rows(None)), dict(gate=_in(3 * A16)), dict(dg=_rows(8 * A16)), dict(dd=_rows(7 * A16, row=8)), dict(drate=20 * A16),
    dict(drate=6 * A16), dict(dh0=22 * A16), dict(dlast=23 * A16 + 4), dict(dx=_rows(2 * A16 + 128)), dict(ws=None), dict(ws=6 * A16), dict(ws=22 * A16)])
def test_recurrence_backward_refuses_bad_arguments(lib, kw):
    assert _backward(lib, **kw) == attn.ERR_INVALID_ARG


def test_recurrence_backward_workspace_and_places(lib):
    assert _backward(lib, size=0) == attn.ERR_ALLOC
    if NO_GPU:
        assert _backward(lib) == attn.ERR_CUDA
        assert _backward(lib, dx=_rows(4 * A16)) == attn.ERR_CUDA                  # over dh
        packed = dict(x=_in(codes=A16, scales=A16 * 9), decay=_in(codes=2 * A16, scales=A16 * 10))
        assert _backward(lib, **packed, state=None) == attn.ERR_CUDA
        three = [_rows(6 * A16 + 128 * i, batch=192 * 192, row=192) for i in range(3)]
        assert _backward(lib, gate=_in(3 * A16), dx=three[0], dd=three[1], dg=three[2]) == attn.ERR_CUDA   # windows of one tensor


def test_recurrence_workspace(lib):
    rec = layers.GatedRecurrence(64)
    assert rec.workspace_bytes(2, 64) == 0 and rec.workspace_bytes(2, 65) > 0
    assert rec.workspace_bytes(2, 1000, backward=True, state=False) > rec.workspace_bytes(2, 1000, backward=True) > 0
    with pytest.raises(ValueError):
        layers.GatedRecurrence(12)


# ------------------------------------------------------------------ refusals: the product
def _m(p, row=None):
    return layers.Matrix(p, 512 if row is None else row)


def _linear(lib, M=100, K=256, N=512, act=0, transposed=0, flags=0, x=None, w=None, bias=None, residual=None, y=None, u=None, u8=None, ws=30 * A16, size=None):
    desc = layers.LinearDesc(M, K, N, act, transposed, flags)
    n = ctypes.c_size_t(0)
    lib.linfusion_linear_workspace_bytes(ctypes.byref(desc), 0, 0, ctypes.byref(n))
    return lib.linfusion_linear(ctypes.byref(desc), _ref(x or _m(A16)), _ref(w or _m(2 * A16)), bias, _ref(residual), _ref(y or _m(4 * A16)), _ref(u), _ref(u8), ws,
                                n.value if size is None else size, None)


@pytest.mark.parametrize("kw", [
    dict(M=0), dict(K=-8), dict(N=0), dict(transposed=2), dict(x=_m(None)), dict(x=_m(A16 + 8)), dict(x=_m(A16, 248)), dict(x=_m(A16, 260)), dict(x=_m(A16, 0)), dict(w=_m(None)),
    dict(w=_m(2 * A16, 504)), dict(w=_m(2 * A16, 128), transposed=1), dict(y=_m(4 * A16, 504)), dict(y=_m(A16)), dict(y=_m(2 * A16 + 1024)), dict(bias=5 * A16 + 2),
    dict(bias=4 * A16 + 512), dict(residual=_m(4 * A16 + 16)), dict(residual=_m(4 * A16, 1024)), dict(u=_m(4 * A16)), dict(u=_m(6 * A16, 256)),
    dict(u=_m(6 * A16), u8=layers.Packed8Struct(7 * A16, 8 * A16)), dict(u8=layers.Packed8Struct(7 * A16, None)), dict(u8=layers.Packed8Struct(7 * A16 + 8, 8 * A16)),
    dict(u8=layers.Packed8Struct(7 * A16, 7 * A16 + 512)), dict(u8=layers.Packed8Struct(A16, 8 * A16))])
def test_linear_refuses_bad_arguments(lib, kw):
    assert _linear(lib, **kw) == attn.ERR_INVALID_ARG


def test_linear_refuses_what_it_does_not_serve(lib):
    for kw in (dict(K=252), dict(N=508), dict(flags=4), dict(act=5), dict(act=-1)):
        assert _linear(lib, **kw) == attn.ERR_UNSUPPORTED
    if NO_GPU:
        assert _linear(lib) == attn.ERR_CUDA
        assert _linear(lib, residual=_m(4 * A16)) == attn.ERR_CUDA                        # in place
        assert _linear(lib, M=1, x=_m(A16, 0), y=_m(4 * A16, 0)) == attn.ERR_CUDA           # the stride of one row says nothing
        assert _linear(lib, ws=None, size=0) == attn.ERR_CUDA


def _linear_backward(lib, M=100, K=256, N=512, act=3, dy=None, saved=None, w=None, dx=None, dw=None, dbias=20 * A16, ws=30 * A16, size=None, outs=True):
    desc = layers.LinearDesc(M, K, N, act, 0, 0)
    n = ctypes.c_size_t(0)
    saved = saved or layers.LinearSaved(_m(A16), _m(5 * A16))
    lib.linfusion_linear_workspace_bytes(ctypes.byref(desc), 2 if saved.x_packed.codes else 1, 0, ctypes.byref(n))
    dx, dw = (dx or _m(6 * A16), dw or _m(7 * A16)) if outs else (None, None)
    return lib.linfusion_linear_backward(ctypes.byref(desc), _ref(dy or _m(4 * A16)), ctypes.byref(saved), _ref(w or _m(2 * A16)), _ref(dx), _ref(dw), dbias, ws,
                                         n.value if size is None else size, None)


@pytest.mark.parametrize("kw", [
    dict(M=0), dict(dy=_m(None)), dict(dy=_m(4 * A16, 8)), dict(saved=layers.LinearSaved(_m(A16))), dict(saved=layers.LinearSaved(_m(None), _m(5 * A16))),
    dict(saved=layers.LinearSaved(_m(A16), _m(5 * A16), layers.Packed8Struct(8 * A16, 9 * A16))), dict(w=_m(None)), dict(dx=_m(4 * A16)), dict(dw=_m(6 * A16)),
    dict(dw=_m(7 * A16, 504)), dict(dbias=20 * A16 + 4), dict(dbias=6 * A16), dict(ws=None), dict(ws=30 * A16 + 8), dict(ws=5 * A16), dict(outs=False, dbias=None),
    dict(saved=layers.LinearSaved(x_packed=layers.Packed8Struct(8 * A16, None), u=_m(5 * A16)))])
def test_linear_backward_refuses_bad_arguments(lib, kw):
    assert _linear_backward(lib, **kw) == attn.ERR_INVALID_ARG


def test_linear_backward_workspace(lib):
    assert _linear_backward(lib, size=64) == attn.ERR_ALLOC
    lin = layers.Linear(256, 512, "gelu")
    assert lin.workspace_bytes(100, True, True) > lin.workspace_bytes(100, True) >= 100 * 512 * 2
    # a device with another count of SMs asks for its own
    for sms in (1, 8, 148, 160):
        assert lin.workspace_bytes(5000, True, sm_count=sms) >= 5000 * 512 * 2
    if NO_GPU:
        assert _linear_backward(lib) == attn.ERR_CUDA
        packed = layers.LinearSaved(x_packed=layers.Packed8Struct(8 * A16, 9 * A16), u_packed=layers.Packed8Struct(10 * A16, 11 * A16))
        assert _linear_backward(lib, saved=packed) == attn.ERR_CUDA
        assert _linear_backward(lib, outs=False) == attn.ERR_CUDA


def test_python_refuses_what_the_library_cannot_know():
    with pytest.raises(ValueError):
        layers.Linear(12, 8)
    with pytest.raises(ValueError):
        layers.Linear(8, 8, "tanh")
    with pytest.raises(ValueError):
        layers.Linear(8, 8, dtype="fp32")
    lin = layers.Linear(8, 16)
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lin.forward(x, torch.zeros(8, 16, dtype=torch.bfloat16))  # not on a GPU
    with pytest.raises(ValueError):
        lin.forward(x, x, save="half")
    with pytest.raises(AttributeError):
        lin.K = 16
    with pytest.raises(ValueError):
        layers.pack8(torch.zeros(4, 8))
    with pytest.raises(ValueError):
        layers.Packed8(torch.zeros(4, 40, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8))


def test_python_refuses_a_recurrence_without_decay():
    rec, x, rate = layers.GatedRecurrence(8), torch.zeros(1, 4, 8, dtype=torch.bfloat16), torch.ones(8)
    with pytest.raises(ValueError, match="decay: needed"):
        rec.forward(x, None, rate)
    with pytest.raises(ValueError, match="decay: needed"):
        rec.backward(x, x, None, rate)
