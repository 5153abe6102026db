"""What the layers refuse or take, as far as no GPU is needed, beyond the tests of their C entry points."""
import ctypes

import pytest
import torch

from paper_2409_02097_b200 import attn, build, layers

A16 = 1 << 24  # an aligned address that is never read: the calls below are refused, or find no device


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build_library()
    return layers.load_library()


def test_counts_beyond_32_bits_are_refused_not_cut_off(monkeypatch):
    lin, rec = layers.Linear(64, 64), layers.GatedRecurrence(64)
    assert lin.workspace_bytes(2 ** 24) >= 0
    for call in (lambda: lin.workspace_bytes(2 ** 32 + 16), lambda: lin.workspace_bytes(2 ** 31, True), lambda: rec.workspace_bytes(2 ** 32 + 1, 64),
                 lambda: rec.workspace_bytes(1, 2 ** 32 + 640), lambda: layers.Linear(2 ** 32 + 8, 8), lambda: layers.Linear(8, 2 ** 32 + 8),
                 lambda: layers.GatedRecurrence(2 ** 32 + 8)):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    monkeypatch.setattr(layers, "_check_tensor", lambda *a: None)
    big = torch.empty(2 ** 32 + 4, 8, dtype=torch.bfloat16, device="meta")
    for t in (big, big.unsqueeze(0), big.unsqueeze(1)):
        with pytest.raises(ValueError, match="32 bits"):
            layers._pack8_desc(t, "x", "bf16")


class _Stand:
    """A stand-in for a tensor of the given shape, strides and address."""

    def __init__(self, shape, strides, p=A16):
        self.shape, self._strides, self._p = torch.Size(shape), tuple(strides), p

    def stride(self, i=None):
        return self._strides if i is None else self._strides[i]

    def data_ptr(self):
        return self._p


def test_refusals_name_the_tensor():
    say = lambda apart=(), **t: str(layers._refusal(attn.ERR_INVALID_ARG, "linfusion_linear", apart, **t))  # noqa: E731
    good = _Stand((4, 64), (64, 1))
    assert "x: not on a boundary of 16" in say(w=good, x=_Stand((4, 64), (64, 1), A16 + 8))
    assert "workspace: not on a boundary of 256" in say(x=good, workspace=_Stand((512,), (1,), A16 + 16))
    assert "w: a stride of 60 elements" in say(x=good, w=_Stand((64, 60), (60, 1)))
    assert "w: a stride of 60 elements" in say(x=good, w=_Stand((60, 64), (1, 60)))
    assert "dy: rows on top of one another (0" in say(("dy",), x=good, dy=_Stand((4, 64), (0, 1)))
    assert "dy: rows on top of one another (32" in say(("dy",), x=good, dy=_Stand((2, 4, 64), (64, 32, 1)))
    nobody = say(("x", "w", "dy"), x=good, bias=None, w=_Stand((64, 40), (1, 64)), dy=_Stand((2, 4, 64), (512, 128, 1)), dh=_Stand((4, 64), (0, 1)))
    assert nobody.startswith("linfusion_linear: ") and "apart" not in nobody and "stride of" not in nobody
    assert layers._refusal(attn.ERR_ALLOC, "linfusion_linear", x=_Stand((4, 64), (60, 1))).code == attn.ERR_ALLOC


def test_strides_whose_reach_passes_every_address_are_refused(lib):
    """The range of rows is computed in 64 bits: it may not wrap and come out next to nothing."""
    M, n = 2 ** 30 + 1, ctypes.c_size_t(0)
    desc = layers.LinearDesc(M, 64, 64, 0, 0, 0)
    assert lib.linfusion_linear_workspace_bytes(ctypes.byref(desc), 0, 0, ctypes.byref(n)) == attn.OK
    far = [layers.Matrix(A16 * (1 + i), 1 << 34) for i in range(2)]  # 2^64 elements
    near = layers.Matrix(A16 * 4, 64)
    rows = [layers.Matrix(2 ** 45 * (1 + i), 64) for i in range(2)]
    for x, y in ((far[0], rows[1]), (rows[0], far[1])):
        assert lib.linfusion_linear(ctypes.byref(desc), ctypes.byref(x), ctypes.byref(near), None, None, ctypes.byref(y), None, None, 2 ** 50, n.value,
                                    None) == attn.ERR_INVALID_ARG
    if not torch.cuda.is_available():
        assert lib.linfusion_linear(ctypes.byref(desc), ctypes.byref(rows[0]), ctypes.byref(near), None, None, ctypes.byref(rows[1]), None, None, 2 ** 50, n.value,
                                    None) == attn.ERR_CUDA
