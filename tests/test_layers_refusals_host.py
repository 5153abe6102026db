"""What the layers refuse or take, as far as no GPU is needed, beyond the tests of their C entry points."""
import ctypes

import pytest
import torch

from paper_2409_02097_b200 import attn, block, build, layers

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
