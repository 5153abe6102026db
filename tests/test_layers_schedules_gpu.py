"""The products under every schedule that the plans choose: several tiles a pair of CTAs, cut tiles, both at once, every shape of tile, and
calls that follow one another closely."""
import math

import pytest
import torch

import _layers_ref as ref

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def layers():
    from paper_2409_02097_b200 import layers
    return layers


def _randn(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


# D of each size goes to 256 x 256, 256 x 128, 128 x 128 and 128 x 64 tiles; from one chunk of K, fewer than the stages there are, to many
CLOSE = [(2500, 8, 264), (2500, 136, 2120), (282, 256, 1448), (518, 112, 1592), (130, 648, 72), (1, 1288, 8), (512, 4096, 1280)]


def test_calls_close_to_one_another(layers):
    """Launches overlap: a call's blocks come to the shared memory that the call before has just left."""
    calls = []
    for i, (M, K, N) in enumerate(CLOSE):
        x, w = _randn(70 + i, M, K).bfloat16(), (_randn(80 + i, K, N) / math.sqrt(K)).bfloat16()
        lin = layers.Linear(K, N)
        calls.append((lin, x, w, lin.forward(x, w)[0].clone()))
        want = x.double() @ w.double()
        ref.assert_rounded(calls[-1][3], want, (K + 4) * 2.0 ** -23 * (x.double().abs() @ w.double().abs()), "y")
    outs = [[lin.forward(x, w)[0] for lin, x, w, _ in calls] for _ in range(40)]
    torch.cuda.synchronize()
    for run in outs:
        assert all(torch.equal(y, want) for y, (_, _, _, want) in zip(run, calls))
    assert layers.expired() == 0


def test_flags_are_down_after_a_call(layers):
    """The workspace of a cut product begins with its flags: none is up when the call is over, whatever they held before."""
    M, K, N = 512, 8192, 1280
    lin = layers.Linear(K, N)
    x, w = _randn(90, M, K).bfloat16(), (_randn(91, K, N) / math.sqrt(K)).bfloat16()
    want = lin.forward(x, w)[0]
    for fill in (0, 255, 1):
        ws = torch.full((lin.workspace_bytes(M),), fill, dtype=torch.uint8, device="cuda")
        assert ws.numel() > 0 and torch.equal(lin.forward(x, w, workspace=ws)[0], want)
        flags = ws[:512].view(torch.int64)  # of the first blocks
        assert (flags != -1).any() and all(f in (0, int.from_bytes(bytes([fill] * 8), "little", signed=True)) for f in flags.tolist())
        if fill:
            assert (flags == 0).any()
    assert layers.expired() == 0
