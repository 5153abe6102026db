"""The layers at the edges of what they take: padding through checkpoints, large and infinite values, saturated gates and activations."""
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


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _inputs(B, N, C, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[dtype]
    x, decay, gate, dh = (_randn(g, B, N, C).to(t) for _ in range(4))
    return x, decay, gate, torch.exp(-6 * torch.rand(C, generator=g, device="cuda")), _randn(g, B, C), _randn(g, B, C), dh


@pytest.mark.parametrize("shape", [(2, 6, 40), (1, 64, 64), (2, 150, 72), (1, 700, 8)])
@pytest.mark.parametrize("case", range(4))
def test_padding_goes_through_a_checkpoint(layers, shape, case):
    """Padded tokens (decay = -inf, the rest of them anything) count for nothing in a backward pass from pack8()'s checkpoints."""
    B, N, C = shape
    dtype, reverse, saved, gated = ("bf16", "fp16")[case % 2], case in (1, 2), case in (0, 1), case != 3
    x, decay, gate, rate, h0, dlast, dh = _inputs(B, N, C, dtype, 60 + case)
    decay[:, N - N // 3:], x[:, N - N // 3:], gate[:, N - N // 3:] = -math.inf, math.nan, math.inf
    decay[0, N // 2], x[0, N // 2] = -math.inf, math.inf          # one in the middle
    decay[-1, :N // 2, 5] = -math.inf                             # and in a channel of its own
    gate = gate if gated else None
    rec = layers.GatedRecurrence(C, reverse, dtype)
    state = rec.forward(x, decay, rate, gate=gate, h0=h0, save=True)[2] if saved else None
    packed = [None if t is None else layers.pack8(t) for t in (x, decay, gate)]
    got = rec.backward(dh, packed[0], packed[1], rate, gate=packed[2], h0=h0, state=state, dlast=dlast)
    plain = [None if p is None else p.unpack() for p in packed]
    plain[1] = plain[1].masked_fill(plain[1].isnan(), -math.inf)
    assert torch.equal(plain[1] == -math.inf, decay == -math.inf)
    same = rec.backward(dh, plain[0], plain[1], rate, gate=plain[2], h0=h0, state=state, dlast=dlast)
    assert all(torch.equal(got[n], same[n]) for n in same)        # a checkpoint is read as the values that it stands for
    assert all(torch.isfinite(got[n].float()).all() for n in got)
    for n in ("x", "decay", "gate"):
        assert n not in got or (got[n][decay == -math.inf] == 0).all()
    if not saved:
        grads, sizes, f = ref.recurrence_backward(dh, plain[0], plain[1], rate, plain[2], h0, dlast, reverse)
        # as everywhere: sigmoids are good to 2^-19, the scan rounds a few times a token, remembered for `steps` tokens
        slack = 2.0 ** -17 + f["steps"] * 2.0 ** -20
        for n in ("x", "decay", "gate"):
            if n in got:
                ref.assert_rounded(got[n], grads[n], slack.unsqueeze(1) * sizes[n], n)
        ref.assert_near(got["rate"], grads["rate"], slack.amax(0) * sizes["rate"], "rate")
        ref.assert_near(got["h0"], grads["h0"], slack * sizes["h0"] + 1e-30, "h0")
