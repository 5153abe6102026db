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


def _all_values(dtype, low, high):
    """Every number of the storage type between two bounds, in rows of 64."""
    v = torch.arange(-32768, 32768, dtype=torch.int32, device="cuda").to(torch.int16).view(TYPES[dtype])
    v = v[(v.float() >= low) & (v.float() <= high)]
    return torch.cat([v, v.new_zeros(-v.numel() % 64)]).view(-1, 64)


def _tail(a):
    """Phi(-a) and the density, in 64 bits and without cancellation."""
    return 0.5 * torch.special.erfcx(a / math.sqrt(2)) * torch.exp(-a * a / 2), torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gelu_of_every_value_is_rounded_once(layers, dtype):
    """Far below zero too, where the tail of the distribution is all there is."""
    x = _all_values(dtype, -13.0, 8.0)
    y, _ = layers.Linear(64, 64, "gelu", dtype).forward(x, torch.eye(64, device="cuda", dtype=TYPES[dtype]))
    u = x.double()
    want = u.clamp(min=0) - u.abs() * _tail(u.abs())[0]
    # the exponent of exp(-u^2 / 2) is rounded three times in fp32 (122 binary digits of it at u = -13: 122 * 3 * 2^-24 ln 2 = 1.5e-5), the rest is good
    # to 1e-6
    ref.assert_rounded(y, want, 2e-5 * (u.abs() * _tail(u.abs())[0]) + 2.0 ** -24 * u.clamp(min=0), "gelu")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_slope_of_gelu_has_its_digits(layers, dtype):
    u = _all_values(dtype, -13.0, 13.0).view(1, -1)
    N = u.numel()
    lin = layers.Linear(8, N, "gelu", dtype)
    # of a single row the bias' gradient is the slope itself, in fp32
    got = lin.backward(torch.ones_like(u), None, torch.zeros(8, N, device="cuda", dtype=TYPES[dtype]), u=u, need=("bias",))["bias"]
    a = u.double().abs()[0]
    tail, density = _tail(a)
    w = tail - a * density
    want = torch.where(u[0] < 0, w, 1 - w)
    ref.assert_near(got, want, 2e-5 * (tail + a * density) + 2.0 ** -23 * (u[0] >= 0).double() + 1e-36, "the slope")
    special = torch.tensor([[math.inf, -math.inf, math.nan, 0.0, -0.0, 60000.0, -60000.0, 30.5]], device="cuda").to(TYPES[dtype])
    lin = layers.Linear(8, 8, "gelu", dtype)
    got = lin.backward(torch.ones_like(special), None, torch.zeros(8, 8, device="cuda", dtype=TYPES[dtype]), u=special, need=("bias",))["bias"]
    assert got.tolist()[:2] == [1.0, 0.0] and got[2].isnan() and got.tolist()[5:] == [1.0, 0.0, 1.0]
    assert (got[3:5] - 0.5).abs().max() <= 1e-6
    y, _ = lin.forward(torch.eye(8, device="cuda", dtype=TYPES[dtype]), torch.diag(special[0].nan_to_num(0, 0, 0)), bias=special[0])
    assert y[0, 0] == math.inf and (y[:, 1] == 0).all() and y[:, 2].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_slopes_of_large_values_are_their_limits(layers, act, dtype):
    """Finite values up to the end of the type, and infinities (a kept pre-activation that has passed fp16): no infinity times zero."""
    big = [65504.0, 200.0, 129.0, math.inf] + ([1e15, 2e19, 1e25, 3e38] if dtype == "bf16" else [1e3, 1e4, 3e4, 6e4])
    u = torch.tensor([big + [-v for v in big]], device="cuda").to(TYPES[dtype])
    lin, w = layers.Linear(8, 16, act, dtype), torch.zeros(8, 16, device="cuda", dtype=TYPES[dtype])
    got = lin.backward(torch.ones_like(u), None, w, u=u, need=("bias",))["bias"]
    assert got.tolist() == [1.0] * 8 + [0.0] * 8
    u = torch.full_like(u, math.nan)
    assert lin.backward(torch.ones_like(u), None, w, u=u, need=("bias",))["bias"].isnan().all()


def test_slope_of_silu_far_below_zero(layers):
    u = torch.linspace(-80, -20, 64, device="cuda").bfloat16().view(1, -1)
    lin, w = layers.Linear(8, 64, "silu"), torch.zeros(8, 64, device="cuda", dtype=torch.bfloat16)
    got = lin.backward(torch.ones_like(u), None, w, u=u, need=("bias",))["bias"]
    want = ref.act_slope(u[0].double(), "silu")
    # 116 binary digits of the exponent are rounded twice: 116 * 2 * 2^-24 ln 2 = 1e-5
    ref.assert_near(got, want, 1.5e-5 * want.abs(), "the slope")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("wide", [False, True])
def test_gradients_at_saturated_gates(layers, wide, packed, dtype):
    """Gates and decays of 6 to 24 and of -6 to -24: their gradients carry the factor 1 - sigmoid, whose digits a difference would not have."""
    B, N, C = 2, 130, 64
    x, decay, gate, rate, h0, dlast, dh = _inputs(B, N, C, dtype, 65)
    rate = rate * (3.0 if wide else 1.0)
    # the gradients are below fp16's smallest numbers else
    dh, dlast = (dh.float() * 2.0 ** 10).to(TYPES[dtype]), dlast * 2.0 ** 10
    far = torch.linspace(6, 24, N, device="cuda").view(1, N, 1) * torch.where(torch.arange(C, device="cuda") % 2 == 0, 1.0, -1.0)
    gate = (gate.float() + far).to(TYPES[dtype])
    decay = (decay.float() + far.flip(1).roll(1, 2)).to(TYPES[dtype])
    rec = layers.GatedRecurrence(C, dtype=dtype)
    keep = layers.pack8 if packed else (lambda t: t)
    kept = [keep(t) for t in (x, decay, gate)]
    got = rec.backward(dh, kept[0], kept[1], rate, gate=kept[2], h0=h0, dlast=dlast)
    x, decay, gate = (t.unpack() if packed else t for t in kept)
    grads, sizes, f = ref.recurrence_backward(dh, x, decay, rate, gate, h0, dlast)
    slack = (2.0 ** -17 + f["steps"] * 2.0 ** -20).unsqueeze(1)
    # 1 - sigmoid is good to 2^-19 of itself, as the sigmoid is
    ref.assert_rounded(got["decay"], grads["decay"], slack * sizes["decay"] * torch.sigmoid(-decay.double()), "decay")
    ref.assert_rounded(got["gate"], grads["gate"], slack * sizes["gate"] * torch.sigmoid(-gate.double()), "gate")
    ref.assert_rounded(got["x"], grads["x"], slack * sizes["x"], "x")
    # in fp16 what is left of them there, rate e^-6 2^10 e^-17 or so, passes for zero
    still = (gate > 17) & (grads["gate"].abs() > 4 * ref.SMALLEST[TYPES[dtype]])
    assert (still.any() or dtype == "fp16") and (got["gate"][still] != 0).all()


@pytest.mark.parametrize("N", [3, 64, 70, 200])
def test_an_infinite_rate(layers, N):
    """The state is the token's value, and a padded token or the end of the sequence inside a tile leaves it (not infinity times zero)."""
    B, C = 2, 40
    x, decay, gate, rate, h0, dlast, dh = _inputs(B, N, C, "bf16", 66)
    decay[:, 1], x[:, 1] = -math.inf, math.nan
    rate[3::5] = math.inf
    fast = torch.arange(C, device="cuda") % 5 == 3
    rec = layers.GatedRecurrence(C)
    h, last, state = rec.forward(x, decay, rate, gate=gate, h0=h0, save=True)
    v = (torch.sigmoid(gate.double()) * x.double())[:, :, fast]
    v[:, 1] = v[:, 0]
    # the sigmoid is good to 2^-19; h + (v - h) is off by 2^-24 of |v - h| and by 2^-24 of the result: 3 * 2^-24 of the largest value at most, and on the
    # way into a tile the same once more
    slack = 2.0 ** -19 * v.abs() + 2.0 ** -21 * torch.maximum(v.abs().amax(), h0.abs().amax()).double()
    ref.assert_rounded(h[:, :, fast], v, slack, "h")
    ref.assert_near(last[:, fast], v[:, -1], slack[:, -1], "last")
    for kept in (state, None):
        got = rec.backward(dh, x, decay, rate, gate=gate, h0=h0, state=kept, dlast=dlast)
        assert all(torch.isfinite(t.float()).all() for t in got.values())
        assert (got["rate"][fast] == 0).all() and (got["h0"][:, fast] == 0).all() and (got["decay"][:, :, fast] == 0).all()
        G = dh.double()[:, :, fast]
        G[:, -1] += dlast[:, fast].double()
        G[:, 0] += G[:, 1]
        G[:, 1] = 0
        want = torch.sigmoid(gate.double())[:, :, fast] * G
        ref.assert_rounded(got["x"][:, :, fast], want, 2.0 ** -18 * want.abs(), "dx")


@pytest.mark.parametrize("N", [6, 60, 200])
def test_a_rate_of_zero_hides_no_nan(layers, N):
    """Only padding does: a token that counts gives 0 * NaN, also beside a padded one."""
    B, C, at = 1, 40, 4
    x, decay, gate, rate, h0, _, _ = _inputs(B, N, C, "bf16", 67)
    rate[7] = rate[8] = 0
    decay[:, at - 1], x[:, at - 1] = -math.inf, math.nan
    rec = layers.GatedRecurrence(C)
    clean = rec.forward(x, decay, rate, gate=gate, h0=h0)[0]
    assert torch.isfinite(clean.float()).all() and (clean[..., 7:9] == h0[:, None, 7:9].bfloat16()).all()
    x[:, at, 7] = math.nan
    h, last, _ = rec.forward(x, decay, rate, gate=gate, h0=h0)
    assert h[:, at:, 7].isnan().all() and last[:, 7].isnan().all() and torch.equal(h[:, :at], clean[:, :at])
    others = [c for c in range(C) if c != 7]
    assert torch.equal(h[..., others], clean[..., others])


def test_the_bias_gradient_needs_no_weight(layers):
    g = torch.Generator(device="cuda").manual_seed(68)
    dy, u, w, x = (_randn(g, *s).bfloat16() for s in ((70, 40), (70, 40), (24, 40), (70, 24)))
    for act in ("none", "silu"):
        lin = layers.Linear(24, 40, act)
        want = lin.backward(dy, x, w, u=u)["bias"]
        assert torch.equal(lin.backward(dy, None, None, u=u, need=("bias",))["bias"], want)
        assert torch.equal(lin.backward(dy, None, u=u, need=("bias",))["bias"], want)
        for need in (("x",), ("w",), ("w", "bias")):
            with pytest.raises(ValueError, match="w: needed"):
                lin.backward(dy, x, None, u=u, need=need)


def test_refusals_name_the_tensor(layers):
    from paper_2409_02097_b200.attn import LinFusionError
    lin = layers.Linear(64, 32)
    x, w, dy = (torch.zeros(*s, device="cuda", dtype=torch.bfloat16) for s in ((16, 64), (64, 32), (16, 32)))
    with pytest.raises(LinFusionError, match="x: rows on top"):
        lin.forward(x[:1].expand(16, 64), w)
    with pytest.raises(LinFusionError, match="dy: rows on top"):
        lin.backward(dy[:1].expand(16, 32), x, w)
    with pytest.raises(LinFusionError, match="w: not on a boundary"):
        lin.forward(x, torch.zeros(64 * 32 + 4, device="cuda", dtype=torch.bfloat16)[4:].view(64, 32))
    wide = torch.zeros(2, 20, 68, device="cuda", dtype=torch.bfloat16)[..., :64]
    rec, rate = layers.GatedRecurrence(64), torch.ones(64, device="cuda")
    good = torch.zeros(2, 20, 64, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(LinFusionError, match="decay: a stride of 68"):
        rec.forward(good, wide, rate)
    with pytest.raises(LinFusionError, match="h: rows on top"):
        rec.forward(good, good, rate, h=torch.zeros(1, 20, 64, device="cuda", dtype=torch.bfloat16).expand(2, 20, 64))
    with pytest.raises(LinFusionError, match="x: a stride of 68"):
        layers.pack8(wide)
    with pytest.raises(LinFusionError, match="out: a stride of 68"):
        layers.pack8(good).unpack(out=wide)


@pytest.mark.parametrize("case", range(4))
def test_long_sums_keep_their_digits(layers, case):
    """Last and kept states and the gradients that sum over all tokens, in the 2-norm, where states remember a thousand tokens and more."""
    B, N, C = 2, 4099, 64
    dtype, reverse, fast = ("bf16", "fp16")[case % 2], case in (1, 2), case == 3
    x, decay, gate, rate, h0, dlast, dh = _inputs(B, N, C, dtype, 69)
    g = torch.Generator(device="cuda").manual_seed(70)
    rate = torch.exp((3 if fast else -7) * torch.rand(C, generator=g, device="cuda"))
    rec = layers.GatedRecurrence(C, reverse, dtype)
    h, last, state = rec.forward(x, decay, rate, gate=gate, h0=h0, save=True)
    grads, _, f = ref.recurrence_backward(dh, x, decay, rate, gate, h0, dlast, reverse)
    off = lambda got, want: ((got.double() - want).norm() / want.norm()).item()  # noqa: E731
    # a sigmoid is off by 2^-20 at most (1e-6); a step rounds the state, 2^-25 of it in the mean, and up to 2 e^7 = 2200 steps are remembered:
    # sqrt(2200 / 2) * 2^-25 = 1e-6.  Twice their sum for a state, once more for a gradient, which has those of G and of the state
    assert off(last, f["last"]) <= 4e-6 and off(state, f["state"]) <= 4e-6
    for kept in (state, None):
        got = rec.backward(dh, x, decay, rate, gate=gate, h0=h0, state=kept, dlast=dlast)
        assert off(got["rate"], grads["rate"]) <= 6e-6
        # with fast decays nothing of the gradient arrives at the first state but products of thousands of factors
        assert fast or off(got["h0"], grads["h0"]) <= 6e-6
        for n in ("x", "decay", "gate"):
            assert off(got[n], grads[n]) <= 0.7 * ref.HALF_STEP[TYPES[dtype]] + 6e-6  # and one rounding: half a step at most, 0.6 of that in the mean


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_silu_and_gelu_tanh_of_every_value_are_rounded_once(layers, act, dtype):
    x = _all_values(dtype, -80.0 if act == "silu" else -9.0, 8.0)
    y, _ = layers.Linear(64, 64, act, dtype).forward(x, torch.eye(64, device="cuda", dtype=TYPES[dtype]))
    u = x.double()
    want = u * torch.sigmoid(u if act == "silu" else 2 * math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3))
    # the exponent (116 binary digits at -80 and 96 at -9) is rounded twice, or four times: 96 * 4 * 2^-24 ln 2 = 1.6e-5
    ref.assert_rounded(y, want, 2e-5 * want.abs(), act)


def test_the_rates_gradient_over_many_tiles(layers):
    """States that remember dozens of tiles, over a thousand of them: what a tile's decay is off by adds up in the rates' gradients."""
    B, N, C = 2, 40001, 96
    g = torch.Generator(device="cuda").manual_seed(71)
    x, decay, dh = ((_randn(g, B, N, C) * f + a).bfloat16() for f, a in ((1, 0.2), (1.5, 0), (1, 0)))
    rate = torch.exp(-7 * torch.sigmoid(1.5 * _randn(g, C)))
    px, pd = layers.pack8(x), layers.pack8(decay)
    got = layers.GatedRecurrence(C).backward(dh, px, pd, rate)
    want, _, _ = ref.recurrence_backward(dh, px.unpack(), pd.unpack(), rate)
    # a decay next to one is off by 2^-26 in the mean, a state by that of the 2 e^7 / 64 = 34 tiles it remembers, sqrt(17) 2^-26 = 6e-8, and as much
    # again by its own rounding; G alike.  The mean of x is ten times what the states' differences from it sum to: some 4e-7 in all, and twice that
    assert ((got["rate"].double() - want["rate"]).norm() / want["rate"].norm()).item() <= 8e-7
