"""The layers on the GPU against plain 64-bit implementations."""
import math

import pytest
import torch

import _layers_ref as ref

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


@pytest.fixture(scope="module")
def layers():
    from paper_2409_02097_b200 import layers
    return layers


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _window(t, pad=8):
    """The same values as a window of wider rows, and the whole tensor."""
    whole = torch.full((*t.shape[:-1], t.shape[-1] + 2 * pad), 7.0, dtype=t.dtype, device=t.device)
    whole[..., pad:-pad] = t
    return whole[..., pad:-pad], whole


# ---------------------------------------------------------------------------------------------- the 8-bit format
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", [(1, 8), (3, 40), (2, 5, 64), (130, 1288), (4, 3, 7, 96)])
def test_pack8_there_and_back(layers, shape, dtype):
    g = _gen(1)
    x = _randn(g, *shape) * torch.exp2(torch.randint(-30, 14, (*shape[:-1], 1), generator=g, device="cuda").float())
    x = x.to(TYPES[dtype])
    p = layers.pack8(x)
    codes, scales = ref.pack(x, TYPES[dtype])
    assert torch.equal(p.codes, codes) and torch.equal(p.scales, scales)
    assert torch.equal(p.unpack().double(), ref.unpack(codes, scales))  # exact
    again = layers.Packed8(p.codes.clone(), p.scales.clone(), dtype)
    out, whole = _window(torch.zeros_like(x))
    again.unpack(out=out)
    assert torch.equal(out, p.unpack()) and (whole[..., :8] == 7).all() and (whole[..., -8:] == 7).all()
    xw, _ = _window(x)
    q = layers.pack8(xw, out=again)
    assert q is again and torch.equal(q.codes, codes) and torch.equal(q.scales, scales)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_pack8_edges(layers, dtype):
    t = TYPES[dtype]
    f = torch.finfo(t)
    x = torch.zeros(9, 64, device="cuda", dtype=t)
    x[1], x[2, ::3], x[3, 5] = f.max, -f.max, math.nan
    x[4], x[4, 40] = torch.linspace(-2, 2, 64, device="cuda").to(t), -math.inf
    x[5] = f.tiny
    x[6, 0], x[6, 1] = f.smallest_normal * f.eps, 1.0     # the smallest number beside one
    x[7, :32] = torch.tensor([127.0, 126.5, 63.5, 0.5], device="cuda").repeat(8).to(t)  # ties go to even
    x[8, :32] = 127.5 if dtype == "fp16" else 128.0        # just above 127 steps of one
    p = layers.pack8(x)
    codes, scales = ref.pack(x, t)
    assert torch.equal(p.codes, codes) and torch.equal(p.scales, scales)
    got, want = p.unpack().double(), ref.unpack(codes, scales)
    assert torch.equal(torch.nan_to_num(got, 99.0), torch.nan_to_num(want, 99.0)) and torch.equal(got.isnan(), want.isnan())


# ---------------------------------------------------------------------------------------------- the product
def _linear_inputs(M, K, N, dtype, transposed, seed=2):
    g, t = _gen(seed), TYPES[dtype]
    x = _randn(g, M, K).to(t)
    w = (_randn(g, N, K) / math.sqrt(K)).to(t).t() if transposed else (_randn(g, K, N) / math.sqrt(K)).to(t)
    bias, residual, dy = (0.3 * _randn(g, N)).to(t), _randn(g, M, N).to(t), _randn(g, M, N).to(t)
    return x, w, bias, residual, dy


def _products(x, w):
    """x w in 64 bits, and the sizes that enter it."""
    return x.double() @ w.double(), x.double().abs() @ w.double().abs()


def _forward_reference(x, w, bias, residual, act):
    u, size = _products(x, w)
    if bias is not None:
        u, size = u + bias.double(), size + bias.double().abs()
    # fp32 sums of K terms, each addition off by a unit in the last place at most (the tensor cores truncate); slopes of the
    # activations are below 1.13.  The activations themselves: 3e-7 of |u| / 2 (gelu), a few units otherwise.
    slack_u = (x.shape[1] + 4) * 2.0 ** -23 * size
    y = ref.act(u, act)
    slack = 1.13 * slack_u + (0.0 if act in ("none", "relu") else 4e-7) * u.abs()
    if residual is not None:
        y, slack = y + residual.double(), slack + 2.0 ** -23 * (y.abs() + residual.double().abs())
    return u, slack_u, y, slack


SIZES = [(1, 8, 8), (2, 1280, 1280), (5, 2560, 24), (127, 64, 72), (129, 72, 136), (300, 328, 200), (257, 640, 520), (1000, 40, 1288), (2458, 2184, 1240)]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("case", range(5))
def test_linear_forward(layers, size, case):
    act, dtype, transposed = ACTS[case], ("bf16", "fp16")[case % 2], case in (1, 2, 4)
    M, K, N = size
    x, w, bias, residual, _ = _linear_inputs(M, K, N, dtype, transposed)
    bias, residual = (None if case == 2 else bias), (residual if case in (0, 2, 3) else None)
    save = (None, "full", "packed", "packed", "full")[case]
    lin = layers.Linear(K, N, act, dtype)
    y, kept = lin.forward(x, w, bias, residual, save=save)
    u, slack_u, want, slack = _forward_reference(x, w, bias, residual, act)
    ref.assert_rounded(y, want, slack, "y")
    if save == "full":
        ref.assert_rounded(kept, u, slack_u, "u")
    elif save == "packed":
        most = torch.cat([u[:, c:c + 32].abs().amax(-1, keepdim=True).expand(-1, min(32, N - c)) for c in range(0, N, 32)], -1)
        # half a step, whose size the error of the largest value may double
        ref.assert_near(kept.unpack(), u, (most + slack_u) / 127 * 1.01 + 2 * slack_u + 2.0 ** -24, "u in 8 bits")
        assert torch.equal(torch.as_tensor(kept.scales.shape), torch.tensor([M, -(-N // 32)]))
    else:
        assert kept is None
    again, _ = lin.forward(x, w, bias, residual)
    assert torch.equal(y, again)  # the same bits every time
    assert layers.expired() == 0


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("case", range(5))
def test_linear_backward(layers, size, case):
    act, dtype, transposed = ACTS[case], ("fp16", "bf16")[case % 2], case in (0, 3, 4)
    M, K, N = size
    x, w, bias, _, dy = _linear_inputs(M, K, N, dtype, transposed, seed=3)
    t = TYPES[dtype]
    u = (x.double() @ w.double() + bias.double()).to(t)
    packed = case in (1, 3)
    lin = layers.Linear(K, N, act, dtype)
    px, pu = (layers.pack8(x), layers.pack8(u)) if packed else (x, u)
    got = lin.backward(dy, px, w, u=pu if act != "none" else None)
    if packed:
        x, u = px.unpack(), pu.unpack()
        same = lin.backward(dy, x, w, u=u)
        assert all(torch.equal(got[n], same[n]) for n in same)  # a checkpoint is read as the values that it stands for
    slope = ref.act_slope(u.double(), act)
    du = dy.double() * slope
    # the slope is good to 1e-6 of itself or of one; du is rounded to 16 bits before the products, whose sums are off as above
    slope_slack = (0.0 if act in ("none", "relu") else 1e-6) * dy.double().abs() * (1 + u.double().abs())
    du_slack = (0.0 if act == "none" else ref.HALF_STEP[t]) * (du.abs() + slope_slack) + slope_slack + ref.SMALLEST[t]
    xd, wd = x.double().abs(), w.double().abs()
    ref.assert_rounded(got["x"], du @ w.double().t(), du_slack @ wd.t() + (N + 4) * 2.0 ** -23 * ((du.abs() + du_slack) @ wd.t()), "dx")
    ref.assert_rounded(got["w"], x.double().t() @ du, xd.t() @ du_slack + (M + 4) * 2.0 ** -23 * (xd.t() @ (du.abs() + du_slack)), "dw")
    assert got["w"].stride() == w.stride()
    ref.assert_near(got["bias"], du.sum(0), slope_slack.sum(0) + (M + 4) * 2.0 ** -24 * du.abs().sum(0) + 2.0 ** -22 * du.abs().sum(0), "dbias")
    again = lin.backward(dy, px, w, u=pu if act != "none" else None)
    assert all(torch.equal(got[n], again[n]) for n in got)
    for need in (("x",), ("w",), ("bias",), ("bias", "x")):
        part = lin.backward(dy, px if "w" in need else None, w, u=pu if act != "none" else None, need=need)
        assert set(part) == set(need) and all(torch.equal(part[n], got[n]) for n in need)
    assert layers.expired() == 0


def test_linear_cuts_tiles_that_do_not_fill_the_machine(layers):
    """Sizes whose tiles are cut along K take a workspace; any content of it gives the same result."""
    M, K, N = 2458, 2184, 1240
    lin = layers.Linear(K, N)
    assert lin.workspace_bytes(640, True) > 0 and layers.Linear(8192, 1280).workspace_bytes(512) > 0
    x, w, bias, residual, _ = _linear_inputs(512, 8192, 1280, "bf16", False)
    lin = layers.Linear(8192, 1280)
    outs = []
    for fill in (0, 255, 1):
        ws = torch.full((lin.workspace_bytes(512),), fill, dtype=torch.uint8, device="cuda")
        outs.append(lin.forward(x, w, bias, residual, workspace=ws)[0])
        outs.append(lin.forward(x, w, bias, residual, workspace=ws)[0])
    assert all(torch.equal(outs[0], o) for o in outs)
    _, _, want, slack = _forward_reference(x, w, bias, residual, "none")
    ref.assert_rounded(outs[0], want, slack, "y")


def test_linear_strides_and_places(layers):
    M, K, N = 203, 136, 200
    x, w, bias, residual, dy = _linear_inputs(M, K, N, "bf16", False)
    lin = layers.Linear(K, N, "silu")
    want, u = lin.forward(x, w, bias, residual, save="full")
    xw, _ = _window(x)
    ww, _ = _window(w)
    rw, _ = _window(residual)
    y, whole = _window(torch.zeros_like(residual))
    uw, whole_u = _window(torch.zeros_like(residual))
    got, kept = lin.forward(xw, ww, bias, rw, save="full", y=y, u=uw)
    assert got is y and torch.equal(y, want) and torch.equal(kept, u)
    for t in (whole, whole_u):
        assert (t[:, :8] == 7).all() and (t[:, -8:] == 7).all()  # beside the window nothing is written
    place = residual.clone()
    lin.forward(x, w, bias, place, y=place)
    assert torch.equal(place, want)
    three = lin.forward(x.view(7, 29, K), w, bias, residual.view(7, 29, N))[0]
    assert three.shape == (7, 29, N) and torch.equal(three.view(M, N), want)
    grads = lin.backward(dy, x, w, u=u)
    dx, whole_x = _window(torch.zeros_like(x))
    dw, whole_w = _window(torch.zeros_like(w))
    dyw, _ = _window(dy)
    got = lin.backward(dyw, xw, ww, u=uw, dx=dx, dw=dw)
    assert torch.equal(dx, grads["x"]) and torch.equal(dw, grads["w"]) and torch.equal(got["bias"], grads["bias"])
    for t in (whole_x, whole_w):
        assert (t[:, :8] == 7).all() and (t[:, -8:] == 7).all()


def test_a_single_row_without_leading_axes(layers):
    x, w, bias, residual, dy = _linear_inputs(1, 64, 40, "bf16", False)
    lin = layers.Linear(64, 40, "silu")
    y, u = lin.forward(x, w, bias, residual, save="packed")
    y1, u1 = lin.forward(x[0], w, bias, residual[0], save="packed")
    assert y1.shape == (40,) and torch.equal(y1, y[0]) and torch.equal(u1.unpack(), u.unpack()[0]) and torch.equal(u1.scales, u.scales[0])
    want = lin.backward(dy, layers.pack8(x), w, u=u)
    got = lin.backward(dy[0], layers.pack8(x[0]), w, u=layers.Packed8(u1.codes, u1.scales))
    assert torch.equal(got["x"], want["x"][0]) and torch.equal(got["w"], want["w"]) and torch.equal(got["bias"], want["bias"])


def test_linear_what_is_not_finite_stays_in_its_row(layers):
    M, K, N = 140, 64, 72
    x, w, bias, _, _ = _linear_inputs(M, K, N, "fp16", True)
    for act in ACTS:
        lin = layers.Linear(K, N, act, "fp16")
        clean, _ = lin.forward(x, w, bias)
        bad = x.clone()
        bad[3, 5], bad[130, 0] = math.nan, math.inf
        got, kept = lin.forward(bad, w, bias, save="packed")
        rows = [i for i in range(M) if i not in (3, 130)]
        assert torch.equal(got[rows], clean[rows]) and got[3].isnan().all()
        assert kept.unpack()[3].isnan().all() and torch.isfinite(kept.unpack()[rows]).all()
    big = torch.full((4, 64), 60000.0, device="cuda", dtype=torch.float16)
    y, _ = layers.Linear(64, 8, "gelu", "fp16").forward(big, torch.ones(64, 8, device="cuda", dtype=torch.float16))
    assert (y == math.inf).all()  # past the storage type's range


def test_linear_refuses(layers):
    lin = layers.Linear(64, 32, "gelu")
    x, w, bias, residual, dy = _linear_inputs(16, 64, 32, "bf16", False)
    bad = [dict(x=x.half()), dict(x=x[:, :32]), dict(w=w.half()), dict(w=w[:, ::2]), dict(bias=bias.float()), dict(bias=bias[:8]), dict(residual=residual[:8]),
           dict(y=residual.half()), dict(save="packed", u=residual), dict(u=residual), dict(x=x.cpu()), dict(residual=residual.t())]
    for kw in bad:
        args = dict(x=x, w=w, bias=bias, residual=residual)
        args.update(kw)
        with pytest.raises(ValueError):
            lin.forward(**args)
    from paper_2409_02097_b200.attn import LinFusionError
    with pytest.raises(LinFusionError):
        lin.forward(x, w, bias, y=x.view(16, 64)[:, :32])       # over an input
    with pytest.raises(LinFusionError):
        lin.forward(x[:1].expand(16, 64), w, bias)              # rows on top of one another
    with pytest.raises(ValueError):
        lin.backward(dy, x, w)                                  # the pre-activation is needed
    with pytest.raises(ValueError):
        lin.backward(dy, None, w, u=residual)
    with pytest.raises(ValueError):
        lin.backward(dy, layers.pack8(x[:8]), w, u=residual)
    with pytest.raises(ValueError):
        lin.backward(dy, x, w, u=residual, need=())
    with pytest.raises(LinFusionError):
        lin.backward(dy, x, w, u=residual, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))


# ---------------------------------------------------------------------------------------------- the recurrence
def _recurrence_inputs(B, N, C, dtype, seed=5, padded=0, low=-7.0):
    g, t = _gen(seed), TYPES[dtype]
    proj = _randn(g, B, N, 3 * C)
    proj[..., C:2 * C] *= 1.5
    proj = proj.to(t)
    x, decay, gate = (proj[..., k * C:(k + 1) * C] for k in range(3))
    if padded:
        decay[:, N - padded:] = -math.inf
        x[:, N - padded:] = math.nan
        gate[:, N - padded:] = math.inf
    rate = torch.exp(low * torch.rand(C, generator=g, device="cuda"))
    h0, dlast, dh = _randn(g, B, C), _randn(g, B, C), _randn(g, B, N, C).to(t)
    return x, decay, gate, rate, h0, dlast, dh


def _state_slack(f):
    """A sigmoid is good to 2^-20, so is e; steps of the scan round at 2^-24 or so, three of them a token, and are remembered for
    `steps` tokens."""
    return ((2.0 ** -19 + f["steps"] * 2.0 ** -22) * f["most"]).unsqueeze(1)


def _assert_backward(got, dh, x, decay, rate, gate, h0, dlast, reverse, before=None):
    grads, sizes, f = ref.recurrence_backward(dh, x, decay, rate, gate, h0, dlast, reverse, before)
    slack = (2.0 ** -17 + f["steps"] * 2.0 ** -20)  # the state's error and the gradient's, each as above
    assert set(got) == {n for n in grads if n != "h0" or h0 is not None}
    for n in ("x", "decay", "gate"):
        if n in got:
            ref.assert_rounded(got[n], grads[n], slack.unsqueeze(1) * sizes[n], n)
    ref.assert_near(got["rate"], grads["rate"], slack.amax(0) * sizes["rate"], "rate")
    if h0 is not None:
        ref.assert_near(got["h0"], grads["h0"], slack * sizes["h0"] + 1e-30, "h0")


SEQUENCES = [(1, 1, 8), (8, 1, 1280), (2, 7, 40), (3, 8, 64), (2, 9, 64), (2, 63, 72), (1, 64, 136), (2, 65, 64), (2, 129, 200), (3, 531, 328), (1, 1500, 24)]


@pytest.mark.parametrize("shape", SEQUENCES)
@pytest.mark.parametrize("case", range(4))
def test_recurrence_forward(layers, shape, case):
    B, N, C = shape
    dtype, reverse, gated, first = ("bf16", "fp16")[case % 2], case in (1, 2), case != 2, case in (0, 1)
    padded = N // 3 if case == 3 else 0
    x, decay, gate, rate, h0, _, _ = _recurrence_inputs(B, N, C, dtype, padded=padded)
    gate, h0 = (gate if gated else None), (h0 if first else None)
    rec = layers.GatedRecurrence(C, reverse, dtype)
    h, last, state = rec.forward(x, decay, rate, gate=gate, h0=h0, save=True)
    f = ref.recurrence(x, decay, rate, gate, h0, reverse)
    slack = _state_slack(f)
    ref.assert_rounded(h, f["h"], slack.expand_as(f["h"]), "h")
    ref.assert_near(last, f["last"], slack[:, 0] + 1e-30, "last")
    ref.assert_near(state, f["state"], slack.expand_as(f["state"]) + 1e-30, "state")
    again = rec.forward(x, decay, rate, gate=gate, h0=h0)
    assert torch.equal(again[0], h) and torch.equal(again[1], last) and again[2] is None


@pytest.mark.parametrize("shape", SEQUENCES)
@pytest.mark.parametrize("case", range(4))
def test_recurrence_backward(layers, shape, case):
    B, N, C = shape
    dtype, reverse, gated, first = ("fp16", "bf16")[case % 2], case in (0, 3), case != 1, case in (1, 2)
    padded = N // 3 if case == 2 else 0
    x, decay, gate, rate, h0, dlast, dh = _recurrence_inputs(B, N, C, dtype, seed=6, padded=padded)
    gate, h0, dlast = (gate if gated else None), (h0 if first else None), (dlast if case != 3 else None)
    rec = layers.GatedRecurrence(C, reverse, dtype)
    state = rec.forward(x, decay, rate, gate=gate, h0=h0, save=True)[2]
    got = rec.backward(dh, x, decay, rate, gate=gate, h0=h0, state=state, dlast=dlast)
    _assert_backward(got, dh, x, decay, rate, gate, h0, dlast, reverse)
    again = rec.backward(dh, x, decay, rate, gate=gate, h0=h0, state=state, dlast=dlast)
    recomputed = rec.backward(dh, x, decay, rate, gate=gate, h0=h0, dlast=dlast)
    assert all(torch.equal(got[n], again[n]) and torch.equal(got[n], recomputed[n]) for n in got)


@pytest.mark.parametrize("shape", [(2, 5, 40), (1, 64, 64), (3, 200, 136), (2, 300, 8)])
@pytest.mark.parametrize("saved", [False, True])
def test_recurrence_backward_from_checkpoints(layers, shape, saved):
    B, N, C = shape
    x, decay, gate, rate, h0, dlast, dh = _recurrence_inputs(B, N, C, "bf16", seed=7)
    rec = layers.GatedRecurrence(C, reverse=saved)
    px, pd, pg = (layers.pack8(t) for t in (x, decay, gate))
    state = rec.forward(x, decay, rate, gate=gate, h0=h0, save=True)[2] if saved else None
    got = rec.backward(dh, px, pd, rate, gate=pg, h0=h0, state=state, dlast=dlast)
    same = rec.backward(dh, px.unpack(), pd.unpack(), rate, gate=pg.unpack(), h0=h0, state=state, dlast=dlast)
    assert all(torch.equal(got[n], same[n]) for n in same)  # a checkpoint is read as the values that it stands for
    if not saved:
        _assert_backward(got, dh, px.unpack(), pd.unpack(), rate, pg.unpack(), h0, dlast, False)


@pytest.mark.parametrize("rates", ["fast", "zero", "mixed"])
def test_recurrence_rates_outside_the_unit_range(layers, rates):
    B, N, C = 2, 150, 72
    x, decay, gate, rate, h0, dlast, dh = _recurrence_inputs(B, N, C, "fp16", seed=8)
    rate = {"fast": 1 + 20 * rate, "zero": torch.zeros_like(rate), "mixed": torch.where(torch.arange(C, device="cuda") % 3 == 0, 5 * rate, rate)}[rates]
    rec = layers.GatedRecurrence(C, dtype="fp16")
    h, last, state = rec.forward(x, decay, rate, gate=gate, h0=h0, save=True)
    f = ref.recurrence(x, decay, rate, gate, h0)
    slack = _state_slack(f)
    ref.assert_rounded(h, f["h"], slack.expand_as(f["h"]), "h")
    _assert_backward(rec.backward(dh, x, decay, rate, gate=gate, h0=h0, state=state, dlast=dlast), dh, x, decay, rate, gate, h0, dlast, False)


def test_recurrence_a_negative_rate_is_nan_in_its_channel(layers):
    x, decay, gate, rate, h0, dlast, dh = _recurrence_inputs(2, 70, 40, "bf16")
    rec = layers.GatedRecurrence(40)
    bad = rate.clone()
    bad[7] = -0.5
    others = [c for c in range(40) if c != 7]
    for n in (3, 70):
        args = dict(gate=gate[:, :n], h0=h0)
        want, got = (rec.forward(x[:, :n], decay[:, :n], r, **args)[0] for r in (rate, bad))
        assert got[..., 7].isnan().all() and torch.equal(got[..., others], want[..., others])
        want, got = (rec.backward(dh[:, :n], x[:, :n], decay[:, :n], r, **args) for r in (rate, bad))
        assert got["decay"][..., 7].isnan().all() and got["rate"][7].isnan()
        ref.assert_near(got["x"][..., others], want["x"][..., others].double(), 2.0 ** -7 * want["x"][..., others].double().abs() + 1e-6, "the other channels")


def test_recurrence_token_by_token(layers):
    B, N, C = 3, 70, 48
    x, decay, gate, rate, h0, _, _ = _recurrence_inputs(B, N, C, "bf16")
    rec = layers.GatedRecurrence(C)
    whole, last, _ = rec.forward(x, decay, rate, gate=gate, h0=h0)
    carry, steps, t = h0.clone(), [], 0
    while t < N:
        n = 1 if t < 40 else 9  # single tokens, then a few at a time
        n = min(n, N - t)
        h, out, _ = rec.forward(x[:, t:t + n], decay[:, t:t + n], rate, gate=gate[:, t:t + n], h0=carry, last=carry)
        assert out is carry
        steps.append(h)
        t += n
    f = ref.recurrence(x, decay, rate, gate, h0)
    slack = _state_slack(f)
    ref.assert_rounded(torch.cat(steps, 1), f["h"], slack.expand_as(f["h"]), "token by token")
    ref.assert_near(carry, f["last"], slack[:, 0], "the state carried")
    place = h0.clone()  # the last state over the first, with several tiles
    rec.forward(x, decay, rate, gate=gate, h0=place, last=place)
    assert torch.equal(place, last)


def test_recurrence_places(layers):
    B, N, C = 2, 130, 64
    x, decay, gate, rate, h0, dlast, dh = _recurrence_inputs(B, N, C, "bf16", seed=9)
    rec = layers.GatedRecurrence(C)
    h, _, state = rec.forward(x, decay, rate, gate=gate, h0=h0, save=True)
    proj = torch.cat([x, decay, gate], -1)
    xs = [proj[..., i * C:(i + 1) * C] for i in range(3)]
    for i in range(3):  # over each of the inputs, which lie side by side
        p = proj.clone()
        v = [p[..., k * C:(k + 1) * C] for k in range(3)]
        rec.forward(v[0], v[1], rate, gate=v[2], h0=h0, h=v[i])
        assert torch.equal(v[i], h) and all(torch.equal(v[k], xs[k]) for k in range(3) if k != i)
    want = rec.backward(dh, x, decay, rate, gate=gate, h0=h0, state=state, dlast=dlast)
    packed = torch.full((B, N, 3 * C + 16), 7.0, device="cuda", dtype=torch.bfloat16)
    v = [packed[..., 8 + k * C:8 + (k + 1) * C] for k in range(3)]
    got = rec.backward(dh, x, decay, rate, gate=gate, h0=h0, state=state, dlast=dlast, dx=v[0], ddecay=v[1], dgate=v[2])
    assert all(torch.equal(got[n], want[n]) for n in want) and (packed[..., :8] == 7).all() and (packed[..., -8:] == 7).all()
    place, p = dh.clone(), proj.clone()
    v = [p[..., k * C:(k + 1) * C] for k in range(3)]
    got = rec.backward(place, v[0], v[1], rate, gate=v[2], h0=h0, dlast=dlast, dx=place, ddecay=v[1], dgate=v[2])  # in place, states recomputed
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_recurrence_long(layers):
    """More than 32768 tiles, and offsets beyond 2^31 elements: a window of long rows."""
    N, C = 64 * 32768 + 130, 8
    g = _gen(11)
    whole = torch.empty(1, N, 1032, dtype=torch.bfloat16, device="cuda")  # 2.16e9 elements
    x, decay = whole[..., :C], whole[..., 1024:1032]
    x.copy_(_randn(g, 1, N, C))
    decay.copy_(_randn(g, 1, N, C))
    rate = torch.exp(-6 * torch.rand(C, generator=g, device="cuda"))
    for reverse in (False, True):
        rec = layers.GatedRecurrence(C, reverse)
        h, last, state = rec.forward(x, decay, rate, save=True)
        # the last 64 tiles, from the state that was kept before them
        before = state[:, -(-N // 64) - 64]
        at = N - 64 * (-(-N // 64) - 64)
        end = slice(0, at) if reverse else slice(N - at, N)
        f = ref.recurrence(x[:, end], decay[:, end], rate, None, before, reverse)
        slack = _state_slack(f)
        ref.assert_rounded(h[:, end], f["h"], slack.expand_as(f["h"]), "h")
        ref.assert_near(last, f["last"], slack[:, 0], "last")
        # and the first tokens, where nothing comes from before
        start = slice(N - 200, N) if reverse else slice(0, 200)
        f = ref.recurrence(x[:, start], decay[:, start], rate, None, None, reverse)
        ref.assert_rounded(h[:, start], f["h"], _state_slack(f).expand_as(f["h"]), "h")


def test_recurrence_refuses(layers):
    x, decay, gate, rate, h0, dlast, dh = _recurrence_inputs(2, 20, 64, "bf16")
    rec = layers.GatedRecurrence(64)
    bad = [dict(x=x.half()), dict(decay=decay[:, :10]), dict(rate=rate.half()), dict(rate=rate[:8]), dict(rate=None), dict(h0=h0[:1]), dict(gate=gate.float()),
           dict(x=layers.pack8(x)), dict(x=x[..., :32]), dict(state=torch.zeros(2, 1, 64, device="cuda")), dict(h=x.half()), dict(last=h0.double())]
    for kw in bad:
        args = dict(x=x, decay=decay, rate=rate, gate=gate, h0=h0)
        args.update(kw)
        with pytest.raises(ValueError):
            rec.forward(**args)
    with pytest.raises(ValueError):
        rec.backward(dh, layers.pack8(x), decay, rate)             # all in 8 bits or none
    with pytest.raises(ValueError):
        rec.backward(dh, x, decay, rate, dgate=gate)
    with pytest.raises(ValueError):
        rec.backward(dh, x, decay, rate, state=torch.zeros(2, 2, 64, device="cuda"))
    from paper_2409_02097_b200.attn import LinFusionError
    with pytest.raises(LinFusionError):
        rec.backward(dh, x, decay, rate, dx=decay, ddecay=decay)   # two gradients in one place
    with pytest.raises(LinFusionError):
        rec.backward(dh, x, decay, rate, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))


# ---------------------------------------------------------------------------------------------- streams, graphs, together
def _block(layers, C=64, hidden=128, dtype="bf16"):
    """A block of a projection, the recurrence, and the way out with the residual; its forward and backward pass."""
    into, rec, out = layers.Linear(C, 3 * hidden, dtype=dtype), layers.GatedRecurrence(hidden, dtype=dtype), layers.Linear(hidden, C, dtype=dtype)
    up, down = layers.Linear(C, 2 * hidden, "gelu", dtype=dtype), layers.Linear(2 * hidden, C, dtype=dtype)

    def run(s, packed):
        keep = layers.pack8 if packed else (lambda t: t)
        proj, _ = into.forward(s["x"], s["w1"], s["b1"])
        parts = [proj[..., i * hidden:(i + 1) * hidden] for i in range(3)]
        h, _, state = rec.forward(parts[0], parts[1], s["rate"], gate=parts[2], save=True)
        y, _ = out.forward(h, s["w2"], residual=s["x"])
        m, u = up.forward(y, s["w3"], s["b3"], save="packed" if packed else "full")
        z, _ = down.forward(m, s["w4"], residual=y)
        kept = [keep(t) for t in (*parts, s["x"], h, y, m)]
        g4 = down.backward(s["dz"], kept[6], s["w4"], need=("x", "w"))
        g3 = up.backward(g4["x"], kept[5], s["w3"], u=u)
        dy = (g3["x"].float() + s["dz"].float()).to(s["dz"].dtype)  # the residual's gradient
        g2 = out.backward(dy, kept[4], s["w2"], need=("x", "w"))
        dproj = torch.empty_like(proj)
        d = [dproj[..., i * hidden:(i + 1) * hidden] for i in range(3)]
        gr = rec.backward(g2["x"], kept[0], kept[1], s["rate"], gate=kept[2], state=state, dx=d[0], ddecay=d[1], dgate=d[2])
        g1 = into.backward(dproj, kept[3], s["w1"])
        dx = (g1["x"].float() + dy.float()).to(dy.dtype)
        return dict(z=z, x=dx, w1=g1["w"], b1=g1["bias"], rate=gr["rate"], w2=g2["w"], w3=g3["w"], b3=g3["bias"], w4=g4["w"])

    def state(B=2, N=200, seed=12):
        g, t = _gen(seed), TYPES[dtype]
        s = dict(x=_randn(g, B, N, C), dz=_randn(g, B, N, C), b1=0.2 * _randn(g, 3 * hidden), b3=0.2 * _randn(g, 2 * hidden))
        for n, (k, m) in dict(w1=(C, 3 * hidden), w2=(hidden, C), w3=(C, 2 * hidden), w4=(2 * hidden, C)).items():
            s[n] = _randn(g, k, m) / math.sqrt(k)
        s = {n: v.to(t) for n, v in s.items()}
        s["rate"] = torch.exp(-5 * torch.rand(hidden, generator=g, device="cuda"))
        return s

    def exact(s):
        leaves = {n: v.double().requires_grad_(n != "dz") for n, v in s.items()}
        l = leaves  # noqa: E741
        proj = l["x"] @ l["w1"] + l["b1"]
        p = [proj[..., i * hidden:(i + 1) * hidden] for i in range(3)]
        a = torch.exp(-l["rate"] * torch.sigmoid(p[1]))
        v = torch.sigmoid(p[2]) * p[0]
        h, hs = torch.zeros_like(v[:, 0]), []
        for t in range(v.shape[1]):
            h = a[:, t] * h + (1 - a[:, t]) * v[:, t]
            hs.append(h)
        y = torch.stack(hs, 1) @ l["w2"] + l["x"]
        z = torch.nn.functional.gelu(y @ l["w3"] + l["b3"]) @ l["w4"] + y
        names = [n for n in leaves if n != "dz"]
        grads = torch.autograd.grad((z * l["dz"]).sum(), [leaves[n] for n in names])
        return dict(zip(names, grads), z=z.detach())

    return run, state, exact


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("packed", [False, True])
def test_a_block_trained_from_checkpoints(layers, packed, dtype):
    run, state, exact = _block(layers, dtype=dtype)
    s = state()
    got, want = run(s, packed), exact(s)
    for n in want:
        rel = ((got[n].double() - want[n]).norm() / want[n].norm()).item()
        # six or so roundings to 16 bits on the way, each 0.6 of half a step in the 2-norm; checkpoints add errors of 0.8 % (a
        # uniform error of a step of 1 / 60 of the group's rms at most) in the gradients, of which two or three meet
        most = 6 * 0.6 * ref.HALF_STEP[TYPES[dtype]] + (0.025 if packed and n != "z" else 0.0)
        assert rel <= most, (n, rel, most)


def test_captured_and_replayed_with_new_inputs(layers):
    run, state, _ = _block(layers)
    s = state()
    want = [run(state(seed=k), True) for k in (20, 21)]
    run(s, True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(s, True)
    for k, w in zip((20, 21, 20), (want[0], want[1], want[0])):
        for n, v in state(seed=k).items():
            s[n].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], w[n]) for n in w)


def test_two_captured_calls_share_a_workspace(layers):
    K, N, M = 8192, 1280, 512
    lin = layers.Linear(K, N)
    ws = torch.zeros(lin.workspace_bytes(M), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    x, w, _, _, _ = _linear_inputs(M, K, N, "bf16", False)
    x2 = x.flip(0).contiguous()
    want, want2 = lin.forward(x, w)[0], lin.forward(x2, w)[0]
    torch.cuda.synchronize()
    graphs = []
    for t in (x, x2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = lin.forward(t, w, workspace=ws)[0]
        graphs.append((g, y))
    for _ in range(3):
        for (g, y), v in zip(graphs, (want, want2)):
            y.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, v)
    assert layers.expired() == 0


def test_on_other_streams_and_two_at_once(layers):
    run, state, _ = _block(layers)
    sets = [state(seed=30 + k) for k in range(3)]
    want = [run(s, False) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for s, stream in zip(sets, streams):
        with torch.cuda.stream(stream):
            got.append(run(s, False))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(g[n], w[n]) for n in w)
    lin = layers.Linear(64, 64)
    x, w, _, _, _ = _linear_inputs(100, 64, 64, "bf16", False)
    plain = lin.forward(x, w)[0]
    torch.cuda.synchronize()
    side = streams[0]
    y = lin.forward(x, w, stream=side.cuda_stream)[0]
    p = layers.pack8(x, stream=side.cuda_stream)
    back = p.unpack(stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(y, plain) and torch.equal(back, layers.pack8(x).unpack())


def test_one_object_in_several_threads(layers):
    import threading
    lin, rec = layers.Linear(64, 64, "silu"), layers.GatedRecurrence(64)
    sets = [(_linear_inputs(150, 64, 64, "bf16", False, seed=40 + k), _recurrence_inputs(2, 100, 64, "bf16", seed=50 + k)) for k in range(4)]
    want = [(lin.forward(a[0], a[1], a[2])[0], rec.forward(r[0], r[1], r[3], gate=r[2])[0]) for a, r in sets]
    torch.cuda.synchronize()
    wrong = []

    def work(k):
        a, r = sets[k]
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(50):
                y, h = lin.forward(a[0], a[1], a[2])[0], rec.forward(r[0], r[1], r[3], gate=r[2])[0]
                torch.cuda.current_stream().synchronize()
                if not (torch.equal(y, want[k][0]) and torch.equal(h, want[k][1])):
                    wrong.append(k)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
