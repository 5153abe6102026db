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


# (M, K, N), what the plan of 148 SMs makes of it: four and five 256 x 256 tiles for a pair of CTAs, 2.0 256 x 128 (N / 8 odd), 1.4 with K of
# five chunks, two 128 x 128 tiles a CTA, whole and cut tiles together (N / 8 odd), 76 tiles cut over 74 pairs, all of 20 tiles cut
SCHEDULES = [(9000, 136, 2120), (2500, 136, 8200), (1456, 888, 3112), (4099, 320, 1288), (4734, 8, 976), (12562, 1808, 264), (19239, 1800, 144), (512, 4096, 1272)]


@pytest.mark.parametrize("size", SCHEDULES)
@pytest.mark.parametrize("case", range(4))
def test_forward_under_every_schedule(layers, size, case):
    """With a residual, an activation and the pre-activation kept, so that what a tile has in shared and tensor memory is used again by the next."""
    act, save, dtype, transposed = (("gelu", "packed", "bf16", False), ("silu", "full", "fp16", True), ("none", "packed", "fp16", False),
                                    ("gelu_tanh", None, "bf16", True))[case]
    M, K, N = size
    t = TYPES[dtype]
    x, bias, residual = _randn(1, M, K).to(t), (0.3 * _randn(3, N)).to(t), _randn(4, M, N).to(t)
    w = (_randn(2, N, K) / math.sqrt(K)).to(t).t() if transposed else (_randn(2, K, N) / math.sqrt(K)).to(t)
    residual = residual if case != 3 else None
    lin = layers.Linear(K, N, act, dtype)
    y, kept = lin.forward(x, w, bias, residual, save=save)
    u, size_u = x.double() @ w.double() + bias.double(), x.double().abs() @ w.double().abs() + bias.double().abs()
    # sums of K terms in fp32, each addition off by a unit in the last place; slopes below 1.13; the activations good to 1e-6 of themselves and of u
    slack_u = (K + 4) * 2.0 ** -23 * size_u
    want, slack = ref.act(u, act), 1.13 * slack_u + (0.0 if act == "none" else 1e-6) * u.abs()
    if residual is not None:
        want = want + residual.double()
        slack = slack + 2.0 ** -23 * (want.abs() + residual.double().abs())
    ref.assert_rounded(y, want, slack, "y")
    if save == "full":
        ref.assert_rounded(kept, u, slack_u, "u")
    elif save == "packed":
        most = torch.cat([u[:, c:c + 32].abs().amax(-1, keepdim=True).expand(-1, min(32, N - c)) for c in range(0, N, 32)], -1)
        # half a step, whose size the error of the largest value may double
        ref.assert_near(kept.unpack(), u, (most + slack_u) / 127 * 1.01 + 2 * slack_u + 2.0 ** -24, "u in 8 bits")
    place = None if residual is None else residual.clone()
    again, kept_again = lin.forward(x, w, bias, place, save=save, y=place)  # and in place
    assert torch.equal(again, y)
    if save == "packed":
        assert torch.equal(kept.codes, kept_again.codes) and torch.equal(kept.scales, kept_again.scales)
    assert layers.expired() == 0


def test_which_forward_products_are_cut(layers):
    cut = [layers.Linear(K, N).workspace_bytes(M) > 0 for M, K, N in SCHEDULES]
    assert cut == [False, False, False, False, False, True, True, True]


# dw cut into 256 x 128 and 128 x 64 tiles; dx cut; two tiles of dw cut into 148 runs; whole and cut tiles of dw together, and of dx
BACKWARD = [(9000, 136, 2120), (4099, 320, 1288), (2500, 136, 4104), (19069, 104, 72), (4500, 2632, 3624), (1746, 1808, 2520), (7629, 536, 1760)]


@pytest.mark.parametrize("size", BACKWARD)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_backward_under_every_schedule(layers, size, transposed, dtype):
    M, K, N = size
    t = TYPES[dtype]
    x, dy = _randn(5, M, K).to(t), _randn(6, M, N).to(t)
    w = (_randn(7, N, K) / math.sqrt(K)).to(t).t() if transposed else (_randn(7, K, N) / math.sqrt(K)).to(t)
    lin = layers.Linear(K, N, "none", dtype)
    got = lin.backward(dy, x, w)
    xd, wd, dyd = x.double(), w.double(), dy.double()
    ref.assert_rounded(got["x"], dyd @ wd.t(), (N + 4) * 2.0 ** -23 * (dyd.abs() @ wd.abs().t()), "dx")
    ref.assert_rounded(got["w"], xd.t() @ dyd, (M + 4) * 2.0 ** -23 * (xd.abs().t() @ dyd.abs()), "dw")
    ref.assert_near(got["bias"], dyd.sum(0), (M + 4) * 2.0 ** -24 * dyd.abs().sum(0), "dbias")
    again = lin.backward(dy, x, w)
    assert all(torch.equal(got[n], again[n]) for n in got) and layers.expired() == 0


def test_every_backward_pass_above_has_a_cut_product(layers):
    """What a backward pass without an activation takes beyond the columns' sums (three blocks of them an SM at most) are sums of cut tiles."""
    for M, K, N in BACKWARD:
        sums = 3 * 148 * 4 * (N + 16) // -(-N // 256) + 512
        most = max(layers.Linear(K, N).workspace_bytes(M, True, transposed=side, sm_count=148) for side in (False, True))
        assert most > 2 * sums, (M, K, N)


def test_cut_products_on_two_streams_at_once(layers):
    """Each with a workspace of its own; the blocks of both share the machine, and each waits for its own."""
    sets = []
    for i, (M, K, N) in enumerate([(512, 4096, 1272), (19239, 1800, 144)]):
        x, w = _randn(100 + i, M, K).bfloat16(), (_randn(110 + i, K, N) / math.sqrt(K)).bfloat16()
        dy = _randn(120 + i, M, N).bfloat16()
        lin = layers.Linear(K, N)
        want = lin.forward(x, w)[0], lin.backward(dy, x, w)
        sets.append((lin, x, w, dy, want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for out, (lin, x, w, dy, _, stream) in zip(got, sets):
            with torch.cuda.stream(stream):
                out.append((lin.forward(x, w)[0], lin.backward(dy, x, w)))
    torch.cuda.synchronize()
    for out, (_, _, _, _, (y, grads), _) in zip(got, sets):
        for a, b in out:
            assert torch.equal(a, y) and all(torch.equal(b[n], grads[n]) for n in grads)
    assert layers.expired() == 0
