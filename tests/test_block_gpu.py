"""Rotary positions and the norms around a block against 64-bit implementations, forward and backward: widths and
lengths that do not divide the kernels' tiles, strides, shared and per-entry vectors, in-place outputs, guard bands,
streams, graphs, refusals of tensors."""
import pytest
import torch

from paper_2409_02097_b200 import block

import _block_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


# ------------------------------------------------------------------------------------------ rope
# Before its rounding an element u cos - w sin is off by the angle's error (3e-7: one turn in fp32 to 2^-25, times 2 pi, plus
# two units in the last place of the sine and cosine) and three fp32 roundings, each relative to |u| + |w|.
ROPE_SLACK = 1e-6

ROPE_CASES = [
    # B, H, Hk, N, d, pairs, interleaved, layout
    (1, 1, 1, 1, 32, (16,), True, "head_major"),
    (2, 3, 3, 7, 40, (3, 5), True, "token_major"),
    (2, 5, 1, 65, 64, (16, 16), False, "token_major"),
    (1, 4, 2, 129, 80, (10, 10, 10), False, "head_major"),   # P = 30: pieces of two elements
    (3, 2, 2, 50, 128, (16, 24, 24), False, "token_major"),  # P = 64: whole pieces
    (1, 3, 2, 33, 40, (1, 4, 7, 5), False, "token_major"),   # P = 17: single elements
    (2, 2, 2, 31, 64, (12,), False, "head_major"),           # P = 12: pieces of four, forty channels pass
    (1, 2, 2, 70, 256, (40, 44, 44), True, "head_major"),
    (1, 33, 17, 300, 160, (0, 40, 40), True, "token_major"),
    (2, 7, 7, 19, 8, (1,), False, "token_major"),
    (1, 2, 1, 5, 16, (2, 1, 2, 1), True, "head_major"),
    (2, 9, 9, 4099, 64, (8, 8, 8), True, "token_major"),
]


def _rope_case(case, dtype, seed=3, spread=700.0, per_batch=False):
    B, H, Hk, N, d, pairs, interleaved, layout = case
    gen = _gen(seed)
    shape = (lambda h: (B, h, N, d)) if layout == "head_major" else (lambda h: (B, N, h, d))
    q, k = _randn(gen, *shape(H), dtype=dtype), _randn(gen, *shape(Hk), dtype=dtype)
    pos = torch.floor(spread * torch.rand((B, N, len(pairs)) if per_batch else (N, len(pairs)), generator=gen, device="cuda"))
    return q, k, pos


def _check_rope(got, x, pos, case, backward, what, theta=10000.0, slack=ROPE_SLACK):
    _, _, _, _, _, pairs, interleaved, layout = case
    want, size = ref.rope(x, pos, pairs, theta, interleaved, layout == "head_major", backward)
    ref.assert_rounded(got, want, slack * size, what)
    assert torch.equal(got[..., 2 * sum(pairs):], x[..., 2 * sum(pairs):])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", ROPE_CASES, ids=lambda c: "x".join(map(str, c[:5])))
def test_rope_matches_64_bits(case, dtype):
    B, H, Hk, N, d, pairs, interleaved, layout = case
    op = block.AxialRope(d, pairs, interleaved=interleaved, layout=layout, dtype=dtype)
    for per_batch in (False, True):
        q, k, pos = _rope_case(case, DT[dtype], per_batch=per_batch)
        qr, kr = op.forward(q, k, pos)
        dq, dk = op.backward(q, k, pos)
        torch.cuda.synchronize()
        for got, x, back in ((qr, q, False), (kr, k, False), (dq, q, True), (dk, k, True)):
            _check_rope(got, x, pos, case, back, f"{case} {dtype} backward={back}")


def test_rope_far_and_fractional_positions():
    case = (1, 2, 1, 64, 64, (16, 16), True, "head_major")
    q, k, pos = _rope_case(case, torch.float16)
    for pos in (pos + 1.0e6, pos * 16384.0 - 5e6, pos / 3 - 100.25):
        op = block.AxialRope(64, (16, 16), dtype="fp16")
        qr, kr = op.forward(q, k, pos)
        _check_rope(qr, q, pos, case, False, "far q")
        _check_rope(kr, k, pos, case, False, "far k")
    op = block.AxialRope(64, (16, 16), theta=33.5, dtype="fp16")
    _check_rope(op.forward(q, None, pos)[0], q, pos, case, False, "theta", theta=33.5)


@pytest.mark.parametrize("interleaved,pairs", [(True, (20, 20)), (False, (20, 20)), (False, (10, 9))])
def test_rope_strides_in_place_and_guard_bands(interleaved, pairs):
    B, N, H, d = 2, 77, 3, 80
    gen = _gen(4)
    op = block.AxialRope(d, pairs, interleaved=interleaved, layout="token_major")
    pos = torch.randint(0, 99, (N, 2), generator=gen, device="cuda").float()
    case = (B, H, H, N, d, pairs, interleaved, "token_major")
    # Q and K inside one packed projection with room on both sides; V and the guard rows stay as they are
    big = _randn(gen, B + 1, N + 5, 3, H, d)
    before = big.clone()
    q, k = big[:B, 2:N + 2, 0], big[:B, 2:N + 2, 1]
    q0, k0 = q.clone(), k.clone()
    op.forward(q, k, pos, q_out=q, k_out=k)
    _check_rope(q, q0, pos, case, False, "in place q")
    _check_rope(k, k0, pos, case, False, "in place k")
    q.copy_(q0), k.copy_(k0)
    assert torch.equal(big, before)
    # into strided outputs
    out = torch.full((B, N + 2, 2, H, d), 7.0, device="cuda", dtype=torch.bfloat16)
    op.forward(q, k, pos, q_out=out[:, 1:-1, 0], k_out=out[:, 1:-1, 1])
    _check_rope(out[:, 1:-1, 0], q0, pos, case, False, "strided q")
    _check_rope(out[:, 1:-1, 1], k0, pos, case, False, "strided k")
    assert (out[:, 0] == 7).all() and (out[:, -1] == 7).all()
    # an expanded input is read, not copied
    one = _randn(gen, 1, 1, H, d)
    many = one.expand(B, N, H, d)
    _check_rope(op.forward(many, None, pos)[0], many, pos, case, False, "expanded")
    with pytest.raises(Exception):
        op.forward(many, None, pos, q_out=many)


def test_rope_round_trip_keeps_infinities_and_nan_where_they_are():
    op = block.AxialRope(64, (16, 8), interleaved=False, layout="head_major")
    q = _randn(_gen(5), 1, 2, 40, 64)
    q[0, 0, 3, 5], q[0, 1, 7, 60] = float("inf"), float("nan")
    pos = torch.arange(40, device="cuda").float()[:, None].repeat(1, 2)
    out, _ = op.forward(q, None, pos)
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[0, 0, 3, 5] = want[0, 0, 3, 29] = want[0, 1, 7, 60] = True  # the pair (5, 5 + 24); channel 60 passes
    assert torch.equal(bad & ~want, torch.zeros_like(bad)) and bad[0, 1, 7, 60] and bad[0, 0, 3, 5]


def test_rope_refuses_tensors():
    op = block.AxialRope(64, (16, 16), layout="token_major")
    q = _randn(_gen(6), 2, 8, 4, 64)
    pos = torch.zeros(8, 2, device="cuda")
    for bad in (q.half(), q[..., :32], q[:, :, :, ::2], q.cpu(), q[0], torch.empty(2, 0, 4, 64, device="cuda", dtype=q.dtype)):
        with pytest.raises(ValueError):
            op.forward(bad, None, pos)
    for p in (pos.double(), pos[:7], pos[:, :1], pos.cpu(), torch.zeros(2, 8, 2, device="cuda")[:, ::2]):
        with pytest.raises(ValueError):
            op.forward(q, None, p)
    with pytest.raises(ValueError):
        op.forward(q, q[:1], pos)
    odd = torch.zeros(2 * 8 * 4 * 64 + 8, device="cuda", dtype=torch.bfloat16)[4:-4].view(2, 8, 4, 64)  # 8-byte aligned only
    with pytest.raises(block.LinFusionError):
        op.forward(odd, None, pos)
    with pytest.raises(block.LinFusionError):
        op.forward(q, q, pos, q_out=torch.empty_like(q), k_out=q)  # K's output over Q's input


# ------------------------------------------------------------------------------------------ norms
# Each normed value is off by a few fp32 roundings of the row's largest deviation (the mean, the variance and their sums over
# at most 8192 channels in trees of eight: ten roundings) and its products by a few more.
NORM_SLACK = 16 * 2.0 ** -24

NORM_CASES = [
    # B, N, C, pre, post, a, gate, mod, affine
    (1, 1, 8, "layer", "none", False, False, "none", False),
    (2, 3, 40, "rms", "layer", True, True, "batch", True),
    (3, 65, 320, "layer", "rms", True, True, "shared", True),
    (2, 130, 640, "layer", "layer", True, False, "batch", False),
    (1, 257, 1280, "rms", "rms", True, True, "batch", True),
    (2, 1, 1280, "layer", "none", False, False, "batch", True),
    (2, 33, 264, "none", "layer", True, True, "none", True),    # two warps, the second nearly empty
    (2, 5, 72, "none", "none", True, True, "none", False),      # gate and residual alone
    (1, 9, 2056, "layer", "rms", True, True, "batch", True),    # more than 256 threads
    (1, 3, 4104, "rms", "layer", True, True, "shared", True),   # more than 512
    (1, 4, 8192, "layer", "layer", True, True, "batch", True),
    (5, 2000, 256, "layer", "rms", True, True, "batch", True),
    (4, 1031, 136, "rms", "none", True, False, "none", False),
    (2, 4099, 1152, "layer", "layer", True, True, "shared", True),
]


def _norm_case(case, dtype, seed=11, offset=0.3):
    B, N, C, pre, post, a, gate, mod, affine = case
    gen = _gen(seed)
    t = dict(x=_randn(gen, B, N, C, dtype=dtype) + offset)
    if a:
        t["a"] = _randn(gen, B, N, C, dtype=dtype) * 0.5 - offset
    vec = {}
    rows = B if mod != "shared" else 1
    m = (0.3 * torch.randn(rows, 3 * C, generator=gen, device="cuda")).to(dtype)
    m = m[0] if mod == "shared" else m
    if mod != "none" and pre != "none":
        vec["scale"], vec["shift"] = m[..., :C], m[..., C:2 * C]
    if gate:
        vec["gate"] = m[..., 2 * C:]
    if affine:
        for side, kind in (("pre", pre), ("post", post)):
            if kind != "none":
                vec[side + "_weight"] = (1 + 0.2 * torch.randn(C, generator=gen, device="cuda")).to(dtype)
                vec[side + "_bias"] = (0.2 * torch.randn(C, generator=gen, device="cuda")).to(dtype)
    return t, vec


def _norm_op(case, dtype, rs=0.75):
    B, N, C, pre, post, *_ = case
    return block.BlockNorm(C, pre=pre, post=post, eps=1e-5, residual_scale=rs, dtype=dtype)


def _dbl(d):
    return {n: v.double() for n, v in d.items()}


def _check_norm_forward(case, t, vec, y, n, rs=0.75, eps=1e-5):
    _, _, C, pre, post, a, *_ = case
    t, v = _dbl(t), _dbl(vec)
    want = t["x"]
    if a:
        want = ref.norm_after(t["x"], t["a"], v, post, eps, rs)
        h = ref.normed(t["a"], post, eps)
        gate = ref.over_rows(v["gate"]).abs() if "gate" in v else 1.0
        top = h.abs().amax(-1, keepdim=True) if post != "none" else h.abs()
        size = (rs * t["x"]).abs() + gate * (top * (1 + v.get("post_weight", torch.ones(())).abs().to(h.device)) + _abs(v.get("post_bias")))
        ref.assert_rounded(y, want, NORM_SLACK * size, f"y {case}")
        want = y.double()
    if pre != "none":
        h = ref.normed(want, pre, eps)
        out = ref.norm_before(want, v, pre, eps)
        s = 1 + ref.over_rows(v["scale"]).abs() if "scale" in v else 1.0
        b = ref.over_rows(v["shift"]).abs() if "shift" in v else 0.0
        size = s * (h.abs().amax(-1, keepdim=True) * (1 + _abs(v.get("pre_weight"))) + _abs(v.get("pre_bias"))) + b
        ref.assert_rounded(n, out, NORM_SLACK * size, f"n {case}")
    else:
        assert n is None


def _abs(v):
    return 0.0 if v is None else v.abs()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", NORM_CASES, ids=lambda c: "-".join(map(str, c[:5])))
def test_norm_forward_matches_64_bits(case, dtype):
    t, vec = _norm_case(case, DT[dtype])
    y, n = _norm_op(case, dtype).forward(t["x"], t.get("a"), **vec)
    torch.cuda.synchronize()
    if not case[5]:
        assert y is t["x"]
    _check_norm_forward(case, t, vec, y, n)


def _reference_backward(case, t, vec, y, dy, dn, rs=0.75, eps=1e-5):
    """Gradients in 64 bits by differentiation of the definition; and the sums of their terms' absolute values for vectors."""
    _, _, C, pre, post, a, *_ = case
    v = {n: x.double().requires_grad_(True) for n, x in vec.items()}
    out = {}
    total = dy.double() if dy is not None else torch.zeros_like(dn, dtype=torch.float64)
    if pre != "none":
        leaf = y.double().requires_grad_(True)
        names = [n for n in v if n.startswith("pre_") or n in ("scale", "shift")]
        got = torch.autograd.grad((ref.norm_before(leaf, v, pre, eps) * dn.double()).sum(), [leaf] + [v[n] for n in names])
        total = total + got[0]
        out.update(zip(names, got[1:]))
    if not a:
        out["x"] = total
        return out, total
    leaves = [torch.zeros_like(total).requires_grad_(True), t["a"].double().requires_grad_(True)]
    names = [n for n in v if n.startswith("post_") or n == "gate"]
    got = torch.autograd.grad((ref.norm_after(leaves[0], leaves[1], v, post, eps, rs) * total).sum(), leaves + [v[n] for n in names])
    out.update(zip(["x", "a"] + names, got))
    return out, total


def _check_norm_backward(case, t, vec, y, dy, dn, got, rs=0.75, eps=1e-5):
    B, N, C, pre, post, a, *_ = case
    want, total = _reference_backward(case, t, vec, y, dy, dn, rs, eps)
    assert set(want) == set(got), (set(want), set(got))
    v = _dbl(vec)
    s = 1 + ref.over_rows(v["scale"]).abs() if "scale" in v else 1.0
    # the gradient through a norm: rstd times (g, its mean, h times the mean of g h), each of the size of the row's largest
    def through(x, g, kind):
        x, g = x.double(), g.abs()
        var = (x - x.mean(-1, keepdim=True)).square().mean(-1, keepdim=True) if kind == "layer" else x.square().mean(-1, keepdim=True)
        h = ref.normed(x, kind, eps).abs()
        top = g.amax(-1, keepdim=True)
        return (2 * top + h * (g * h).mean(-1, keepdim=True) + h.amax(-1, keepdim=True) * (g * h.amax(-1, keepdim=True)).mean(-1, keepdim=True)) / (var + eps).sqrt()
    size = dy.double().abs() if dy is not None else torch.zeros_like(total)
    if pre != "none":
        size = size + through(y, dn.double() * s * (1 + _abs(v.get("pre_weight"))), pre)
    ref.assert_rounded(got["x"], want["x"], 4 * NORM_SLACK * rs * size if a else 4 * NORM_SLACK * size, f"dx {case}")
    if a:
        g = size * (ref.over_rows(v["gate"]).abs() if "gate" in v else 1.0) * (1 + _abs(v.get("post_weight")))
        ref.assert_rounded(got["a"], want["a"], 4 * NORM_SLACK * (through(t["a"], g, post) if post != "none" else g), f"da {case}")
    # Column sums: at most 2 N / 148 sequential additions in a group and the groups after them (fewer than 200 in a row here),
    # each off by 2^-24 of the sum of absolute values, and the terms by the slack above.
    h_pre = ref.normed(y.double(), pre, eps).abs() if pre != "none" else None
    h_post = (ref.normed(t["a"].double(), post, eps).abs() if post != "none" else t["a"].double().abs()) if a else None
    for name in want:
        if name in ("x", "a"):
            continue
        w = got[name]
        assert w.dtype == torch.float32 and w.shape == want[name].shape == vec[name].shape
        if name in ("scale", "shift", "pre_weight", "pre_bias"):
            terms = dn.double().abs() * s * (1 + (h_pre + h_pre.amax(-1, keepdim=True)) * (1 + _abs(v.get("pre_weight"))) + _abs(v.get("pre_bias")))
        else:
            terms = (size + total.abs()) * (1 + (h_post + h_post.amax(-1, keepdim=True)) * (1 + _abs(v.get("post_weight"))) + _abs(v.get("post_bias")))
        bound = (200 * 2.0 ** -24 + 4 * NORM_SLACK) * (terms.sum(1) if w.dim() == 2 else terms.sum((0, 1)))
        assert ((w.double() - want[name]).abs() <= bound).all(), f"{name} {case}"


def _grads_of(case, dtype, seed=12):
    B, N, C, pre, post, a, *_ = case
    gen = _gen(seed)
    dy = _randn(gen, B, N, C, dtype=DT[dtype]) if a else None
    dn = _randn(gen, B, N, C, dtype=DT[dtype]) if pre != "none" else None
    return dy, dn


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", NORM_CASES, ids=lambda c: "-".join(map(str, c[:5])))
def test_norm_backward_matches_64_bits(case, dtype):
    t, vec = _norm_case(case, DT[dtype])
    op = _norm_op(case, dtype)
    y, _ = op.forward(t["x"], t.get("a"), **vec)
    dy, dn = _grads_of(case, dtype)
    got = op.backward(y if case[3] != "none" else None, t.get("a"), dy=dy, dn=dn, **vec)
    torch.cuda.synchronize()
    _check_norm_backward(case, t, vec, y, dy, dn, got)
    # the same without the vectors' gradients, and in place: the same bits
    less = op.backward(y, t.get("a"), dy=dy, dn=dn, need_vectors=False, **vec)
    assert set(less) == ({"x", "a"} if case[5] else {"x"})
    assert all(torch.equal(less[n], got[n]) for n in less)
    if case[5]:
        dy2, a2 = dy.clone(), t["a"].clone()
        over = op.backward(y, a2, dy=dy2, dn=dn, dx=dy2, da=a2, **vec)
        assert all(torch.equal(over[n], got[n]) for n in got)
        if dn is not None:  # a branch whose stream has no gradient of its own
            alone = op.backward(y, t["a"], dy=None, dn=dn, **vec)
            zero = op.backward(y, t["a"], dy=torch.zeros_like(dy), dn=dn, **vec)
            assert all(torch.equal(alone[n], zero[n]) for n in zero)


def test_norm_rows_with_a_large_mean_and_constant_rows():
    case = (1, 6, 640, "layer", "layer", True, True, "batch", True)
    t, vec = _norm_case(case, torch.float16)
    t["x"] += 1000.0
    t["a"] = t["a"] * 0.01 - 300.0
    t["a"][0, 2] = 5.0                                      # no variance: normed to zero
    op = _norm_op(case, "fp16")
    y, n = op.forward(t["x"], t["a"], **vec)
    # the mean is off by 2^-24 of the row's values a few times over, which the small deviations then carry
    v = _dbl(vec)
    h = (t["a"].double() - t["a"].double().mean(-1, keepdim=True)).abs()
    want = ref.norm_after(t["x"].double(), t["a"].double(), v, "layer", 1e-5, 0.75)
    rstd = 1 / (t["a"].double().var(-1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    slack = NORM_SLACK * (0.75 * 1100 + v["gate"][:, None].abs() * (1 + v["post_weight"].abs()) * (rstd * (300 + h)))
    ref.assert_rounded(y, want, slack, "y")
    assert torch.isfinite(n).all()
    z, _ = op.forward(torch.zeros_like(t["x"]), torch.zeros_like(t["a"]), gate=vec["gate"])
    assert (z == 0).all()


def test_norm_strides_in_place_and_guard_bands():
    B, N, C = 3, 37, 328
    case = (B, N, C, "layer", "rms", True, True, "batch", True)
    t, vec = _norm_case(case, torch.bfloat16)
    op = _norm_op(case, "bf16")
    y0, n0 = op.forward(t["x"], t["a"], **vec)
    big = torch.full((B, N + 4, 3 * C + 16), 9.0, device="cuda", dtype=torch.bfloat16)
    view = lambda i: big[:, 2:N + 2, i * (C + 8):i * (C + 8) + C]  # noqa: E731
    y, n = view(0), torch.full((B + 1, N + 1, C), 9.0, device="cuda", dtype=torch.bfloat16)
    y.copy_(t["x"])
    op.forward(y, t["a"], y=y, n=n[:B, :N], **vec)           # x in place, rows and batches apart
    assert torch.equal(y, y0) and torch.equal(n[:B, :N], n0)
    assert (n[B:] == 9).all() and (n[:, N:] == 9).all()
    assert (big[:, :2] == 9).all() and (big[:, N + 2:] == 9).all() and (big[:, 2:N + 2, C:] == 9).all()
    xt = t["x"].transpose(0, 1).contiguous().transpose(0, 1)  # sequence-first memory
    y1, n1 = op.forward(xt, t["a"], **vec)
    assert torch.equal(y1, y0) and torch.equal(n1, n0)
    with pytest.raises(block.LinFusionError):
        op.forward(t["x"], t["a"], n=t["x"], **vec)
    with pytest.raises(block.LinFusionError):
        op.forward(big[:, 2:N + 2, 4:4 + C], t["a"], **vec)


def test_norm_batch_of_one_and_shared_vectors_agree():
    case = (1, 50, 320, "layer", "rms", True, True, "batch", True)
    t, vec = _norm_case(case, torch.bfloat16)
    op = _norm_op(case, "bf16")
    dy, dn = _grads_of(case, "bf16")
    shared = {n: (v[0] if v.dim() == 2 else v) for n, v in vec.items()}
    y, _ = op.forward(t["x"], t["a"], **vec)
    a, b = op.backward(y, t["a"], dy=dy, dn=dn, **vec), op.backward(y, t["a"], dy=dy, dn=dn, **shared)
    for n in a:
        assert torch.equal(a[n].reshape(b[n].shape), b[n])


@pytest.mark.parametrize("expanded", [("gate",), ("scale",), ("shift",), ("gate", "scale", "shift")])
@pytest.mark.parametrize("case", [(2, 37, 320, "layer", "rms", True, True, "batch", True), (3, 130, 1280, "rms", "layer", True, True, "batch", False)],
                         ids=lambda c: "-".join(map(str, c[:5])))
def test_expanded_vectors_get_a_gradient_for_each_entry(case, expanded):
    # one vector seen by all entries through a batch stride of zero: the same values made dense give the same gradients, and
    # their sum over the entries is what the vector itself gets
    B, N, C, *_ = case
    t, vec = _norm_case(case, torch.bfloat16)
    op = _norm_op(case, "bf16")
    dy, dn = _grads_of(case, "bf16")
    one = {n: vec[n][:1] for n in expanded}
    wide = dict(vec, **{n: v.expand(B, C) for n, v in one.items()})
    dense = dict(vec, **{n: v.repeat(B, 1) for n, v in one.items()})
    y, n0 = op.forward(t["x"], t["a"], **dense)
    y1, n1 = op.forward(t["x"], t["a"], **wide)
    assert torch.equal(y, y1) and torch.equal(n0, n1)
    want = op.backward(y, t["a"], dy=dy, dn=dn, **dense)
    _check_norm_backward(case, t, dense, y, dy, dn, want)
    torch.full((1 << 22,), float("nan"), device="cuda")  # what the next call's outputs may be made of
    got = op.backward(y, t["a"], dy=dy, dn=dn, **wide)
    assert set(got) == set(want) and all(got[n].shape == want[n].shape and torch.equal(got[n], want[n]) for n in want)


def test_norm_refuses_tensors():
    op = block.BlockNorm(64, pre="layer", post="rms")
    x = _randn(_gen(1), 2, 4, 64)
    g = _randn(_gen(2), 2, 64)
    for kw in (dict(a=x.half()), dict(a=x[:1]), dict(a=x, gate=g[:, :32]), dict(a=x, gate=g[:1].float()), dict(a=x, post_weight=g),
               dict(a=x.cpu()), dict(a=x, y=x[:, :3])):
        with pytest.raises(ValueError):
            op.forward(x, **kw)
    for kw in (dict(), dict(a=x, scale=g), dict(a=x, n=x)):
        with pytest.raises(block.LinFusionError):
            op.forward(x, **kw)
    with pytest.raises(ValueError):
        op.backward(x, x)
    with pytest.raises(block.LinFusionError):
        op.backward(x, x, dy=x.clone(), dn=x.clone(), gate=g, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))


def test_streams_graphs_and_same_bits():
    case = (2, 700, 640, "layer", "rms", True, True, "batch", True)
    t, vec = _norm_case(case, torch.bfloat16)
    op = _norm_op(case, "bf16")
    rope = block.AxialRope(64, (16, 16), layout="token_major")
    dy, dn = _grads_of(case, "bf16")
    pos = torch.randint(0, 64, (700, 2), device="cuda").float()

    def all_of_it():
        y, n = op.forward(t["x"], t["a"], **vec)
        q, k = rope.forward(n.view(2, 700, 10, 64), y.view(2, 700, 10, 64), pos)
        return [y, n, q, k] + [g for _, g in sorted(op.backward(y, t["a"], dy=dy, dn=dn, **vec).items())]

    first = all_of_it()
    torch.cuda.synchronize()
    outs = []
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(8):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(all_of_it())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(first, o))
    # two graphs of the same objects, replayed at the same time on their own streams
    graphs = []
    for s in streams[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            held = all_of_it()
        graphs.append((g, held, s))
    for g, held, s in graphs:
        for h in held:
            h.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for g, _, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for _, held, _ in graphs for a, b in zip(first, held))


def test_given_streams_get_their_own_memory():
    """What a call allocates for itself belongs to the stream that it was given: the current stream, which takes and overwrites
    memory all the while, must not be handed the workspace or an output of work that still runs."""
    from paper_2409_02097_b200 import attn
    x, a = (torch.randn(2, 6000, 1280, device="cuda").bfloat16() for _ in range(2))
    gate = torch.randn(2, 1280, device="cuda").bfloat16()
    norm = block.BlockNorm(1280, "layer", "rms")
    op = attn.LinFusionAttention(2, 8, 3000, 64)
    q, k, v, dy = (torch.randn(2, 8, 3000, 64, device="cuda").bfloat16() for _ in range(4))
    rope = block.AxialRope(64, (16, 16))
    pos = torch.rand(3000, 2, device="cuda")
    calls = lambda **kw: [*norm.backward(x, a, gate=gate, dn=a, **kw).values(), *norm.forward(x, a, gate=gate, **kw),  # noqa: E731
                          *op.backward(q, k, v, dy, **kw), *rope.forward(q, k, pos, **kw)]
    want = calls()
    sizes = {norm.workspace_bytes(2, 6000), op.backward_workspace_bytes(), x.numel() * 2, q.numel() * 2, 1280 * 4, 2 * 1280 * 4}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):
        got = calls(stream=side.cuda_stream)
        for n in sizes:
            for _ in range(3):
                torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))
    op.close()


def test_tensors_of_more_than_2_to_the_31_elements():
    # the last rows, whose offsets need more than 32 bits, equal those of a small call on the same rows
    free = torch.cuda.mem_get_info()[0]
    if free < 40 << 30:
        pytest.skip("needs 40 GB")
    N, C = 1_700_001, 1280
    x = torch.empty(1, N, C, device="cuda", dtype=torch.bfloat16).normal_()
    norm = block.BlockNorm(C)
    _, n = norm.forward(x)
    _, few = norm.forward(x[:, -5:])
    assert torch.equal(n[:, -5:], few)
    dx = norm.backward(x, dn=n, dx=torch.empty_like(x), need_vectors=False)["x"]
    assert torch.equal(dx[:, -5:], norm.backward(x[:, -5:], dn=few, need_vectors=False)["x"])
    del n, dx
    q = x.view(1, N, 20, 64)
    rope = block.AxialRope(64, (16, 16), layout="token_major")
    pos = torch.rand(N, 2, device="cuda") * 100
    out, _ = rope.forward(q, None, pos)
    assert torch.equal(out[:, -5:], rope.forward(q[:, -5:], None, pos[-5:].contiguous())[0])


def test_configurations_are_fixed():
    for op in (block.AxialRope(64, (16, 16)), block.BlockNorm(64)):
        with pytest.raises(AttributeError):
            op.dtype = "fp16"


def test_the_default_stream_can_be_named():
    from paper_2409_02097_b200 import attn
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with attn.allocating_on(0, side.device.index):
            assert torch.cuda.current_stream().cuda_stream == 0
        with attn.allocating_on(None, side.device.index):
            assert torch.cuda.current_stream() == side
        with attn.allocating_on(torch.cuda.Stream().cuda_stream, side.device.index):
            assert torch.cuda.current_stream().cuda_stream not in (0, side.cuda_stream)


def test_strides_of_axes_of_one_do_not_matter():
    x = torch.randn(1, 33, 64, device="cuda").bfloat16()
    odd = x.as_strided((1, 33, 64), (3, 64, 1))
    norm = block.BlockNorm(64)
    assert torch.equal(norm.forward(odd)[1], norm.forward(x)[1])
    assert torch.equal(norm.backward(odd, dn=odd)["x"], norm.backward(x, dn=x)["x"])
    rope = block.AxialRope(64, (32,), layout="token_major")
    pos = torch.arange(33, device="cuda").float().unsqueeze(1)
    q = x.as_strided((1, 33, 1, 64), (5, 64, 7, 1))
    assert torch.equal(rope.forward(q, None, pos)[0], rope.forward(x.view(1, 33, 1, 64), None, pos)[0])


@pytest.mark.parametrize("interleaved,pairs", [(True, (16, 16)), (False, (16, 16)), (False, (9, 6))])
@pytest.mark.parametrize("theta", [1.0, 0.25, 1e-2, 1e-4, 1e-7])
def test_rope_theta_below_one(theta, interleaved, pairs):
    # angles up to 2^24 radians are good to what ROPE_SLACK counts; beyond, to 2^-46 of the angle, and still rotations
    case = (1, 2, 1, 300, 64, pairs, interleaved, "head_major")
    q, k, _ = _rope_case(case, torch.float16)
    op = block.AxialRope(64, pairs, theta=theta, interleaved=interleaved, dtype="fp16")
    top = max(theta ** (-(n - 1) / n) for n in pairs)  # the largest frequency
    gen = _gen(8)
    for reach in (2.0 ** 24, 2.0 ** 24 * top):          # of the angles: within the bound, and coordinates near 2^24 whatever theta is
        pos = (torch.rand(300, 2, generator=gen, device="cuda") * 2 - 1) * (reach / top)
        qr, kr = op.forward(q, k, pos)
        slack = ROPE_SLACK + 2.0 ** -46 * reach if reach > 2.0 ** 24 else ROPE_SLACK
        if slack < 0.5:
            _check_rope(qr, q, pos, case, False, f"theta {theta} {reach}", theta=theta, slack=slack)
            _check_rope(kr, k, pos, case, False, f"theta {theta} {reach}", theta=theta, slack=slack)
        for got, x in ((qr, q), (kr, k)):
            rel = (got.double().square().sum(-1) / x.double().square().sum(-1) - 1).abs().max().item()
            assert rel <= 3 * 2.0 ** -11, f"not a rotation: {rel:.3e}"


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("N,C", [(9, 72), (9, 320), (7, 1280), (5, 4104)])
def test_a_row_of_nan_or_infinity_stays_one_row(N, C, kind, value):
    case = (2, N, C, kind, kind, True, True, "batch", True)
    t, vec = _norm_case(case, torch.bfloat16)
    op = _norm_op(case, "bf16")
    y0, n0 = op.forward(t["x"], t["a"], **vec)
    dy, dn = _grads_of(case, "bf16")
    clean = op.backward(y0, t["a"], dy=dy, dn=dn, **vec)
    row, other = (1, N // 2), torch.ones(2, N, dtype=torch.bool, device="cuda")
    other[row] = False
    for which in ("x", "a"):
        bad = dict(t, **{which: t[which].clone()})
        bad[which][row][C - 1] = value
        y, n = op.forward(bad["x"], bad["a"], **vec)
        assert torch.equal(y[other], y0[other]) and torch.equal(n[other], n0[other])
        v = _dbl(vec)
        want_y = ref.norm_after(bad["x"].double(), bad["a"].double(), v, kind, 1e-5, 0.75)
        assert torch.equal(torch.isnan(y), torch.isnan(want_y)) and torch.equal(torch.isinf(y), torch.isinf(want_y))
        assert torch.equal(torch.isnan(n), torch.isnan(ref.norm_before(y.double(), v, kind, 1e-5)))
    for which in ("y", "a", "dy", "dn"):
        bad = dict(y=y0, a=t["a"], dy=dy, dn=dn)
        bad[which] = bad[which].clone()
        bad[which][row][C - 1] = value
        got = op.backward(bad["y"], bad["a"], dy=bad["dy"], dn=bad["dn"], **vec)
        assert torch.equal(got["x"][other], clean["x"][other]) and torch.equal(got["a"][other], clean["a"][other])
        for name in ("gate", "scale", "shift"):  # the other entry's vectors
            assert torch.equal(got[name][0], clean[name][0])
        want, _ = _reference_backward(case, dict(t, a=bad["a"]), vec, bad["y"], bad["dy"], bad["dn"])
        assert not torch.isfinite(got["x"][row]).all() or which == "a"
        for name in ("x", "a"):
            assert torch.equal(torch.isfinite(got[name][row]), torch.isfinite(want[name][row])), f"{which} {name}"
