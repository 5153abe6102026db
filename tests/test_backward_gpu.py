"""The attention's backward pass against its 64-bit formulas: every pair of widths, both layouts, types, phi, with and
without the normalizer, ragged lengths, a saved and a recomputed state, the halves of token-sharded use, and a block's
operators one after the other, forward and back."""
import math

import pytest
import torch

from paper_2409_02097_b200 import attn, block, sharding

import _block_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6

# Before its rounding an element of a gradient is off by what the operands' tails leave (2^-16 of the terms' sizes) and by
# fp32 sums over tokens: in chunks and tiles, off by about sqrt(terms) 2^-24 of their sizes, far below.  2^-13 leaves room
# for the products' own truncated fp32 accumulation.
SLACK = 2.0 ** -13


def _rms_limit(dtype):
    """A value rounded to nearest is off by an error that is uniform in half a step: half / sqrt 3 of it in the mean square at
    most (where mantissas are near one); and 2^-14 for everything before the rounding."""
    return ref.HALF_STEP[DT[dtype]] / math.sqrt(3) + 2.0 ** -14


def _inputs(B, H, N, dk, dv, dtype, seed=21, mean=0.0, grad_scale=None, kind=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda w: torch.randn((B, H, N, w), generator=g, device="cuda")  # noqa: E731
    q, k, v, dy = r(dk), r(dk), r(dv) + mean, r(dv) * (grad_scale or (64.0 if dtype == "fp16" else 1.0))
    if kind == 1:
        q, k = q.abs(), k.abs()
    return [t.to(DT[dtype]) for t in (q, k, v, dy)]


def _mean_term(dtype, N, mean):
    """What a mean of the values (spread 1) adds to the relative error of dQ in the mean square.  S is carried as head + tail, off
    by at most 2^-17 (bf16) or 2^-23 (fp16: two steps of 11 bits, rounded) of each element, uniformly: 1 / sqrt 3 of it in the mean
    square.  S_a is about z_a mean + sqrt(N E f^2), z_a = N E f with E f = 1.16 and E f^2 = 1.84 for f = elu + 1 of a normal variable:
    t - c z keeps the second part only, so the error counts z mean / sqrt(N E f^2) = 0.85 sqrt N mean times as much:
    0.49 * 2^-17 sqrt N mean.  Twice that."""
    return (2.0 ** -17 if dtype == "bf16" else 2.0 ** -23) * math.sqrt(N) * mean


def _check(got, tensors, dtype, what, eps=EPS, kind=0, normalize=True, slack=SLACK, rms=True, extra=0.0):
    want, sizes = ref.attention_backward(*tensors, eps, kind, normalize)
    for name, x, w, size in zip(("dq", "dk", "dv"), got, want, sizes):
        ref.assert_rounded(x, w, slack * size, f"{what} {name}")
        if rms and dtype == "bf16" or rms and w.abs().mean() > 1e-3:  # (fp16 gradients near the subnormal numbers round more coarsely)
            rel = ((x.double() - w).norm() / w.norm()).item()
            assert rel <= _rms_limit(dtype) + (extra if name == "dq" else 0.0), f"{what} {name}: {rel:.3e}"


def _major(t, layout):
    return t if layout == "head_major" else t.transpose(1, 2).contiguous()


PAIRS = [(32, 32), (40, 40), (64, 64), (80, 80), (128, 128), (160, 160), (128, 64), (80, 40), (32, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("layout", ["head_major", "token_major"])
@pytest.mark.parametrize("dk,dv", PAIRS)
def test_every_pair_of_widths(dk, dv, layout, dtype):
    for (B, H, N) in ((2, 3, 77), (1, 2, 1030)):
        tensors = _inputs(B, H, N, dk, dv, dtype)
        op = attn.LinFusionAttention(B, H, N, dv, eps=EPS, variant="split", layout=layout, dtype=dtype, d_qk=dk if dk != dv else 0)
        got = op.backward(*[_major(t, layout) for t in tensors])
        torch.cuda.synchronize()
        _check([_major(g, layout) for g in got], tensors, dtype, f"{B}x{H}x{N} {dk}x{dv} {layout} {dtype}")
        op.close()


# Sizes that the tcgen05 kernels take: enough tiles (narrow widths) or work (features of 80 and 128), runs of a CTA that end
# inside a slab, slabs of a few tiles only, last tiles with one and with 127 tokens.
TC_CASES = [(2, 4, 4200, 64, 64), (1, 13, 2689, 64, 64), (3, 45, 300, 64, 64), (2, 4, 4353, 40, 40), (1, 9, 4095, 32, 32), (2, 5, 3500, 32, 64),
            (1, 5, 4001, 128, 128), (2, 7, 3199, 80, 80), (1, 5, 8100, 128, 64), (2, 7, 6100, 80, 40), (2, 20, 513, 128, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("layout", ["head_major", "token_major"])
@pytest.mark.parametrize("case", TC_CASES, ids=lambda c: "x".join(map(str, c)))
def test_large_sizes(case, layout, dtype):
    B, H, N, dk, dv = case
    tensors = _inputs(B, H, N, dk, dv, dtype, mean=0.5)
    op = attn.LinFusionAttention(B, H, N, dv, eps=EPS, variant="split", layout=layout, dtype=dtype, d_qk=dk if dk != dv else 0)
    given = [_major(t, layout) for t in tensors]
    ws = torch.empty(op.backward_workspace_bytes(), dtype=torch.uint8, device="cuda")
    got = op.backward(*given, workspace=ws)
    assert op.backward_status(ws) == attn.OK
    _check([_major(g, layout) for g in got], tensors, dtype, f"{case} {layout} {dtype}")
    again = op.backward(*given, state=op.backward_state(*given[1:3]), workspace=ws)
    assert op.backward_status(ws) == attn.OK and all(torch.equal(a, b) for a, b in zip(got, again))
    op.close()


# Sizes at which the tensor cores' kernels take the first stream (the state) too: runs of many tiles of one slab, and of a CTA
# across slabs of 17 tiles each.
LONG_CASES = [(2, 5, 8300, 64, 64), (5, 20, 2100, 64, 64), (1, 3, 70001, 40, 40), (2, 5, 16100, 32, 64), (1, 5, 15500, 128, 64),
              (2, 7, 16300, 80, 40), (1, 5, 30400, 128, 128), (5, 20, 2100, 128, 128), (1, 7, 43400, 80, 80)]


@pytest.mark.parametrize("dtype,layout", [("bf16", "head_major"), ("fp16", "token_major")])
@pytest.mark.parametrize("case", LONG_CASES, ids=lambda c: "x".join(map(str, c)))
def test_long_slabs(case, layout, dtype):
    B, H, N, dk, dv = case
    # gradients of a size that leaves dK and dV, sums of N terms of w dY, among fp16's normal numbers
    tensors = _inputs(B, H, N, dk, dv, dtype, mean=0.5, grad_scale=64.0 if dtype == "fp16" else 1.0)
    op = attn.LinFusionAttention(B, H, N, dv, eps=EPS, variant="split", layout=layout, dtype=dtype, d_qk=dk if dk != dv else 0)
    given = [_major(t, layout) for t in tensors]
    ws = torch.empty(op.backward_workspace_bytes(), dtype=torch.uint8, device="cuda")
    got = op.backward(*given, workspace=ws)
    assert op.backward_status(ws) == attn.OK
    _check([_major(g, layout) for g in got], tensors, dtype, f"{case} {layout} {dtype}", rms=dtype == "bf16",
           extra=_mean_term(dtype, N, 0.5))
    op.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,N", [(64, 640_001), (128, 640_130)])
def test_one_long_slab(d, N, dtype):
    # more than 32 tiles in a run: accumulators change hands inside a slab, and 148 CTAs share it
    tensors = _inputs(1, 1, N, d, d, dtype, mean=1.0, grad_scale=1024.0)
    op = attn.LinFusionAttention(1, 1, N, d, eps=EPS, variant="split", dtype=dtype)
    ws = torch.empty(op.backward_workspace_bytes(), dtype=torch.uint8, device="cuda")
    got = op.backward(*tensors, workspace=ws)
    assert op.backward_status(ws) == attn.OK
    _check(got, tensors, dtype, f"one slab of {N} x {d} {dtype}", rms=dtype == "bf16", extra=_mean_term(dtype, N, 1.0))
    op.close()


@pytest.mark.parametrize("kind,normalize,eps", [(1, True, 0.5), (0, True, 10.0), (0, False, 1e-6), (1, False, 1e-6)])
@pytest.mark.parametrize("case", [(2, 4, 4200, 64, 64), (1, 5, 4001, 128, 128)], ids=lambda c: "x".join(map(str, c)))
def test_large_sizes_phi_eps_and_normalizer(case, kind, normalize, eps):
    B, H, N, dk, dv = case
    tensors = _inputs(B, H, N, dk, dv, "bf16", kind=kind)
    op = attn.LinFusionAttention(B, H, N, dv, phi=kind, eps=eps, normalize=normalize, variant="split")
    _check(op.backward(*tensors), tensors, "bf16", f"{case} phi {kind} eps {eps} normalize {normalize}", eps=eps, kind=kind, normalize=normalize)
    op.close()


@pytest.mark.parametrize("N", [2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 4097])
@pytest.mark.parametrize("d", [40, 64, 160])
def test_ragged_lengths(d, N):
    tensors = _inputs(2, 2, N, d, d, "bf16", seed=N)
    op = attn.LinFusionAttention(2, 2, N, d, eps=EPS)
    _check(op.backward(*tensors), tensors, "bf16", f"N={N} d={d}", rms=N > 8)
    op.close()


@pytest.mark.parametrize("d", [40, 64, 160])
def test_one_token(d):
    # Y is V times den / (den + eps): dQ and dK are differences of equal terms, zero up to fp32 rounding of the terms
    for dtype in ("bf16", "fp16"):
        tensors = _inputs(3, 2, 1, d, d, dtype)
        op = attn.LinFusionAttention(3, 2, 1, d, eps=EPS, dtype=dtype)
        _check(op.backward(*tensors), tensors, dtype, f"one token {d}", rms=False)
        op.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kind,normalize,eps", [(1, True, 1e-6), (1, True, 0.5), (0, True, 0.0), (0, True, 10.0), (0, False, 1e-6), (1, False, 1e-6)])
def test_phi_eps_and_normalizer(kind, normalize, eps, dtype):
    B, H, N, d = 1, 3, 333, 64
    scale = 1.0 if dtype == "bf16" or normalize else 2.0 ** -4
    tensors = _inputs(B, H, N, d, d, dtype, kind=kind, grad_scale=scale)
    op = attn.LinFusionAttention(B, H, N, d, phi=kind, eps=eps, normalize=normalize, dtype=dtype)
    _check(op.backward(*tensors), tensors, dtype, f"phi {kind} eps {eps} normalize {normalize}", eps=eps, kind=kind, normalize=normalize)
    op.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 80])
def test_values_with_a_mean_and_features_of_unequal_size(d, dtype):
    B, H, N = 2, 2, 3000
    q, k, v, dy = _inputs(B, H, N, d, d, dtype, mean=3.0)
    k[..., 0] -= 6.0      # z of very different sizes
    k[..., 1] += 5.0
    q[..., 2] -= 8.0
    tensors = [q, k, v, dy]
    op = attn.LinFusionAttention(B, H, N, d, eps=EPS, dtype=dtype)
    _check(op.backward(*tensors), tensors, dtype, "mean", rms=False)
    op.close()


def test_tiny_and_large_gradients_bf16():
    for scale in (2.0 ** -60, 2.0 ** 60):
        tensors = _inputs(1, 2, 300, 64, 64, "bf16", grad_scale=scale)
        op = attn.LinFusionAttention(1, 2, 300, 64, eps=EPS)
        _check(op.backward(*tensors), tensors, "bf16", f"scale {scale}")
        op.close()


@pytest.mark.parametrize("variant,shape", [("split", (2, 4, 500, 64)), ("stream", (1, 4, 5000, 64)), ("fused", (2, 8, 1024, 80)),
                                           ("cluster", (2, 8, 150, 160)), ("fused", (2, 20, 576, 64)), ("auto", (2, 8, 4096, 40))])
def test_state_saved_by_the_forward_pass(variant, shape):
    B, H, N, d = shape
    tensors = _inputs(B, H, N, d, d, "bf16")
    op = attn.LinFusionAttention(B, H, N, d, eps=EPS, variant=variant)
    op.forward(*tensors[:3])
    state = op.save_state()
    S, z = op.read_state()
    assert torch.equal(state.cpu()[:, :d * d].reshape(B, H, d, d), torch.from_numpy(S))
    assert torch.equal(state.cpu()[:, d * d:].reshape(B, H, d), torch.from_numpy(z))
    want, sizes = ref.attention_backward(*tensors, EPS)
    for name, x, w in zip(("dq", "dk", "dv"), op.backward(*tensors, state=state), want):
        # the forward's state carries phi(K) rounded to 16 bits: half a step on every term of S and z, and for phi itself as much again
        rel = ((x.double() - w).norm() / w.norm()).item()
        assert rel <= 4 * 2.0 ** -8 / math.sqrt(3), f"{variant} {name}: {rel:.3e}"
    # a state of its own, exact to fp32: as good as recomputed, whichever call makes it
    again = op.backward_state(*tensors[1:3])
    _check(op.backward(*tensors, state=again), tensors, "bf16", "state of its own")
    assert all(torch.equal(a, b) for a, b in zip(op.backward(*tensors), op.backward(*tensors, state=again)))
    op.close()


def test_token_shards_give_the_whole():
    B, H, N, d = 1, 4, 1500, 64
    tensors = _inputs(B, H, N, d, d, "bf16")
    cuts = [sharding.token_shard(N, r, 3) for r in range(3)]
    ops = [attn.LinFusionAttention(B, H, e - b, d, eps=EPS, variant="split") for b, e in cuts]
    parts = [[t[:, :, b:e].contiguous() for t in tensors] for b, e in cuts]
    state = sum(op.backward_state(p[1], p[2]) for op, p in zip(ops, parts))
    firsts = [op.backward_q(p[0], p[3], state) for op, p in zip(ops, parts)]
    grad = sum(g for _, g in firsts)
    seconds = [op.backward_kv(p[1], p[2], grad) for op, p in zip(ops, parts)]
    got = [torch.cat(ts, dim=2) for ts in ([f[0] for f in firsts], [s[0] for s in seconds], [s[1] for s in seconds])]
    _check(got, tensors, "bf16", "shards")
    for op in ops:
        op.close()


def test_outputs_stay_inside_their_buffers_and_inputs_are_kept():
    for (B, H, N, d, layout) in ((1, 3, 77, 40, "head_major"), (2, 2, 129, 64, "token_major"), (1, 1, 33, 160, "head_major"),
                                 (2, 9, 2049, 40, "head_major"), (1, 7, 6100, 80, "token_major"), (3, 4, 3500, 64, "token_major")):
        tensors = [_major(t, layout) for t in _inputs(B, H, N, d, d, "bf16")]
        kept = [t.clone() for t in tensors]
        op = attn.LinFusionAttention(B, H, N, d, eps=EPS, variant="split", layout=layout)
        n = tensors[0].numel()
        bands = [torch.full((n + 1024,), 5.0, device="cuda", dtype=torch.bfloat16) for _ in range(3)]
        ws = torch.full((op.backward_workspace_bytes() + 4096,), 77, device="cuda", dtype=torch.uint8)
        outs = [b[512:512 + n].view(tensors[0].shape) for b in bands]
        off = (-ws.data_ptr()) % 256 + 256
        op.backward(*tensors, dq=outs[0], dk=outs[1], dv=outs[2], workspace=ws[off:off + op.backward_workspace_bytes()])
        torch.cuda.synchronize()
        for b in bands:
            assert (b[:512] == 5).all() and (b[512 + n:] == 5).all()
        assert (ws[:off] == 77).all() and (ws[off + op.backward_workspace_bytes():] == 77).all()
        assert all(torch.equal(a, b) for a, b in zip(tensors, kept))
        # without a word in a workspace read before it is written: the same bits from another filling
        again = op.backward(*tensors)
        assert all(torch.equal(a, b) for a, b in zip(outs, again))
        op.close()


def test_refusals_of_tensors():
    op = attn.LinFusionAttention(1, 2, 64, 64)
    q, k, v, dy = _inputs(1, 2, 64, 64, 64, "bf16")
    for bad in (q.half(), q[:, :1], q.cpu(), q.transpose(1, 2)):
        with pytest.raises(ValueError):
            op.backward(bad, k, v, dy)
    with pytest.raises(ValueError):
        op.backward(q, k, v, dy, state=torch.zeros(2, 64 * 64, device="cuda"))
    for kw in (dict(dq=q), dict(dk=v), dict(dv=dy), dict(workspace=torch.empty(1024, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(attn.LinFusionError):
            op.backward(q, k, v, dy, **kw)
    out = torch.empty_like(q)
    with pytest.raises(attn.LinFusionError):
        op.backward(q, k, v, dy, dq=out, dk=out)
    op.close()


def test_streams_graphs_and_same_bits():
    shapes = [(2, 8, 64, 160), (2, 10, 900, 64), (1, 8, 2000, 40), (2, 8, 4096, 64), (1, 5, 4001, 128)]
    cases = []
    for B, H, N, d in shapes:
        op = attn.LinFusionAttention(B, H, N, d, eps=EPS)
        tensors = _inputs(B, H, N, d, d, "bf16")
        cases.append((op, tensors, op.backward(*tensors)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(20):  # the same objects on three streams at once, forwards among them
        for s in streams:
            with torch.cuda.stream(s):
                for op, tensors, first in cases:
                    outs.append((op.backward(*tensors), first))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for got, first in outs for a, b in zip(got, first))
    graphs = []
    for s in streams[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            held = [op.backward(*tensors) for op, tensors, _ in cases]
        graphs.append((g, held, s))
    for _, held, _ in graphs:
        for h in held:
            for x in h:
                x.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for g, _, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for _, held, _ in graphs:
        for h, (_, _, first) in zip(held, cases):
            assert all(torch.equal(a, b) for a, b in zip(h, first))
    for op, _, _ in cases:
        op.close()


def test_a_block_forward_and_back():
    """Norm before, projections, rotary positions, attention, gated residual and the next norm; then the gradients of the
    input and of every vector, against differentiation in 64 bits of the same chain."""
    B, N, H, d = 2, 300, 5, 64
    C = H * d
    g = torch.Generator(device="cuda").manual_seed(31)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, w = r(B, N, C).bfloat16(), [(r(C, C) / math.sqrt(C)).bfloat16() for _ in range(3)]
    mod = (0.3 * r(B, 3 * C)).bfloat16()
    scale, shift, gate = mod[:, :C], mod[:, C:2 * C], mod[:, 2 * C:]
    weight = (1 + 0.1 * r(C)).bfloat16()
    pos = torch.stack([torch.arange(N, device="cuda") // 20, torch.arange(N, device="cuda") % 20], -1).float()
    up_y, up_n = r(B, N, C).bfloat16(), r(B, N, C).bfloat16()

    before = block.BlockNorm(C, pre="layer")
    after = block.BlockNorm(C, pre="layer", post="rms")
    rope = block.AxialRope(d, (16, 16), layout="token_major")
    op = attn.LinFusionAttention(B, H, N, d, eps=EPS, variant="split", layout="token_major")
    heads = lambda t: t.view(B, N, H, d)  # noqa: E731
    _, n = before.forward(x, scale=scale, shift=shift)
    q0, k0, v = (heads(n @ m) for m in w)
    q, k = rope.forward(q0, k0, pos)
    a = op.forward(q, k, v)
    state = op.save_state()
    y, n2 = after.forward(x, a.view(B, N, C), gate=gate, post_weight=weight)
    back = after.backward(y, a.view(B, N, C), gate=gate, post_weight=weight, dy=up_y, dn=up_n)
    dq, dk, dv = op.backward(q, k, v, heads(back["a"]), state=state)
    dq, dk = rope.backward(dq, dk, pos)
    dn = sum(t.view(B, N, C) @ m.t() for t, m in zip((dq, dk, dv), w))
    first = before.backward(x, scale=scale, shift=shift, dy=back["x"], dn=dn)
    torch.cuda.synchronize()
    assert op.status() == attn.OK

    leaf = {n_: t.double().requires_grad_(True) for n_, t in dict(x=x, scale=scale, shift=shift, gate=gate, weight=weight).items()}
    lw = [m.double() for m in w]
    vec = dict(scale=leaf["scale"], shift=leaf["shift"])
    nn = ref.norm_before(leaf["x"], vec, "layer", 1e-6)
    qq, kk, vv = ((nn @ m).view(B, N, H, d) for m in lw)
    turn = lambda t: _rope_differentiable(t, pos)  # noqa: E731
    yy = ref.attention(turn(qq).transpose(1, 2), turn(kk).transpose(1, 2), vv.transpose(1, 2), EPS).transpose(1, 2).reshape(B, N, C)
    stream = ref.norm_after(leaf["x"], yy, dict(gate=leaf["gate"], post_weight=leaf["weight"]), "rms", 1e-6, 1.0)
    out = ref.norm_before(stream, {}, "layer", 1e-6)
    loss = (stream * up_y.double()).sum() + (out * up_n.double()).sum()
    want = torch.autograd.grad(loss, list(leaf.values()))
    got = (first["x"], first["scale"], first["shift"], back["gate"], back["post_weight"])
    for name, a_, b_ in zip(leaf, got, want):
        # about a dozen 16-bit roundings in a row, the phi(K) and S of the forward among them; the RMS norm divides by the small
        # size of the attention's output, whose own relative error it passes on
        rel = ((a_.double() - b_).norm() / b_.norm()).item()
        assert rel <= 12 * 2.0 ** -8, f"{name}: {rel:.3e}"
    ref_y = ((y.double() - stream).norm() / stream.norm()).item()
    assert ref_y <= 12 * 2.0 ** -8 and ((n2.double() - out).norm() / out.norm()).item() <= 12 * 2.0 ** -8
    op.close()


def _rope_differentiable(x, pos):
    freq = torch.tensor([10000.0 ** (-i / 16) for i in range(16)], dtype=torch.float64, device=x.device)
    angle = torch.cat([pos[:, :1].double() * freq, pos[:, 1:].double() * freq], -1)[None, :, None]
    u, w = x[..., 0::2], x[..., 1::2]
    return torch.stack([u * angle.cos() - w * angle.sin(), u * angle.sin() + w * angle.cos()], -1).flatten(-2)


@pytest.mark.parametrize("layout,d", [("head_major", 64), ("token_major", 80)])
def test_tensors_of_more_than_2_to_the_31_elements(layout, d):
    # the last slab, whose offsets need more than 32 bits, against the formulas
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 90 GB")
    H = 2_200_000_000 // (d * 500_009) + 1
    N = 500_009
    shape = (1, H, N, d) if layout == "head_major" else (1, N, H, d)
    g = torch.Generator(device="cuda").manual_seed(5)
    tensors = [torch.empty(shape, device="cuda", dtype=torch.bfloat16).normal_(generator=g) for _ in range(4)]
    op = attn.LinFusionAttention(1, H, N, d, eps=EPS, variant="split", layout=layout)
    ws = torch.empty(op.backward_workspace_bytes(), dtype=torch.uint8, device="cuda")
    got = op.backward(*tensors, workspace=ws)
    assert op.backward_status(ws) == attn.OK
    last = lambda t: (t[:, -1:] if layout == "head_major" else t[:, :, -1:].transpose(1, 2)).contiguous()  # noqa: E731
    _check([last(t) for t in got], [last(t) for t in tensors], "bf16", f"beyond 2^31 {layout} {d}")
    op.close()


@pytest.mark.parametrize("N", [2, 130])
def test_many_slabs(N):
    B, H, d = 4095, 16, 64
    tensors = _inputs(B, H, N, d, d, "bf16")
    op = attn.LinFusionAttention(B, H, N, d, eps=EPS, variant="split")
    got = op.backward(*tensors)
    for part in (slice(0, 2), slice(B - 2, B)):
        _check([g[part] for g in got], [t[part] for t in tensors], "bf16", f"{B * H} slabs of {N}", rms=N > 8)
    op.close()


def test_an_expired_wait_is_reported():
    """A wait that nothing ends gives up after its time, in the workspace's status word and in the device's count, which
    answers for calls whose workspace has gone."""
    op, tensors = attn.LinFusionAttention(1, 2, 64, 64, eps=EPS), _inputs(1, 2, 64, 64, 64, "bf16")
    other = attn.LinFusionAttention(1, 2, 64, 64, eps=EPS)
    op.backward(*tensors)
    assert op.backward_status() == attn.OK
    ws = torch.empty(op.backward_workspace_bytes(), dtype=torch.uint8, device="cuda")
    op.backward(*tensors, workspace=ws)
    assert op.backward_status(ws) == attn.OK
    stream = torch.cuda.current_stream().cuda_stream
    assert op._lib.linfusion_attn_selftest_backward_wait(op.desc, ws.data_ptr(), stream) == attn.OK
    assert op.backward_status(ws) == attn.ERR_TIMEOUT
    assert op.backward_status() == attn.ERR_TIMEOUT and op.backward_status() == attn.OK
    assert other.backward_status() == attn.ERR_TIMEOUT
    assert attn.LinFusionAttention(1, 2, 64, 64).backward_status() == attn.OK  # made after it was read
    again = op.backward(*tensors, workspace=ws)                                # the context goes on
    assert op.backward_status(ws) == attn.OK and op.backward_status() == attn.OK
    _check(again, tensors, "bf16", "after a wait that expired", rms=False)


MASKED = [(1, 2, 300, 64, 64), (2, 4, 4200, 64, 64), (1, 5, 4001, 128, 128), (1, 2, 200, 160, 160), (2, 4, 4353, 40, 40)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", MASKED, ids=lambda c: "x".join(map(str, c)))
def test_masked_keys_and_queries(case, dtype):
    # keys of -inf have phi = 0: they take no part and get no gradient; queries of -inf have no weight on anything
    B, H, N, dk, dv = case
    q, k, v, dy = _inputs(B, H, N, dk, dv, dtype)
    k[:, :, N // 3:N // 2] = -math.inf
    k[:, -1] = -math.inf       # the last head's keys, all of them: its state is zero, den is eps
    q[:, :, 5:40] = -math.inf
    op = attn.LinFusionAttention(B, H, N, dv, eps=EPS, variant="split", dtype=dtype)
    got = op.backward(q, k, v, dy)
    _check(got, (q, k, v, dy), dtype, f"masked {case} {dtype}", rms=False)
    assert (got[1][:, :, N // 3:N // 2] == 0).all() and (got[0][:, :, 5:40] == 0).all()
    assert all((g[:, -1] == 0).all() for g in got)
    op.close()


@pytest.mark.parametrize("case", MASKED, ids=lambda c: "x".join(map(str, c)))
def test_a_query_on_a_feature_of_small_keys_fp16(case):
    # z of one feature 2^-22 of the others', and queries with their weight on it: w f there is some 2^20 times the others'
    B, H, N, dk, dv = case
    tensors = _inputs(B, H, N, dk, dv, "fp16")
    q, k, v, dy = tensors
    k[..., 0] = -15.25
    q[:, :, 1:9] = -20.0
    q[:, :, 1:9, 0] = 3.0
    op = attn.LinFusionAttention(B, H, N, dv, eps=0.0, variant="split", dtype="fp16")
    got = op.backward(*tensors)
    want, sizes = ref.attention_backward(*tensors, 0.0)
    # phi(K) enters as two fp16 numbers of one grid where it is small: off by 2^-25 (half of its smallest number), times |dS|
    fq, z = ref.phi(q.double()), ref.phi(k.double()).sum(-2)
    dS = (fq / (fq @ z.unsqueeze(-1))).transpose(-1, -2) @ dy.double()
    extra = (0.0, 0.0, 2.0 ** -25 * dS.abs().sum(-2, keepdim=True))
    for name, x, w, size, e in zip(("dq", "dk", "dv"), got, want, sizes, extra):
        ref.assert_rounded(x, w, SLACK * size + e, f"{case} {name}")
    op.close()


@pytest.mark.parametrize("N,d", [(200, 64), (4200, 64), (4001, 128), (200, 160)])
def test_keys_of_zero_where_phi_is_the_identity_fp16(N, d):
    # z = 0, den = eps: w f is a million times f, and dV = dS^T 0 is zero all the same
    tensors = _inputs(1, 5, N, d, d, "fp16", kind=1, grad_scale=2.0 ** -10)
    tensors[1][:, -1] = 0
    op = attn.LinFusionAttention(1, 5, N, d, phi=1, eps=EPS, variant="split", dtype="fp16")
    dq, dk, dv = op.backward(*tensors)
    assert (dv[:, -1] == 0).all() and (dq[:, -1] == 0).all() and not torch.isnan(dk).any()
    _check([t[:, :-1] for t in (dq, dk, dv)], [t[:, :-1] for t in tensors], "fp16", f"identity {N} {d}", kind=1, rms=False)
    op.close()


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", [(1, 3, 300, 64, 64), (2, 4, 4200, 64, 64), (1, 5, 4001, 128, 128), (1, 3, 70, 160, 160)], ids=lambda c: "x".join(map(str, c)))
def test_a_nan_goes_where_the_formulas_take_it(case, dtype, normalize):
    # one NaN in Q, K, V or dY of the first head, the state that of clean K and V; the other heads are as without it
    B, H, N, dk, dv = case
    clean = _inputs(B, H, N, dk, dv, dtype, grad_scale=2.0 ** -4)
    op = attn.LinFusionAttention(B, H, N, dv, eps=EPS, variant="split", dtype=dtype, normalize=normalize)
    state = op.backward_state(*clean[1:3])
    before = op.backward(*clean, state=state)
    q, k, v, dy = (t.double() for t in clean)
    fk = ref.phi(k)
    S, z = fk.transpose(-1, -2) @ v, fk.sum(-2)
    for which in range(4):
        bad = [t.clone() for t in clean]
        bad[which][0, 0, N - 2, 5] = math.nan
        got = op.backward(*bad, state=state)
        q, k, v, dy = (t[0, 0].double() for t in bad)
        f, t = ref.phi(q), dy @ S[0, 0].T
        w = 1 / (f @ z[0, 0] + EPS)[:, None] if normalize else torch.ones_like(f[:, :1])
        c = w * (f * t).sum(-1, keepdim=True) if normalize else torch.zeros_like(w)
        dS, dz = (w * f).T @ dy, -(c * w * f).sum(0)
        want = (ref.phi_slope(q) * w * (t - c * z[0, 0]), ref.phi_slope(k) * (v @ dS.T + (dz if normalize else 0.0)), ref.phi(k) @ dS)
        for name, x, x0, y in zip(("dq", "dk", "dv"), got, before, want):
            # where the formulas are clean nothing is NaN, and the other way round (a term of NaN is one whatever it is multiplied by)
            assert torch.equal(torch.isnan(x[0, 0]), torch.isnan(y)), f"{'qkvg'[which]} {name}"
            assert torch.equal(x[:, 1:], x0[:, 1:])
    op.close()


# Means some hundred times the spread over sqrt(N): before its rounding dQ would be off by 2^-18 sqrt(N) mean (bf16), more than
# the rounding, were the mean carried through the products.
MEAN_CASES = [((1, 2, 65600, 64, 64), 8.0), ((2, 20, 9000, 64, 64), 20.0), ((1, 2, 65600, 128, 128), 8.0), ((1, 3, 33000, 80, 80), 8.0),
              ((1, 3, 33000, 128, 64), 8.0), ((2, 7, 16100, 80, 40), 16.0), ((1, 2, 5000, 160, 160), 24.0), ((1, 2, 20000, 32, 32), 12.0),
              ((1, 2, 1000, 40, 40), 60.0)]


@pytest.mark.parametrize("saved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case,mean", MEAN_CASES, ids=lambda c: "x".join(map(str, c)) if isinstance(c, tuple) else f"mean{c:g}")
def test_the_mean_of_the_values_costs_no_bits_of_dq(case, mean, dtype, saved):
    B, H, N, dk, dv = case
    # (spread / mean) of the values as they are stored: a step of bf16 at the mean is some of the spread, the reference reads the same
    tensors = _inputs(B, H, N, dk, dv, dtype, mean=mean, grad_scale=1024.0 if dtype == "fp16" else 1.0)
    op = attn.LinFusionAttention(B, H, N, dv, eps=EPS, variant="split", dtype=dtype, d_qk=dk if dk != dv else 0)
    state = None
    if saved:  # what an exact forward pass would leave
        f, v = ref.phi(tensors[1].double()), tensors[2].double()
        state = torch.cat([(f.transpose(-1, -2) @ v).flatten(-2), f.sum(-2)], -1).float().view(B * H, -1).contiguous()
    dq = op.backward(*tensors, state=state)[0]
    want = ref.attention_backward(*tensors, EPS)[0][0]
    rel = ((dq.double() - want).norm() / want.norm()).item()
    # What S itself is off by, t - c z takes 0.85 sqrt(N) mean times as large.  fp32: 2^-25, uniformly.  A recomputed state is
    # summed by the tensor core, which truncates the running sum after each of n <= 32 * 8 steps of 16 tokens: off by 0 to 2^-23 of it,
    # that is by a common part, a multiple of z, which leaves with the mean, and a part of 2^-23 / sqrt 12 in the mean square;
    # over n steps of a sum that grows evenly, 2^-23 sqrt(n / 36).
    grown = 0.85 * math.sqrt(N) * mean
    extra = grown * (2 * 2.0 ** -25 / math.sqrt(3) + (0.0 if saved else 2.0 ** -23 * math.sqrt(256 / 36)))
    assert rel <= _rms_limit(dtype) + extra, f"{rel:.3e}"
    op.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", [(1, 2, 300, 64, 64), (2, 4, 4200, 64, 64), (1, 5, 4001, 128, 128), (1, 5, 8100, 128, 64), (1, 2, 70, 160, 160)],
                         ids=lambda c: "x".join(map(str, c)))
def test_an_eps_that_counts_and_values_with_a_mean(case, dtype):
    # eps from far below den to far above it, tokens of small den among others: the mean does not cancel there
    B, H, N, dk, dv = case
    tensors = _inputs(B, H, N, dk, dv, dtype, mean=3.0, grad_scale=16.0)
    tensors[0][:, :, ::7] = -12.0
    tensors[0][:, :, 1::7, 3:] = -20.0
    for eps in (1e-3, 1.0, 2e4):
        op = attn.LinFusionAttention(B, H, N, dv, eps=eps, variant="split", dtype=dtype, d_qk=dk if dk != dv else 0)
        _check(op.backward(*tensors), tensors, dtype, f"{case} {dtype} eps {eps}", eps=eps, rms=False)
        whole, grad_state = op.backward_q(tensors[0], tensors[3], op.backward_state(*tensors[1:3]))
        f = ref.phi(tensors[0].double())
        S = ref.phi(tensors[1].double()).transpose(-1, -2) @ tensors[2].double()
        z = ref.phi(tensors[1].double()).sum(-2)
        w = 1 / (f @ z.unsqueeze(-1) + eps)
        t = tensors[3].double() @ S.transpose(-1, -2)
        dz = -(w * f * (w * (f * t).sum(-1, keepdim=True))).sum(-2)
        sizes = (w * f * (w * (f * (tensors[3].double().abs() @ S.abs().transpose(-1, -2))).sum(-1, keepdim=True))).sum(-2)
        err = (grad_state[:, dk * dv:].view(B, H, dk).double() - dz).abs()
        assert (err <= SLACK * sizes).all(), f"dz {case} eps {eps}: {(err / sizes).max().item():.3e}"
        op.close()


def test_state_saved_after_a_forward_on_host_buffers():
    # large enough for two groups of slabs, which one sub-handle works through in turn
    B, H, N, d = 1, 2, 262144, 64
    tensors = _inputs(B, H, N, d, d, "bf16")[:3]
    op = attn.LinFusionAttention(B, H, N, d, eps=EPS)
    op.forward(*tensors)
    want = op.save_state()
    op.forward(tensors[0], torch.zeros_like(tensors[1]), tensors[2])  # another state
    host = [t.cpu().pin_memory() for t in tensors]
    y = torch.empty_like(host[0]).pin_memory()
    op.forward_host(*host, y)
    got = op.save_state()
    torch.cuda.synchronize()
    # the same terms, added in the order of another split of the tokens
    for slab in range(H):
        assert ((got[slab] - want[slab]).norm() / want[slab].norm()).item() <= 1e-5
    S, z = op.read_state()
    assert torch.equal(got.cpu()[:, :d * d].reshape(B, H, d, d), torch.from_numpy(S))
    op.close()


def test_threads_that_share_a_stream():
    """Calls of several threads on one stream, their workspaces and outputs from one pool: what a thread's call holds is not
    handed to another before its kernels are enqueued."""
    import threading
    shapes = [(2, 4, 900, 64), (1, 8, 300, 40), (1, 3, 2000, 128), (2, 2, 64, 160)]
    jobs = []
    for B, H, N, d in shapes:
        op, tensors = attn.LinFusionAttention(B, H, N, d, eps=EPS, variant="split"), _inputs(B, H, N, d, d, "bf16", seed=N)
        jobs.append((op, tensors, op.backward(*tensors)))
    stream, wrong = torch.cuda.Stream(), []
    stream.wait_stream(torch.cuda.current_stream())

    def work(op, tensors, want):
        with torch.cuda.stream(stream):
            for _ in range(50):
                got = op.backward(*tensors)
                state = op.backward_state(*tensors[1:3])
                dq, grad = op.backward_q(tensors[0], tensors[3], state)
                parts = (dq, *op.backward_kv(tensors[1], tensors[2], grad))
                if not all(torch.equal(a, c) and torch.equal(b, c) for a, b, c in zip(got, parts, want)):
                    wrong.append(op.shape)

    threads = [threading.Thread(target=work, args=job) for job in jobs for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong
    for op, _, _ in jobs:
        assert op.backward_status() == attn.OK
        op.close()


@pytest.mark.parametrize("variant,shape", [("split", (2, 4, 500, 64)), ("stream", (1, 4, 5000, 64)), ("fused", (2, 8, 1024, 80)), ("cluster", (2, 8, 150, 160)),
                                           ("fused", (2, 20, 576, 64)), ("split", (1, 4, 4100, 128)), ("auto", (2, 8, 4096, 40))])
def test_state_saved_by_a_forward_pass_in_fp16(variant, shape):
    # S and z of the forward carry phi(K) rounded to 16 bits, the same in both: half a step on every term, and for phi itself as
    # much again; a mean of the values leaves with the multiple of z
    B, H, N, d = shape
    for mean in (0.0, 2.0):
        tensors = _inputs(B, H, N, d, d, "fp16", mean=mean, grad_scale=256.0)
        op = attn.LinFusionAttention(B, H, N, d, eps=EPS, variant=variant, dtype="fp16")
        op.forward(*tensors[:3])
        want, _ = ref.attention_backward(*tensors, EPS)
        for name, x, w in zip(("dq", "dk", "dv"), op.backward(*tensors, state=op.save_state()), want):
            rel = ((x.double() - w).norm() / w.norm()).item()
            assert rel <= 4 * 2.0 ** -11 / math.sqrt(3), f"{variant} mean {mean} {name}: {rel:.3e}"
        op.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", [(2, 8, 16400, 160, 160), (1, 3, 16391, 32, 32)], ids=lambda c: "x".join(map(str, c)))
def test_long_slabs_of_the_widths_that_have_no_tcgen05_kernel(case, dtype):
    B, H, N, dk, dv = case
    tensors = _inputs(B, H, N, dk, dv, dtype, mean=0.5, grad_scale=256.0 if dtype == "fp16" else 1.0)
    op = attn.LinFusionAttention(B, H, N, dv, eps=EPS, variant="split", dtype=dtype)
    _check(op.backward(*tensors), tensors, dtype, f"{case} {dtype}", rms=dtype == "bf16", extra=_mean_term(dtype, N, 0.5))
    op.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", [(1, 3, 300, 64, 64), (2, 4, 4200, 64, 64), (1, 5, 4001, 128, 128), (1, 2, 150, 160, 160)], ids=lambda c: "x".join(map(str, c)))
def test_features_of_both_signs(case, dtype):
    # phi(x) = x with an eps that keeps f . z + eps away from zero: z of either sign, and the eps term counts for every token
    B, H, N, dk, dv = case
    q, k, v, dy = _inputs(B, H, N, dk, dv, dtype, mean=2.0, grad_scale=16.0)
    eps = 60.0 * math.sqrt(N * dk)  # |f . z| is some sqrt(N dk)
    op = attn.LinFusionAttention(B, H, N, dv, phi=1, eps=eps, variant="split", dtype=dtype)
    _check(op.backward(q, k, v, dy), (q, k, v, dy), dtype, f"{case} {dtype}", eps=eps, kind=1, rms=False)
    op.close()
