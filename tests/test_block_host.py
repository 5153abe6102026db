"""The operators around the attention and its backward pass, as far as no GPU is needed: formulas against finite
differences, and what the C entry points refuse before they touch CUDA."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import oracle
from paper_2409_02097_b200 import attn, block, build

import _block_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A16 = 1 << 20  # an aligned address that is never read: the calls below are refused, or find no device


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return block.load_library()


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "linfusion_block.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(linfusion_[a-z_]+)\s*\(", text))
    assert set(block.EXPORTED) == names
    for name in names:
        assert hasattr(lib, name)


# ------------------------------------------------------------------ formulas against differences
def _difference(f, x, i, h=1e-5):
    up, down = x.clone(), x.clone()
    up.view(-1)[i] += h
    down.view(-1)[i] -= h
    return (f(up) - f(down)) / (2 * h)


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("kind", [0, 1])
def test_attention_gradient_formula_against_differences_of_the_oracle(kind, normalize):
    g = torch.Generator().manual_seed(5)
    N, dk, dv, eps = 7, 5, 3, 1e-3
    q, k, v, dy = (torch.randn(1, N, w, generator=g, dtype=torch.float64) for w in (dk, dk, dv, dv))
    if kind == 1:
        q, k = q.abs() + 0.1, k.abs() + 0.1

    def loss(q, k, v):
        call = oracle.linear if normalize else oracle.linear_unnormalized
        args = (q.numpy(), k.numpy(), v.numpy()) + ((eps,) if normalize else ())
        return float((call(*args, phi_kind=kind) * dy.numpy()).sum())

    grads, _ = ref.attention_backward(q, k, v, dy, eps, kind, normalize)
    for which, x in enumerate((q, k, v)):
        for i in range(x.numel()):
            args = [q, k, v]
            def f(t, which=which):
                args[which] = t
                return loss(*args)
            d = _difference(f, x, i)
            assert abs(d - grads[which].view(-1)[i].item()) <= 1e-7 * (1 + abs(d))  # differences: h^2 + 1e-16 / h


def test_attention_gradients_sum_over_shards_of_the_tokens():
    g = torch.Generator().manual_seed(6)
    q, k, v, dy = (torch.randn(2, 9, w, generator=g, dtype=torch.float64) for w in (4, 4, 6, 6))
    (dq, dk, dv), _ = ref.attention_backward(q, k, v, dy, 1e-6)
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
    got = torch.autograd.grad((ref.attention(*leaves, 1e-6) * dy).sum(), leaves)
    for a, b in zip((dq, dk, dv), got):
        assert torch.allclose(a, b, rtol=1e-10, atol=1e-12)


@pytest.mark.parametrize("interleaved", [True, False])
def test_rope_backward_is_the_transpose(interleaved):
    g = torch.Generator().manual_seed(7)
    x, y = (torch.randn(1, 2, 5, 16, generator=g, dtype=torch.float64) for _ in range(2))
    pos = torch.randint(0, 900, (5, 2), generator=g).float()
    fwd, _ = ref.rope(x, pos, (3, 4), 1e4, interleaved, True, False)
    bwd, _ = ref.rope(y, pos, (3, 4), 1e4, interleaved, True, True)
    assert abs((fwd * y).sum() - (x * bwd).sum()) < 1e-10


# ------------------------------------------------------------------ refusals
def _refused(rc, codes=(attn.ERR_INVALID_ARG,)):
    assert rc in codes, rc


def _rope_call(lib, q=None, k=None, pos=A16, pos_b=0, **kw):
    d = dict(B=2, N=8, d=64, n_axes=2, pairs=(16, 16), interleaved=1, backward=0, theta=1e4, flags=0)
    d.update(kw)
    desc = block.RopeDesc(d["B"], d["N"], d["d"], d["n_axes"], (ctypes.c_int32 * 4)(*d["pairs"]), d["interleaved"], d["backward"],
                          d["theta"], d["flags"])
    q = q if q is not None else _rope_tensor()
    return lib.linfusion_rope(ctypes.byref(desc), ctypes.byref(q), None if k is None else ctypes.byref(k), pos, pos_b, None)


def _rope_tensor(in_=A16 * 2, out=A16 * 4, heads=4, in_b=2048, in_t=256, in_h=64, out_b=2048, out_t=256, out_h=64):
    return block.RopeTensor(in_, out, heads, in_b, in_t, in_h, out_b, out_t, out_h)


@pytest.mark.parametrize("kw", [dict(B=0), dict(N=0), dict(d=0), dict(d=60), dict(n_axes=0), dict(n_axes=5), dict(pairs=(16, 17)),
                                dict(pairs=(-1, 4)), dict(pairs=(0, 0)), dict(interleaved=2), dict(backward=-1), dict(theta=0.0),
                                dict(theta=float("nan")), dict(pos=0), dict(pos=A16 + 2), dict(pos_b=-1)])
def test_rope_refuses_bad_arguments(lib, kw):
    _refused(_rope_call(lib, **kw))


@pytest.mark.parametrize("kw", [dict(d=264), dict(B=65536), dict(flags=1), dict(flags=0x10)])
def test_rope_refuses_what_it_does_not_serve(lib, kw):
    _refused(_rope_call(lib, **kw), (attn.ERR_UNSUPPORTED,))


@pytest.mark.parametrize("t", [
    dict(in_=0), dict(out=0), dict(in_=A16 + 8), dict(out=A16 * 4 + 4), dict(in_t=260), dict(out_h=4), dict(in_b=-8), dict(heads=-1),
    dict(out_t=0), dict(out_h=0), dict(out_b=0), dict(out_t=128),          # output rows on top of one another
    dict(out=A16 * 2 + 16), dict(out=A16 * 2, out_t=512, out_b=4096),      # over the input, but not in place
])
def test_rope_refuses_bad_tensors(lib, t):
    _refused(_rope_call(lib, q=_rope_tensor(**t)))


def test_rope_refuses_overlapping_q_and_k(lib):
    _refused(_rope_call(lib, q=_rope_tensor(), k=_rope_tensor(in_=A16 * 6)))               # one output
    _refused(_rope_call(lib, q=_rope_tensor(), k=_rope_tensor(in_=A16 * 4, out=A16 * 8)))  # K's input is Q's output
    _refused(_rope_call(lib, q=_rope_tensor(), k=_rope_tensor(in_=A16 * 6, out=A16 * 4 + 64)))
    # interlaced outputs of one packed tensor are no overlap (refused here for want of a device only)
    packed = [_rope_tensor(in_=A16 * 16 + 2 * 256 * i, out=A16 * 4 + 2 * 256 * i, in_b=6144, in_t=768, out_b=6144, out_t=768)
              for i in (0, 1)]
    rc = _rope_call(lib, q=packed[0], k=packed[1])
    assert rc == attn.ERR_CUDA or torch.cuda.is_available()
    head_major = [_rope_tensor(in_=A16 * 16 + 2 * 2048 * i, out=A16 * 4 + 2 * 2048 * i, in_b=6144, in_t=64, in_h=512, out_b=6144,
                               out_t=64, out_h=512) for i in (0, 1)]
    if not torch.cuda.is_available():
        assert _rope_call(lib, q=head_major[0], k=head_major[1]) == attn.ERR_CUDA
    lapped = [packed[0], _rope_tensor(in_=A16 * 16, out=A16 * 4 + 2 * 192, in_b=6144, in_t=768, out_b=6144, out_t=768)]
    _refused(_rope_call(lib, q=lapped[0], k=lapped[1]))
    empty = _rope_tensor(heads=0)
    _refused(_rope_call(lib, q=empty))


def _norm_call(lib, backward=False, bias=0, **kw):
    d = dict(B=2, N=8, C=64, pre=1, post=2, eps=1e-6, rs=1.0, flags=0, x=A16, a=A16 * 2, y=A16 * 3, n=A16 * 4, dy=A16 * 5, dn=A16 * 6,
             dx=A16 * 7, da=A16 * 8, row=64, batch=512, gate=(A16 * 9, 64), scale=(A16 * 10, 64), shift=(A16 * 11, 64), pre_weight=0,
             pre_bias=0, post_weight=0, post_bias=0, grads={}, ws=A16 * 16, ws_bytes=1 << 30, out_row=None)
    d.update(kw)
    desc = block.NormDesc(d["B"], d["N"], d["C"], d["pre"], d["post"], d["eps"], d["rs"], d["flags"])
    vec = block.NormVectors(d["gate"], d["scale"], d["shift"], d["pre_weight"], d["pre_bias"], d["post_weight"], d["post_bias"])
    rows = lambda name: None if not d[name] else ctypes.byref(  # noqa: E731
        block.Rows(d[name], d["batch"], d["out_row"] if d["out_row"] is not None and name in ("y", "n", "dx", "da") else d["row"]))
    if not backward:
        return lib.linfusion_block_norm(ctypes.byref(desc), rows("x"), rows("a"), ctypes.byref(vec), rows("y"), rows("n"), None)
    grads = block.NormGrads(*[d["grads"].get(n) for n in ("gate", "scale", "shift", "pre_weight", "pre_bias", "post_weight", "post_bias")])
    return lib.linfusion_block_norm_backward(ctypes.byref(desc), rows("y"), rows("a"), ctypes.byref(vec), rows("dy"), rows("dn"),
                                             rows("dx"), rows("da"), ctypes.byref(grads), d["ws"], d["ws_bytes"], None)


def _without_device(rc):
    """The arguments are in order: the call got as far as the device."""
    assert rc == attn.ERR_CUDA or torch.cuda.is_available(), rc


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only where no kernel can run")
def test_norm_accepts_good_arguments_up_to_the_device(lib):
    _without_device(_norm_call(lib))
    _without_device(_norm_call(lib, y=A16, gate=(0, 0)))                    # y in place of x
    _without_device(_norm_call(lib, backward=True, grads=dict(gate=A16 * 20)))
    _without_device(_norm_call(lib, backward=True, dx=A16 * 5, da=A16 * 2, ws=0))  # over dy and over a; nothing wanted


@pytest.mark.parametrize("kw", [
    dict(B=0), dict(N=0), dict(C=0), dict(eps=-1.0), dict(eps=float("nan")), dict(rs=float("inf")), dict(x=0), dict(x=A16 + 8),
    dict(y=0), dict(n=0), dict(row=60), dict(batch=-8), dict(row=0), dict(out_row=32), dict(y=A16 + 64), dict(n=A16), dict(n=A16 * 3),
    dict(n=A16 * 10), dict(scale=(0, 0)), dict(gate=(A16 * 9 + 2, 64)), dict(pre_weight=A16 + 2), dict(a=0), dict(a=0, y=0, post=0),
    dict(pre=0), dict(pre=0, n=0), dict(post=0, post_weight=A16 * 12), dict(pre=0, n=0, scale=(0, 0), shift=(0, 0), pre_bias=A16 * 12),
])
def test_norm_refuses_bad_arguments(lib, kw):
    _refused(_norm_call(lib, **kw))


@pytest.mark.parametrize("kw", [dict(C=60), dict(C=8200), dict(flags=2), dict(pre=3), dict(post=-1), dict(B=65536)])
def test_norm_refuses_what_it_does_not_serve(lib, kw):
    _refused(_norm_call(lib, **kw), (attn.ERR_UNSUPPORTED,))


@pytest.mark.parametrize("kw", [
    dict(y=0), dict(dn=0), dict(dx=0), dict(da=0), dict(dx=A16 * 6), dict(dx=A16 * 3), dict(da=A16 * 5), dict(da=A16 * 7), dict(dx=A16 * 9),
    dict(pre=0, scale=(0, 0), shift=(0, 0)), dict(pre=0, scale=(0, 0), shift=(0, 0), dn=0, dy=0), dict(grads=dict(pre_weight=A16 * 20)),
    dict(grads=dict(gate=A16 * 20 + 1)), dict(grads=dict(post_bias=A16 * 20)), dict(out_row=32), dict(da=A16 * 2 + 128),
])
def test_norm_backward_refuses_bad_arguments(lib, kw):
    _refused(_norm_call(lib, backward=True, **kw))


def test_norm_workspace_is_pure_host(lib):
    small = block.BlockNorm(1280).workspace_bytes(2, 64)
    large = block.BlockNorm(1280).workspace_bytes(2, 16384)
    assert 0 < small <= large and large % 256 == 0
    assert block.BlockNorm(1280).workspace_bytes(2, 1 << 20) == large      # bounded by the SMs, not by the rows
    with pytest.raises(attn.LinFusionError):
        block.BlockNorm(1284).workspace_bytes(2, 64)


def test_constructors_refuse():
    with pytest.raises(ValueError):
        block.AxialRope(64, (16, 17))
    with pytest.raises(ValueError):
        block.AxialRope(64, ())
    with pytest.raises(ValueError):
        block.AxialRope(64, (8,), layout="rows")
    with pytest.raises(ValueError):
        block.AxialRope(64, (8,), dtype="fp32")
    with pytest.raises(ValueError):
        block.BlockNorm(64, pre="batch")
    rope = block.AxialRope(64, (16, 16))
    with pytest.raises(ValueError):
        rope.forward(None, None, torch.zeros(4, 2))
    with pytest.raises(ValueError):
        rope.forward(torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16), None, torch.zeros(4, 2))  # not on a GPU
    with pytest.raises(ValueError):
        block.BlockNorm(64).forward(torch.zeros(1, 4, 64, dtype=torch.bfloat16))


def _backward_call(lib, desc=None, ws_bytes=1 << 40, **kw):
    p = dict(q=1, k=2, v=3, dy=4, state=0, dq=5, dk=6, dv=7, ws=8)
    p.update(kw)
    desc = desc if desc is not None else attn.make_desc(1, 2, 16, 64)
    at = lambda n: p[n] * A16  # noqa: E731
    return lib.linfusion_attn_backward(ctypes.byref(desc), *[at(n) for n in ("q", "k", "v", "dy", "state", "dq", "dk", "dv", "ws")],
                                       ws_bytes, None)


def test_attention_backward_refusals(lib):
    for kw in (dict(B=0), dict(N=0), dict(eps=-1.0), dict(device=-1)):
        args = dict(B=1, H=2, N=16, d=64)
        args.update(kw)
        _refused(_backward_call(lib, attn.make_desc(**args)))
    for kw in (dict(d=48), dict(phi=5), dict(variant=9), dict(variant=0x80), dict(H=70000)):
        args = dict(B=1, H=2, N=16, d=64)
        args.update(kw)
        _refused(_backward_call(lib, attn.make_desc(**args)), (attn.ERR_UNSUPPORTED,))
    _refused(_backward_call(lib, ws=0))
    _refused(lib.linfusion_attn_backward(ctypes.byref(attn.make_desc(1, 2, 16, 64)), *[A16] * 8, A16 + 16, 1 << 40, None))
    assert lib.linfusion_attn_backward(None, *[A16] * 9, 1 << 40, None) == attn.ERR_INVALID_ARG
    assert lib.linfusion_attn_save_state(None, A16, None) == attn.ERR_INVALID_ARG


def test_attention_backward_workspace_follows_the_split(lib):
    def ws(*a, sm=148, **kw):
        n = ctypes.c_size_t(0)
        assert lib.linfusion_attn_backward_workspace_bytes(ctypes.byref(attn.make_desc(*a, **kw)), sm, ctypes.byref(n)) == attn.OK
        return n.value
    slab = lambda dk, dv, n: (n * (dk * dv + dk) * 4 + 255) // 256 * 256  # noqa: E731
    # state, its gradient, and at least one partial
    assert ws(2, 8, 64, 160) >= 3 * slab(160, 160, 16)
    assert ws(2, 10, 1 << 19, 64) == ws(2, 10, 1 << 20, 64)  # bounded by the SMs
    assert ws(2, 10, 4096, 64) == ws(2, 10, 4096, 64, variant="stream")  # the forward's variant plays no part
    assert lib.linfusion_attn_backward_workspace_bytes(ctypes.byref(attn.make_desc(1, 1, 1, 64)), 0, None) == attn.ERR_INVALID_ARG


def test_strides_whose_reach_has_no_sense_are_refused(lib):
    # (n - 1) * stride would pass 64 bits: refused, not wrapped
    far = 1 << 55
    for kw in (dict(in_t=far), dict(out_t=far), dict(in_b=far), dict(out_h=far)):
        _refused(_rope_call(lib, N=1 << 20, B=3, q=_rope_tensor(**kw)))
    _refused(_rope_call(lib, pos_b=1 << 60))
    for backward in (False, True):
        _refused(_norm_call(lib, backward=backward, N=1 << 20, row=far))
        _refused(_norm_call(lib, backward=backward, B=1 << 12, batch=far))
        _refused(_norm_call(lib, backward=backward, B=1 << 12, gate=(A16 * 9, far)))
    if not torch.cuda.is_available():  # an axis of one row: its stride is not looked at
        _without_device(_norm_call(lib, B=1, batch=3, gate=(A16 * 9, 3)))
        _without_device(_rope_call(lib, B=1, q=_rope_tensor(in_b=-5, out_b=5)))


def test_gradients_per_entry_are_known_bits(lib):
    text = open(os.path.join(ROOT, "include", "linfusion_block.h")).read()
    for name, bit in block.PER_ENTRY.items():
        assert re.search(rf"#define LINFUSION_PER_ENTRY_{name.upper()} {bit}u", text)

    def call(per_entry):
        desc = block.NormDesc(2, 8, 64, block.NORM_LAYER, block.NORM_RMS, 1e-6, 1.0, 0)
        rows = [ctypes.byref(block.Rows(A16 * i, 512, 64)) for i in range(1, 7)]
        shared = block.NormVectors((A16 * 9, 0), (A16 * 10, 0), (A16 * 11, 0))
        grads = block.NormGrads(gate=A16 * 20, per_entry=per_entry)
        return lib.linfusion_block_norm_backward(ctypes.byref(desc), rows[0], rows[1], ctypes.byref(shared), *rows[2:],
                                                 ctypes.byref(grads), A16 * 16, 1 << 30, None)

    _refused(call(8))
    if not torch.cuda.is_available():
        _without_device(call(7))


def test_rope_refuses_a_theta_whose_frequencies_have_no_fp32(lib):
    for theta, pairs in ((1e-40, (16, 16)), (5e-324, (4, 4)), (1e-300, (2, 0))):
        _refused(_rope_call(lib, theta=theta, pairs=pairs))
    if not torch.cuda.is_available():
        _without_device(_rope_call(lib, theta=1e-300, pairs=(1, 1)))  # one pair an axis: its frequency is 1
        _without_device(_rope_call(lib, theta=1e-4, pairs=(16, 16)))


@pytest.mark.parametrize("name,at", [
    ("ws", A16 * 5), ("ws", A16 * 8), ("ws", A16 * 20), ("ws", A16 * 9), ("ws", A16 * 3), ("ws", A16 * 7 - 4096),  # over dy, da, a gradient, the gate, y, into dx
    ("gate", A16 * 7), ("gate", A16 * 2 + 64), ("gate", A16 * 6 + 2 * 15 * 64 + 124), ("gate", A16 * 10), ("gate", A16 * 16 + 256),  # dx, a, dn's last bytes, the scale, the workspace
    ("scale", A16 * 20 + 508), ("shift", A16 * 20 - 256), ("shift", A16 * 12), ("post_weight", A16 * 20 + 256),      # another gradient, a weight
])
def test_norm_backward_refuses_sums_over_anything_else(lib, name, at):
    # B = 2, N = 8, C = 64: a tensor has 2048 bytes, a gradient of two entries 512, the partials 16 KB
    grads = dict(gate=A16 * 20)
    if name != "ws":
        grads[name] = at
    _refused(_norm_call(lib, backward=True, post_weight=A16 * 12, grads=grads, **({"ws": at} if name == "ws" else {})))


def test_norm_backward_takes_neighbouring_sums(lib):
    if not torch.cuda.is_available():
        near = dict(gate=A16 * 20, scale=A16 * 20 + 512, shift=A16 * 20 + 1024, post_weight=A16 * 20 + 1536)
        _without_device(_norm_call(lib, backward=True, post_weight=A16 * 12, grads=near, ws=A16 * 20 + 2048))
        _without_device(_norm_call(lib, backward=True, post_weight=A16 * 12, grads={}, ws=A16 * 5))  # nothing wanted, nothing used


def test_rope_refuses_heads_that_pass_32_bits_together(lib):
    far = 1 << 40
    many = [_rope_tensor(in_=far * (2 * i + 2), out=far * (2 * i + 3), heads=1 << 30, in_t=0, out_t=8, in_h=8, out_h=8) for i in (0, 1)]
    _refused(_rope_call(lib, q=many[0], k=many[1], B=1, N=1, d=8, pairs=(2, 2)), (attn.ERR_UNSUPPORTED,))
    if not torch.cuda.is_available():
        many[1].heads = (1 << 30) - 1
        _without_device(_rope_call(lib, q=many[0], k=many[1], B=1, N=1, d=8, pairs=(2, 2)))
