"""The operators around one attention layer of a trained block, as they are measured.

Four kinds of case, each a forward or a backward pass that a training or sampling program makes:

  rope       rotary positions with several axes on Q and K (``block.AxialRope``), forward and backward
  norm       the norms before and after a block with its gate, residual scale and modulation
             (``block.BlockNorm``), forward and backward
  attention  the backward pass of the normalized linear attention (``LinFusionAttention.backward``)

``run`` computes them in elementary torch operations in 32 bits, or, with ``own`` set, by the calls a user
makes of this package.  ``exact`` computes the same outputs in 64 bits from the definitions.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS_ATTENTION = 1e-6
EPS_NORM = 1e-6
THETA = 10000.0


# -------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one small image (32 x 32 latents) at head width 64, token-major as projections leave it: latency counts
        dict(name="rope_image_32", op="rope", backward=False, dtype="bf16", layout="token_major", B=2, H=10, Hk=10,
             N=1024, d=64, pairs="16,16", interleaved=True, per_batch=False, packed=False),
        # a short video clip of 16 frames of 45 x 80 latents, width 128, three axes
        dict(name="rope_video_16x45x80", op="rope", backward=False, dtype="bf16", layout="token_major", B=1, H=16, Hk=16,
             N=57600, d=128, pairs="16,24,24", interleaved=False, per_batch=False, packed=False),
        # gradients of Q and K of a 128 x 128 level, fp16, head-major
        dict(name="rope_backward_128", op="rope", backward=True, dtype="fp16", layout="head_major", B=2, H=10, Hk=10,
             N=16384, d=64, pairs="16,16", interleaved=True, per_batch=False, packed=False),
        # Q and K as views of one packed projection, odd token count, positions of each batch entry, part of the width rotated
        dict(name="rope_packed_ragged", op="rope", backward=False, dtype="bf16", layout="token_major", B=3, H=8, Hk=8,
             N=2531, d=80, pairs="10,10,10", interleaved=False, per_batch=True, packed=True),
        # the norm before a block at the lowest level of a UNet (8 x 8 tokens, CFG pair): one launch, latency
        dict(name="norm_before_8x8", op="norm", backward=False, dtype="bf16", B=2, N=64, C=1280, pre="layer", post="none",
             a=False, gate=False, mod="batch", affine=False, rs=1.0),
        # after one block and before the next in one pass: gated residual, post-norm, modulated pre-norm, 128 x 128 x 2
        dict(name="norm_both_128", op="norm", backward=False, dtype="bf16", B=2, N=16384, C=1280, pre="layer", post="rms",
             a=True, gate=True, mod="batch", affine=True, rs=1.0),
        # its backward pass, gradients of every vector among the outputs
        dict(name="norm_both_backward_128", op="norm", backward=True, dtype="bf16", B=2, N=16384, C=1280, pre="layer",
             post="rms", a=True, gate=True, mod="batch", affine=True, rs=1.0),
        # odd token count, narrow rows, fp16, gate and modulation shared by the batch, scaled residual
        dict(name="norm_both_backward_ragged", op="norm", backward=True, dtype="fp16", B=3, N=4099, C=320, pre="rms",
             post="layer", a=True, gate=True, mod="shared", affine=True, rs=0.7071067811865476),
        # SD-v1.5's lowest level: 64 tokens, width 160
        dict(name="attention_backward_64x160", op="attention", dtype="bf16", layout="head_major", B=2, H=8, N=64, d=160,
             dk=160, saved=True, normalize=True, mean=0.0),
        # SD-v1.5's first level at 512 x 512, width 40, the state recomputed from K and V
        dict(name="attention_backward_4096x40", op="attention", dtype="bf16", layout="head_major", B=2, H=8, N=4096, d=40,
             dk=40, saved=False, normalize=True, mean=0.0),
        # SD-XL's first level at 1024 x 1024, fp16, token-major, values with a mean
        dict(name="attention_backward_4096x64", op="attention", dtype="fp16", layout="token_major", B=2, H=10, N=4096, d=64,
             dk=64, saved=True, normalize=True, mean=1.0),
        # SD-XL's second level at 16384 x 8192
        dict(name="attention_backward_131072x64", op="attention", dtype="bf16", layout="head_major", B=2, H=20, N=131072,
             d=64, dk=64, saved=True, normalize=True, mean=0.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "norm", "attention"])
    dtype = rng.choice(["bf16", "fp16"])
    if op == "rope":
        d = rng.choice([32, 40, 64, 80, 128, 160])
        axes = rng.randint(1, 4)
        rotated = d // 2 if rng.random() < 0.5 else rng.randint(axes, d // 2)
        cuts = sorted(rng.sample(range(1, rotated), axes - 1))
        pairs = [b - a for a, b in zip([0] + cuts, cuts + [rotated])]
        B, H = rng.randint(1, 4), rng.randint(1, 24)
        packed = rng.random() < 0.3
        Hk = H if packed else rng.choice([H, max(1, H // 2), 1])
        N = _log(rng, 1, max(1, min(60000, 117_000_000 // (B * H * d))))
        return dict(op=op, backward=rng.random() < 0.5, dtype=dtype, layout=rng.choice(["head_major", "token_major"]), B=B,
                    H=H, Hk=Hk, N=N, d=d, pairs=",".join(map(str, pairs)), interleaved=rng.random() < 0.5,
                    per_batch=rng.random() < 0.4, packed=packed)
    if op == "norm":
        C = 8 * _log(rng, 4, 640)
        B = rng.randint(1, 5)
        N = _log(rng, 1, max(1, min(40000, 41_000_000 // (B * C))))
        a = rng.random() < 0.75
        post = rng.choice(["none", "layer", "rms"]) if a else "none"
        pre = rng.choice(["none", "layer", "rms"]) if a else rng.choice(["layer", "rms"])
        return dict(op=op, backward=rng.random() < 0.6, dtype=dtype, B=B, N=N, C=C, pre=pre, post=post, a=a,
                    gate=a and rng.random() < 0.8, mod=rng.choice(["none", "batch", "shared"]), affine=rng.random() < 0.5,
                    rs=rng.choice([1.0, 0.5, 1.25]))
    d = rng.choice([32, 40, 64, 64, 80, 128, 160])
    dk = {64: rng.choice([64, 64, 128, 32]), 40: rng.choice([40, 80])}.get(d, d)
    B, H = rng.randint(1, 3), rng.randint(1, 20)
    # from two tokens on: with one, Y is V whatever Q and K are, and their gradients are zero but for eps
    N = _log(rng, 2, max(2, min(131072, 167_000_000 // (B * H * max(d, dk)))))
    return dict(op=op, dtype=dtype, layout=rng.choice(["head_major", "token_major"]), B=B, H=H, N=N, d=d, dk=dk,
                saved=rng.random() < 0.5, normalize=dtype == "fp16" or rng.random() < 0.8, mean=rng.choice([0.0, 0.0, 1.0]))


# -------------------------------------------------------------------------------------- inputs
def _pairs(case):
    return [int(p) for p in case["pairs"].split(",")]


def _qk_shape(case, heads):
    B, N, d = case["B"], case["N"], case["d"]
    return (B, heads, N, d) if case["layout"] == "head_major" else (B, N, heads, d)


def _prepare_rope(case, gen, dtype):
    s = {}
    H, Hk, B, N = case["H"], case["Hk"], case["B"], case["N"]
    randn = lambda shape: torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)  # noqa: E731
    if case["packed"]:  # one projection's output holds Q, K and V side by side
        if case["layout"] == "token_major":
            qkv = randn((B, N, 3, H, case["d"]))
            s["q"], s["k"] = qkv[:, :, 0], qkv[:, :, 1]
        else:
            qkv = randn((B, 3, H, N, case["d"]))
            s["q"], s["k"] = qkv[:, 0], qkv[:, 1]
    else:
        s["q"], s["k"] = randn(_qk_shape(case, H)), randn(_qk_shape(case, Hk))
    axes = len(_pairs(case))
    # tokens of a (time, height, width) grid in reading order; with per_batch each entry's grid starts elsewhere
    side = max(1, round(N ** (1.0 / axes)))
    n = torch.arange(N, device="cuda")
    ax = [(n // side ** (axes - 1 - i)) % (side if i else N + 1) for i in range(axes)]
    pos = torch.stack(ax, dim=-1).float()
    if case["per_batch"]:
        pos = pos + torch.randint(0, 500, (B, 1, axes), generator=gen, device="cuda").float()
    s["pos"] = pos.contiguous()
    return s


def _norm(x, kind):
    if kind == "layer":
        x = x - x.mean(dim=-1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS_NORM)


def _prepare_norm(case, gen, dtype):
    B, N, C = case["B"], case["N"], case["C"]
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)  # noqa: E731
    s = dict(x=(randn(B, N, C) + 0.3).to(dtype))
    if case["a"]:
        s["a"] = (0.5 * randn(B, N, C) - 0.1).to(dtype)
    if case["mod"] != "none" or case["gate"]:
        # scale, shift and gate are thirds of one projection of the conditioning vector
        rows = (1 if case["mod"] == "shared" else B, 3 * C)
        mod = (0.3 * randn(*rows)).to(dtype)
        mod = mod[0] if case["mod"] == "shared" else mod
        if case["mod"] != "none" and case["pre"] != "none":
            s["scale"], s["shift"] = mod[..., :C], mod[..., C:2 * C]
        if case["gate"]:
            s["gate"] = mod[..., 2 * C:]
    if case["affine"]:
        for side in ("pre", "post"):
            if case[side] != "none":
                s[side + "_weight"] = (1 + 0.2 * randn(C)).to(dtype)
                if case[side] == "layer":
                    s[side + "_bias"] = (0.2 * randn(C)).to(dtype)
    if case["backward"]:
        if case["a"]:  # the stream after the block, as the forward pass left it
            p = _norm(s["a"].float(), case["post"]) if case["post"] != "none" else s["a"].float()
            if case["gate"]:
                p = p * _vector(s, "gate", p)
            s["y"] = (case["rs"] * s.pop("x").float() + p).to(dtype)
            s["dy"] = randn(B, N, C).to(dtype)
        else:
            s["y"] = s.pop("x")
        if case["pre"] != "none":
            s["dn"] = randn(B, N, C).to(dtype)
    return s


def _phi(x):
    return torch.where(x > 0, x + 1, torch.exp(torch.clamp(x, max=0)))


def _prepare_attention(case, gen, dtype):
    B, H, N, d, dk = (case[n] for n in ("B", "H", "N", "d", "dk"))
    shape = (lambda w: (B, H, N, w)) if case["layout"] == "head_major" else (lambda w: (B, N, H, w))
    randn = lambda w: torch.randn(shape(w), generator=gen, device="cuda", dtype=torch.float32)  # noqa: E731
    s = dict(q=randn(dk).to(dtype), k=randn(dk).to(dtype), v=(randn(d) + case["mean"]).to(dtype),
             # fp16 gradients come loss-scaled
             dy=(randn(d) * (64.0 if dtype == torch.float16 else 1.0)).to(dtype))
    if case["saved"]:  # S | z as the forward pass computes it, kept for the backward pass
        k, v = _heads_first(case, s["k"]).float(), _heads_first(case, s["v"]).float()
        f = _phi(k)
        S, z = f.transpose(-1, -2) @ v, f.sum(dim=-2)
        s["state"] = torch.cat([S.reshape(B * H, dk * d), z.reshape(B * H, dk)], dim=-1).contiguous()
    return s


def _heads_first(case, t):
    return t if case["layout"] == "head_major" else t.transpose(1, 2)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]
    s = {"rope": _prepare_rope, "norm": _prepare_norm, "attention": _prepare_attention}[case["op"]](case, gen, dtype)
    s["case"] = case
    if own:  # the plan or handle that a program makes once per layer shape
        if case["op"] == "attention":
            from paper_2409_02097_b200 import attn
            s["plan"] = attn.LinFusionAttention(case["B"], case["H"], case["N"], case["d"], eps=EPS_ATTENTION, variant="split",
                                                layout=case["layout"], normalize=case["normalize"], dtype=case["dtype"],
                                                d_qk=case["dk"] if case["dk"] != case["d"] else 0)
        else:
            from paper_2409_02097_b200 import block
            if case["op"] == "rope":
                s["plan"] = block.AxialRope(case["d"], _pairs(case), theta=THETA, interleaved=case["interleaved"],
                                            layout=case["layout"], dtype=case["dtype"])
            else:
                s["plan"] = block.BlockNorm(case["C"], pre=case["pre"], post=case["post"], eps=EPS_NORM,
                                            residual_scale=case["rs"], dtype=case["dtype"])
    return s


# -------------------------------------------------------------------------------------- plain forms
def _rotate(x, cos, sin, rotated, interleaved):
    """Pairs of channels (2p, 2p + 1), or (p, p + rotated / 2), turned by their angles; the other channels pass."""
    turned = x[..., :rotated]
    if interleaved:
        u, w = turned[..., 0::2], turned[..., 1::2]
        out = torch.stack([u * cos - w * sin, u * sin + w * cos], dim=-1).flatten(-2)
    else:
        u, w = turned[..., :rotated // 2], turned[..., rotated // 2:]
        out = torch.cat([u * cos - w * sin, u * sin + w * cos], dim=-1)
    return torch.cat([out, x[..., rotated:]], dim=-1)


def _run_rope(case, s):
    pairs = _pairs(case)
    inside = torch.cat([torch.arange(p, device="cuda", dtype=torch.float64) / p for p in pairs])
    axis = torch.repeat_interleave(torch.arange(len(pairs), device="cuda"), torch.tensor(pairs, device="cuda"))
    angle = s["pos"].double()[..., axis] * THETA ** -inside  # far positions: the angle in 64 bits
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if case["backward"]:
        sin = -sin
    heads_at = -3 if case["layout"] == "head_major" else -2
    cos, sin = cos.unsqueeze(heads_at), sin.unsqueeze(heads_at)
    return {n: _rotate(s[n].float(), cos, sin, 2 * sum(pairs), case["interleaved"]).to(s[n].dtype) for n in ("q", "k")}


def _vector(s, name, like):
    """A per-channel vector of the batch entry ([B, C]) or of all of them ([C]) in 32 bits, over the rows of `like`."""
    v = s[name].float()
    return v.unsqueeze(-2) if v.dim() == 2 else v.expand(like.shape[0], 1, -1)


def _sum_rows(t, vector):
    return t.sum(dim=1) if vector.dim() == 2 else t.sum(dim=(0, 1))


def _norm_backward(x, g, kind):
    """Gradient through x -> norm(x) for the gradient g of its result."""
    if kind == "layer":
        x = x - x.mean(dim=-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS_NORM)
    h = x * r
    dx = g - h * (g * h).mean(dim=-1, keepdim=True)
    if kind == "layer":
        dx = dx - g.mean(dim=-1, keepdim=True)
    return dx * r


def _run_norm(case, s):
    dtype, out = DTYPES[case["dtype"]], {}
    if not case["backward"]:
        y = s["x"].float()
        if case["a"]:
            p = s["a"].float()
            if case["post"] != "none":
                p = _norm(p, case["post"])
                if "post_weight" in s:
                    p = p * s["post_weight"].float()
                if "post_bias" in s:
                    p = p + s["post_bias"].float()
            if case["gate"]:
                p = p * _vector(s, "gate", p)
            out["y"] = (case["rs"] * y + p).to(dtype)
            y = out["y"].float()
        if case["pre"] != "none":
            n = _norm(y, case["pre"])
            if "pre_weight" in s:
                n = n * s["pre_weight"].float()
            if "pre_bias" in s:
                n = n + s["pre_bias"].float()
            if "scale" in s:
                n = n * (1 + _vector(s, "scale", n)) + _vector(s, "shift", n)
            out["n"] = n.to(dtype)
        return out
    y = s["y"].float()
    total = s["dy"].float() if "dy" in s else torch.zeros_like(y)
    if case["pre"] != "none":
        g, h = s["dn"].float(), _norm(y, case["pre"])
        if "scale" in s:
            w = h * s["pre_weight"].float() if "pre_weight" in s else h
            w = w + s["pre_bias"].float() if "pre_bias" in s else w
            out["scale"], out["shift"] = _sum_rows(g * w, s["scale"]), _sum_rows(g, s["shift"])
            g = g * (1 + _vector(s, "scale", g))
        if "pre_bias" in s:
            out["pre_bias"] = g.sum(dim=(0, 1))
        if "pre_weight" in s:
            out["pre_weight"] = (g * h).sum(dim=(0, 1))
            g = g * s["pre_weight"].float()
        total = total + _norm_backward(y, g, case["pre"])
    if not case["a"]:
        out["x"] = total.to(dtype)
        return out
    out["x"] = (case["rs"] * total).to(dtype)
    a, g = s["a"].float(), total
    h = _norm(a, case["post"]) if case["post"] != "none" else a
    if case["gate"]:
        p = h * s["post_weight"].float() if "post_weight" in s else h
        p = p + s["post_bias"].float() if "post_bias" in s else p
        out["gate"] = _sum_rows(g * p, s["gate"])
        g = g * _vector(s, "gate", g)
    if "post_bias" in s:
        out["post_bias"] = g.sum(dim=(0, 1))
    if "post_weight" in s:
        out["post_weight"] = (g * h).sum(dim=(0, 1))
        g = g * s["post_weight"].float()
    out["a"] = (_norm_backward(a, g, case["post"]) if case["post"] != "none" else g).to(dtype)
    return out


def _run_attention(case, s):
    B, H, d, dk = case["B"], case["H"], case["d"], case["dk"]
    q, k, v, g = (_heads_first(case, s[n]).float() for n in ("q", "k", "v", "dy"))
    fq, fk = _phi(q), _phi(k)
    if case["saved"]:
        S, z = s["state"][:, :dk * d].view(B, H, dk, d), s["state"][:, dk * d:].view(B, H, dk)
    else:
        S, z = fk.transpose(-1, -2) @ v, fk.sum(dim=-2)
    t = g @ S.transpose(-1, -2)
    if case["normalize"]:
        w = 1 / (fq @ z.unsqueeze(-1) + EPS_ATTENTION)
        c = (fq * t).sum(dim=-1, keepdim=True) * w
        t = w * (t - c * z.unsqueeze(-2))
        fw = fq * w
        dz = -(fw * c).sum(dim=-2, keepdim=True)
    else:
        fw, dz = fq, 0.0
    dS = fw.transpose(-1, -2) @ g
    slope = lambda x: torch.exp(torch.clamp(x, max=0))  # noqa: E731  the slope of phi: 1 above zero, exp(x) below
    grads = dict(q=t * slope(q), k=(v @ dS.transpose(-1, -2) + dz) * slope(k), v=fk @ dS)
    return {n: _heads_first(case, x).contiguous().to(s[n].dtype) for n, x in grads.items()}


# -------------------------------------------------------------------------------------- one pass
def _run_own(case, s):
    if case["op"] == "rope":
        call = s["plan"].backward if case["backward"] else s["plan"].forward
        q, k = call(s["q"], s["k"], s["pos"])
        return {"q": q, "k": k}
    if case["op"] == "norm":
        given = {n: s[n] for n in ("a", "gate", "scale", "shift", "pre_weight", "pre_bias", "post_weight", "post_bias") if n in s}
        if case["backward"]:
            return s["plan"].backward(s["y"], dy=s.get("dy"), dn=s.get("dn"), **given)
        y, n = s["plan"].forward(s["x"], **given)
        return {name: t for name, t in (("y", y), ("n", n)) if t is not None and not (name == "y" and not case["a"])}
    dq, dk, dv = s["plan"].backward(s["q"], s["k"], s["v"], s["dy"], state=s.get("state"))
    return {"q": dq, "k": dk, "v": dv}


def run(s):
    case = s["case"]
    if own:
        return _run_own(case, s)
    return {"rope": _run_rope, "norm": _run_norm, "attention": _run_attention}[case["op"]](case, s)


# -------------------------------------------------------------------------------------- work
def work(case):
    B, N = case["B"], case["N"]
    if case["op"] == "rope":
        values = B * N * (case["H"] + case["Hk"]) * case["d"]
        pairs = sum(_pairs(case))
        pos = (B if case["per_batch"] else 1) * N * len(_pairs(case)) * 4
        return {"bytes": 4 * values + pos, "flops": 6 * B * N * (case["H"] + case["Hk"]) * pairs}
    if case["op"] == "norm":
        C, rows = case["C"], B * N
        pre = case["pre"] != "none"
        if case["backward"]:  # reads dy and a (with a branch), y and dn (with a norm before); writes dx (and da)
            tensors = (4 + 2 * pre) if case["a"] else 3
        else:                 # reads x (and a); writes y (with a branch) and n
            tensors = 1 + pre + (2 if case["a"] else 0)
        return {"bytes": 2 * tensors * rows * C, "flops": (30 if case["backward"] else 15) * rows * C}
    d, dk, H = case["d"], case["dk"], case["H"]
    # reads Q, K, V, dY, writes dQ, dK, dV; four products of dk x d a token (five where S is recomputed)
    return {"bytes": 2 * B * H * N * (4 * dk + 3 * d) + (4 * B * H * dk * (d + 1) if case["saved"] else 0),
            "flops": 2 * B * H * N * dk * d * (4 if case["saved"] else 5)}


# -------------------------------------------------------------------------------------- 64 bits
def _exact_rope(case, s):
    pairs = _pairs(case)
    turn = []
    for i, p in enumerate(pairs):  # one complex factor for each token and pair
        freq = torch.tensor([THETA ** (-j / p) for j in range(p)], dtype=torch.float64, device="cuda")
        turn.append(torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"][..., i:i + 1].double() * freq))
    turn = torch.cat(turn, dim=-1)
    turn = (turn.conj() if case["backward"] else turn).resolve_conj()
    turn = turn.unsqueeze(-3) if case["layout"] == "head_major" else turn.unsqueeze(-2)
    P, out = sum(pairs), {}
    for n in ("q", "k"):
        x = s[n].double()
        first, second = (x[..., 0:2 * P:2], x[..., 1:2 * P:2]) if case["interleaved"] else (x[..., :P], x[..., P:2 * P])
        z = torch.complex(first.contiguous(), second.contiguous()) * turn
        r = x.clone()
        if case["interleaved"]:
            r[..., 0:2 * P:2], r[..., 1:2 * P:2] = z.real, z.imag
        else:
            r[..., :P], r[..., P:2 * P] = z.real, z.imag
        out[n] = r
    return out


def _exact_normed(x, kind):
    if kind == "layer":
        return (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + EPS_NORM)
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS_NORM)


def _exact_after(case, x, a, t):
    p = a if case["post"] == "none" else _exact_normed(a, case["post"])
    p = p * t.get("post_weight", 1.0) + t.get("post_bias", 0.0)
    if "gate" in t:
        p = p * (t["gate"][:, None] if t["gate"].dim() == 2 else t["gate"])
    return case["rs"] * x + p


def _exact_before(case, y, t):
    n = _exact_normed(y, case["pre"]) * t.get("pre_weight", 1.0) + t.get("pre_bias", 0.0)
    if "scale" in t:
        over = lambda v: v[:, None] if v.dim() == 2 else v  # noqa: E731
        n = n * (1 + over(t["scale"])) + over(t["shift"])
    return n


def _exact_norm(case, s):
    dtype, out = DTYPES[case["dtype"]], {}
    t = {n: x.double() for n, x in s.items() if torch.is_tensor(x)}
    if not case["backward"]:
        y = t["x"]
        if case["a"]:
            out["y"] = _exact_after(case, y, t["a"], t)
            y = out["y"].to(dtype).double()  # the norm is that of the stored stream
        if case["pre"] != "none":
            out["n"] = _exact_before(case, y, t)
        return out
    # the gradients of <dy, y> + <dn, before(y)>, and of the branch behind y, by differentiation of the definition
    vectors = [n for n in ("scale", "shift", "pre_weight", "pre_bias", "gate", "post_weight", "post_bias") if n in t]
    for n in vectors:
        t[n].requires_grad_(True)
    total = t.get("dy", torch.zeros_like(t["y"]))
    if case["pre"] != "none":
        y = t["y"].clone().requires_grad_(True)
        names = [n for n in vectors if n.startswith("pre_") or n in ("scale", "shift")]
        got = torch.autograd.grad((_exact_before(case, y, t) * t["dn"]).sum(), [y] + [t[n] for n in names])
        total = total + got[0]
        out.update(zip(names, got[1:]))
    if not case["a"]:
        out["x"] = total
        return out
    x, a = torch.zeros_like(total).requires_grad_(True), t["a"].clone().requires_grad_(True)
    names = [n for n in vectors if n.startswith("post_") or n == "gate"]
    got = torch.autograd.grad((_exact_after(case, x, a, t) * total).sum(), [x, a] + [t[n] for n in names])
    out.update(zip(["x", "a"] + names, got))
    return out


def _exact_attention(case, s):
    """The gradients of <dY, Y>, Y of the definition, by differentiation, one slab at a time."""
    q, k, v, g = (_heads_first(case, s[n]) for n in ("q", "k", "v", "dy"))
    grads = [torch.empty(x.shape, dtype=torch.float64, device="cuda") for x in (q, k, v)]
    feature = lambda x: torch.nn.functional.elu(x) + 1  # noqa: E731
    for b in range(case["B"]):
        for h in range(case["H"]):
            leaf = [x[b, h].double().requires_grad_(True) for x in (q, k, v)]
            fq, fk = feature(leaf[0]), feature(leaf[1])
            y = fq @ (fk.t() @ leaf[2])
            if case["normalize"]:
                y = y / (fq @ fk.sum(0) + EPS_ATTENTION)[:, None]
            for to, x in zip(grads, torch.autograd.grad((y * g[b, h].double()).sum(), leaf)):
                to[b, h] = x
    return {n: _heads_first(case, x).contiguous() for n, x in zip(("q", "k", "v"), grads)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "norm": _exact_norm, "attention": _exact_attention}[case["op"]](case, s)
