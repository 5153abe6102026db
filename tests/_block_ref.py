"""Plain 64-bit implementations of the operators around the attention and of its backward pass, on any device, for
the tests.  Written from the definitions in the headers; nothing of the package is used."""
import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # a rounding is off by at most this, relative
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # ... and below the normal numbers by at most this


def rope(x, pos, pairs, theta, interleaved, head_major, backward):
    """x [B,H,N,d] or [B,N,H,d]; pos [N,A] or [B,N,A] -> (rotated, bound of the sizes that enter each element)."""
    x = x.double()
    B = x.shape[0]
    pos = pos.double()
    if pos.dim() == 2:
        pos = pos[None].expand(B, -1, -1)
    angles = []
    for a, n in enumerate(pairs):
        for i in range(n):
            angles.append(pos[:, :, a] * float(theta) ** (-i / n))
    angle = torch.stack(angles, dim=-1)            # [B, N, P]
    angle = angle[:, None] if head_major else angle[:, :, None]
    if backward:
        angle = -angle
    P = sum(pairs)
    u_at = [2 * p if interleaved else p for p in range(P)]
    w_at = [2 * p + 1 if interleaved else p + P for p in range(P)]
    u, w = x[..., u_at], x[..., w_at]
    out, size = x.clone(), torch.zeros_like(x)
    out[..., u_at] = u * angle.cos() - w * angle.sin()
    out[..., w_at] = u * angle.sin() + w * angle.cos()
    size[..., u_at] = u.abs() + w.abs()
    size[..., w_at] = u.abs() + w.abs()
    return out, size


def normed(x, kind, eps):
    if kind == "layer":
        return (x - x.mean(-1, keepdim=True)) / (x.var(-1, unbiased=False, keepdim=True) + eps).sqrt()
    if kind == "rms":
        return x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    return x


def over_rows(v):
    return v[:, None] if v.dim() == 2 else v


def norm_after(x, a, vec, post, eps, rs):
    h = normed(a, post, eps) * vec.get("post_weight", 1.0) + vec.get("post_bias", 0.0)
    return rs * x + (over_rows(vec["gate"]) if "gate" in vec else 1.0) * h


def norm_before(y, vec, pre, eps):
    h = normed(y, pre, eps) * vec.get("pre_weight", 1.0) + vec.get("pre_bias", 0.0)
    if "scale" in vec:
        h = h * (1 + over_rows(vec["scale"])) + over_rows(vec["shift"])
    return h


def phi(x, kind=0):
    return x if kind == 1 else torch.where(x > 0, x + 1, torch.exp(x.clamp(max=0)))


def phi_slope(x, kind=0):
    return torch.ones_like(x) if kind == 1 else torch.exp(x.clamp(max=0))


def attention(q, k, v, eps, kind=0, normalize=True):
    """[..., N, d] in 64 bits."""
    fq, fk = phi(q, kind), phi(k, kind)
    y = fq @ (fk.transpose(-1, -2) @ v)
    return y / (fq @ fk.sum(-2).unsqueeze(-1) + eps) if normalize else y


def attention_backward(q, k, v, g, eps, kind=0, normalize=True):
    """The formulas of the header in 64 bits; heads first.  Returns (dq, dk, dv) and for each the sizes that enter its
    elements: the same sums with every term's absolute value."""
    q, k, v, g = (t.double() for t in (q, k, v, g))
    fq, fk = phi(q, kind), phi(k, kind)
    S, z = fk.transpose(-1, -2) @ v, fk.sum(-2)
    Sa = fk.abs().transpose(-1, -2) @ v.abs()
    t, ta = g @ S.transpose(-1, -2), g.abs() @ Sa.transpose(-1, -2)
    if normalize:
        w = 1 / (fq @ z.unsqueeze(-1) + eps)
        c, ca = (fq * t).sum(-1, keepdim=True) * w, (fq.abs() * ta).sum(-1, keepdim=True) * w.abs()
        t, ta = w * (t - c * z.unsqueeze(-2)), w.abs() * (ta + ca * z.abs().unsqueeze(-2))
        fw = fq * w
        dz, dza = -(fw * c).sum(-2, keepdim=True), (fw.abs() * ca).sum(-2, keepdim=True)
    else:
        fw, dz, dza = fq, 0.0, 0.0
    dS, dSa = fw.transpose(-1, -2) @ g, fw.abs().transpose(-1, -2) @ g.abs()
    grads = (t * phi_slope(q, kind), (v @ dS.transpose(-1, -2) + dz) * phi_slope(k, kind), fk @ dS)
    sizes = (ta * phi_slope(q, kind), (v.abs() @ dSa.transpose(-1, -2) + dza) * phi_slope(k, kind), fk.abs() @ dSa)
    return grads, sizes


def assert_rounded(got, want, slack, what):
    """`got` (16-bit) is `want` rounded once, up to `slack` of error before the rounding."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    half = HALF_STEP[got.dtype]
    err = (got.double() - want).abs()
    # the value that was rounded is within slack of want: its rounding is off by half a step of it
    most = half * (want.abs() + slack) + slack + SMALLEST[got.dtype]
    worst = (err - most).max().item() if err.numel() else 0.0
    assert torch.isfinite(got.double()).all() and worst <= 0, f"{what}: over by {worst:.3e}, largest error {err.max().item():.3e}"
