"""Plain 64-bit implementations of the layers (products with an epilogue, the gated recurrence, the 8-bit format), on any device, for
the tests.  Written from the definitions in the header; nothing of the package is used.  Beside each result the sizes that enter its
elements: the same sums with every term's absolute value, for the bounds of the errors."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # a rounding is off by at most this, relative
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # ... and below the normal numbers by at most this
EXPONENTS = {torch.bfloat16: (-126, 121), torch.float16: (-24, 9)}
EVERY = 64


# ------------------------------------------------------------------ activations
def act(u, kind):
    if kind == "relu":
        return torch.where(u < 0, torch.zeros_like(u), u)
    if kind == "silu":
        return u * torch.sigmoid(u)
    if kind == "gelu":
        return 0.5 * u * (1 + torch.erf(u / math.sqrt(2)))
    if kind == "gelu_tanh":
        return 0.5 * u * (1 + torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3)))
    return u


def act_slope(u, kind):
    if kind == "relu":
        return (u > 0).to(u.dtype)
    if kind == "silu":
        s = torch.sigmoid(u)
        return s * (1 + u * (1 - s))
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(u / math.sqrt(2))) + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (u + 0.044715 * u ** 3))
        return 0.5 * (1 + t) + 0.5 * u * (1 - t * t) * c * (1 + 3 * 0.044715 * u * u)
    return torch.ones_like(u)


# ------------------------------------------------------------------ the 8-bit format
def pack(x, dtype):
    """(codes, scale bytes) one group after the other."""
    x = x.double()
    C = x.shape[-1]
    lo, hi = EXPONENTS[dtype]
    codes, scales = torch.empty(x.shape, dtype=torch.int8, device=x.device), []
    for c in range(0, C, 32):
        g = x[..., c:c + 32]
        fine = torch.isfinite(g)
        most = torch.where(fine, g.abs(), torch.zeros_like(g)).amax(-1)
        e = torch.full(most.shape, lo, dtype=torch.float64, device=x.device)
        for k in range(lo, hi):  # the smallest with most <= 127 * 2^e
            e = torch.where(most > 127 * 2.0 ** k, torch.full_like(e, k + 1), e)
        q = torch.round(torch.where(fine, g, torch.zeros_like(g)) * torch.exp2(-e).unsqueeze(-1)).clamp(-127, 127)
        codes[..., c:c + 32] = torch.where(fine, q, torch.full_like(q, -128)).to(torch.int8)
        scales.append((e + 127).to(torch.uint8))
    return codes, torch.stack(scales, dim=-1)


def unpack(codes, scales):
    step = torch.exp2(scales.double() - 127).repeat_interleave(32, dim=-1)[..., :codes.shape[-1]]
    return torch.where(codes == -128, torch.full_like(step, math.nan), codes.double() * step)


# ------------------------------------------------------------------ the recurrence
def recurrence(x, decay, rate, gate=None, h0=None, reverse=False):
    """h of every token, the last state, the states before every 64th token, all by going through the tokens; and for every channel the
    largest value that enters, and over how many tokens the state remembers (at most N)."""
    x, decay, rate = x.double(), decay.double(), rate.double()
    L = rate * torch.sigmoid(decay)
    e = -torch.expm1(-L)
    v = x if gate is None else x * torch.sigmoid(gate.double())
    v = torch.where(decay == -math.inf, torch.zeros_like(v), v)
    B, N, C = x.shape
    h = torch.zeros(B, C, dtype=torch.float64, device=x.device) if h0 is None else h0.double()
    out, states, before = torch.empty_like(x), [], torch.empty_like(x)
    most = torch.maximum(v.abs().amax(1), h.abs())
    for i in range(N):
        t = N - 1 - i if reverse else i
        if i % EVERY == 0:
            states.append(h)
        before[:, t] = h
        h = h + e[:, t] * (v[:, t] - h)
        out[:, t] = h
    steps = torch.clamp(1 / e.clamp(min=1e-30).amin(1), max=float(N))
    return dict(h=out, last=h, state=torch.stack(states, 1), before=before, e=e, v=v, most=most, steps=steps)


def recurrence_backward(dh, x, decay, rate, gate=None, h0=None, dlast=None, reverse=False, before=None):
    """The formulas of the header; `before`: the state before every token (None: from the forward pass).  (gradients, sizes)"""
    f = recurrence(x, decay, rate, gate, h0, reverse)
    before = f["before"] if before is None else before
    e, v = f["e"], f["v"]
    x, decay, rate, dh = x.double(), decay.double(), rate.double(), dh.double()
    s = torch.sigmoid(decay)
    q = torch.ones_like(x) if gate is None else torch.sigmoid(gate.double())
    B, N, C = x.shape
    zero = torch.zeros(B, C, dtype=torch.float64, device=x.device)
    carry = zero if dlast is None else dlast.double()
    size = carry.abs()
    G, Gs = torch.empty_like(x), torch.empty_like(x)
    for i in range(N - 1, -1, -1):
        t = N - 1 - i if reverse else i
        G[:, t], Gs[:, t] = dh[:, t] + carry, dh[:, t].abs() + size
        carry, size = (1 - e[:, t]) * G[:, t], (1 - e[:, t]) * Gs[:, t]
    counts = decay != -math.inf
    clean = lambda t: torch.where(counts, t, torch.zeros_like(t))  # noqa: E731
    x, q = clean(x), clean(q)
    dL = (1 - e) * G * (v - before)
    dLs = Gs * (v.abs() + f["most"].unsqueeze(1))
    grads = dict(x=q * e * G, decay=rate * s * (1 - s) * dL, rate=(s * dL).sum((0, 1)), h0=carry)
    sizes = dict(x=q * e * Gs, decay=rate.abs() * s * dLs, rate=(s * dLs).sum((0, 1)), h0=size)
    if gate is not None:
        grads["gate"], sizes["gate"] = e * G * x * q * (1 - q), e * Gs * x.abs() * q
    return grads, sizes, f


# ------------------------------------------------------------------ comparisons
def assert_rounded(got, want, slack, what):
    """`got` (16-bit) is `want` rounded once, up to `slack` of error before the rounding."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    half = HALF_STEP[got.dtype]
    err = (got.double() - want).abs()
    most = half * (want.abs() + slack) + slack + SMALLEST[got.dtype]
    worst = (err - most).max().item() if err.numel() else 0.0
    assert torch.isfinite(got.double()).all() and worst <= 0, f"{what}: over by {worst:.3e}, largest error {err.max().item():.3e}"


def assert_near(got, want, slack, what):
    assert got.shape == want.shape, (what, got.shape, want.shape)
    err = (got.double() - want).abs()
    worst = (err - slack).max().item()
    assert torch.isfinite(got.double()).all() and worst <= 0, f"{what}: over by {worst:.3e}, largest error {err.max().item():.3e}"
