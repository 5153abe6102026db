"""The products, the recurrence and the 8-bit checkpoints of a trained block, as they are measured.

Three kinds of case:

  linear      a matrix product with bias, activation and residual in its epilogue (``layers.Linear``): forward (with the
              pre-activation kept, in 8 bits too), backward, and backward from 8-bit checkpoints
  recurrence  a gated linear recurrence over the tokens, each channel for itself (``layers.GatedRecurrence``): forward (from
              one token on), backward, and backward from 8-bit checkpoints
  pack8       a 16-bit tensor into 8 bits and back (``layers.pack8``)

``run`` computes them in elementary torch operations in 32 bits, or, with ``own`` set, by the calls a user makes of this
package.  ``exact`` computes the same outputs in 64 bits from the definitions.

The 8-bit format: 32 consecutive channels share a power of two 2^e, the smallest with max|x| <= 127 * 2^e within the
storage type's range of e; the scale byte holds e + 127, the codes x * 2^-e rounded to whole numbers of -127 .. 127.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EXPONENTS = {torch.bfloat16: (-126, 121), torch.float16: (-24, 9)}
GROUP = 32  # channels that share a scale
EVERY = 64  # a saved state of the recurrence for each so many tokens


# -------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the conditioning vectors of a pair of images through a layer of 1280: latency, the weights are all there is to read
        dict(name="linear_two_rows", op="linear", what="forward", dtype="bf16", M=2, K=1280, N=1280, act="silu", bias=True,
             residual=False, save=False, transposed=True),
        # the projection behind the attention of a pair of 64 x 64 levels, added to the residual stream
        dict(name="linear_out_8192x1280", op="linear", what="forward", dtype="bf16", M=8192, K=1280, N=1280, act="none", bias=True,
             residual=True, save=False, transposed=False),
        # the same layer with odd token count, narrow input, fp16: backward, with the pre-activation at hand
        dict(name="linear_backward_ragged", op="linear", what="backward", dtype="fp16", M=4099, K=320, N=1288, act="silu", bias=True,
             residual=False, save=True, transposed=True),
        # the first layer of a feed-forward at a pair of 128 x 128 levels, its pre-activation kept in 8 bits
        dict(name="linear_forward8_32768x640", op="linear", what="forward8", dtype="bf16", M=32768, K=640, N=2560, act="gelu", bias=True,
             residual=False, save=True, transposed=False),
        # its backward pass, from 8-bit checkpoints of its input and pre-activation
        dict(name="linear_backward8_32768x640", op="linear", what="backward8", dtype="bf16", M=32768, K=640, N=2560, act="gelu",
             bias=True, residual=False, save=True, transposed=False),
        # one token for each of eight sequences, the state carried from call to call: latency
        dict(name="recurrence_one_token", op="recurrence", what="forward", dtype="bf16", B=8, N=1, C=1280, gate=True, h0=True,
             save=False, reverse=False, padded=0, saved=False),
        # a pair of 64 x 64 levels in reading order
        dict(name="recurrence_forward_4096", op="recurrence", what="forward", dtype="bf16", B=2, N=4096, C=1280, gate=True, h0=False,
             save=True, reverse=False, padded=0, saved=False),
        # odd lengths, narrow rows, backwards in the tokens, padding, no saved states: backward
        dict(name="recurrence_backward_ragged", op="recurrence", what="backward", dtype="fp16", B=3, N=2531, C=328, gate=False, h0=True,
             save=False, reverse=True, padded=17, saved=False),
        # a pair of 128 x 128 levels: backward
        dict(name="recurrence_backward_16384", op="recurrence", what="backward", dtype="bf16", B=2, N=16384, C=640, gate=True, h0=False,
             save=False, reverse=False, padded=0, saved=True),
        # one long sequence of 512 x 256 tokens: backward from 8-bit checkpoints
        dict(name="recurrence_backward8_131072", op="recurrence", what="backward8", dtype="bf16", B=1, N=131072, C=640, gate=True,
             h0=False, save=False, reverse=True, padded=0, saved=True),
        # the lowest level of a UNet (8 x 8 tokens, a pair) into 8 bits and back: latency
        dict(name="pack8_8x8", op="pack8", dtype="bf16", M=128, C=1280),
        # odd rows and width, fp16, the largest level
        dict(name="pack8_ragged", op="pack8", dtype="fp16", M=61441, C=648),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "recurrence", "recurrence", "pack8"])
    dtype = rng.choice(["bf16", "fp16"])
    if op == "linear":
        K, N = 8 * _log(rng, 4, 640), 8 * _log(rng, 4, 640)
        M = _log(rng, 1, max(1, min(33000, 53_000_000_000 // (K * N), 84_000_000 // max(K, N))))
        what = rng.choice(["forward", "forward", "forward8", "backward", "backward8"])
        act = rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"])
        return dict(op=op, what=what, dtype=dtype, M=M, K=K, N=N, act=act, bias=rng.random() < 0.7, residual=rng.random() < 0.5,
                    save=act != "none" and (what != "forward" or rng.random() < 0.5), transposed=rng.random() < 0.5)
    if op == "recurrence":
        B, C = rng.randint(1, 6), 8 * _log(rng, 1, 320)
        N = _log(rng, 1, max(1, min(131072, 66_000_000 // (B * C))))
        what = rng.choice(["forward", "backward", "backward8"])
        return dict(op=op, what=what, dtype=dtype, B=B, N=N, C=C, gate=rng.random() < 0.7, h0=rng.random() < 0.5,
                    save=what == "forward" and rng.random() < 0.5, reverse=rng.random() < 0.5,
                    padded=rng.randint(1, N // 2) if N > 8 and rng.random() < 0.3 else 0, saved=what != "forward" and rng.random() < 0.6)
    C = 8 * _log(rng, 1, 640)
    return dict(op=op, dtype=dtype, M=_log(rng, 1, max(1, 40_000_000 // C)), C=C)


# -------------------------------------------------------------------------------------- the 8-bit format
def _pack(x, dtype):
    """(codes int8 [..., C], scale bytes uint8 [..., ceil(C / 32)]) of values of the storage type, or about to be rounded to it."""
    C = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, -C % GROUP)).unflatten(-1, (-1, GROUP))
    part, power = torch.frexp(x.abs().amax(dim=-1))
    e = (power - torch.where(part <= 127 / 128, 7, 6)).clamp(*EXPONENTS[dtype])
    codes = torch.round(torch.ldexp(x, -e.unsqueeze(-1))).clamp(-127, 127)
    return codes.flatten(-2)[..., :C].to(torch.int8), (e + 127).to(torch.uint8)


def _unpack(packed):
    codes, scales = packed
    C = codes.shape[-1]
    e = torch.repeat_interleave(scales, GROUP, dim=-1)[..., :C].int() - 127
    return torch.ldexp(codes.float(), e)


# -------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)  # noqa: E731
    s = {"linear": _prepare_linear, "recurrence": _prepare_recurrence, "pack8": _prepare_pack8}[case["op"]](case, randn, dtype)
    s["case"] = case
    if own:  # the plan that a program makes once per layer
        from paper_2409_02097_b200 import layers
        if case["op"] == "linear":
            s["plan"] = layers.Linear(case["K"], case["N"], activation=case["act"], dtype=case["dtype"])
        elif case["op"] == "recurrence":
            s["plan"] = layers.GatedRecurrence(case["C"], reverse=case["reverse"], dtype=case["dtype"])
    return s


def _outliers(x):
    """Activations as layers leave them: one channel in 61 is larger than the others."""
    x[..., ::61] *= 8
    return x


def _prepare_linear(case, randn, dtype):
    M, K, N = case["M"], case["K"], case["N"]
    s = dict(x=_outliers(randn(M, K)).to(dtype))
    if case["transposed"]:  # kept [outputs, inputs], seen as [inputs, outputs]
        s["w"] = (randn(N, K) / math.sqrt(K)).to(dtype).t()
    else:
        s["w"] = (randn(K, N) / math.sqrt(K)).to(dtype)
    if case["bias"]:
        s["bias"] = (0.2 * randn(N)).to(dtype)
    if case["residual"] and case["what"].startswith("forward"):
        s["residual"] = randn(M, N).to(dtype)
    if case["what"].startswith("backward"):  # fp16 gradients come loss-scaled
        s["dy"] = (randn(M, N) * (16.0 if dtype == torch.float16 else 1.0)).to(dtype)
        if case["save"]:  # the pre-activation as the forward pass left it
            s["u"] = _product(s).to(dtype)
        if case["what"] == "backward8":
            s.update({n + "8": _pack(s.pop(n).float(), dtype) for n in ("x", "u") if n in s})
    return s


def _prepare_recurrence(case, randn, dtype):
    B, N, C = case["B"], case["N"], case["C"]
    names = ("x", "decay") + (("gate",) if case["gate"] else ())
    # the projections lie side by side in one tensor, as a product leaves them
    proj = randn(B, N, len(names) * C)
    s = {n: proj[..., k * C:(k + 1) * C] for k, n in enumerate(names)}
    s["x"] += 0.2
    s["decay"] *= 1.5
    if case["padded"]:  # tokens that count for nothing: their decay is switched off
        s["decay"][:, N - case["padded"]:] = -math.inf
    proj = proj.to(dtype)
    s = {n: proj[..., k * C:(k + 1) * C] for k, n in enumerate(names)}
    # memories of a few to some thousand tokens
    s["rate"] = torch.exp(-7.0 * torch.sigmoid(1.5 * randn(C)))
    if case["h0"]:
        s["h0"] = randn(B, C)
    if case["what"] != "forward":
        s["dh"] = randn(B, N, C).to(dtype)
        if case["h0"]:
            s["dlast"] = randn(B, C)
        if case["saved"]:  # the states before every 64th token, as the forward pass kept them
            s["state"] = _chunk_states(_forward(_gates(case, s), s.get("h0")), s.get("h0")).float()
        if case["what"] == "backward8":  # infinities have no place in 8 bits: padding is saved as a number that decays nothing
            for n in names:
                t = s.pop(n)
                t = t.float().clamp(min=-96.0) if n == "decay" else t.float()
                s[n + "8"] = _pack(t, dtype)
    return s


def _prepare_pack8(case, randn, dtype):
    return dict(x=_outliers(randn(case["M"], case["C"])).to(dtype))


# -------------------------------------------------------------------------------------- plain forms
def _act(u, kind):
    if kind == "relu":
        return torch.clamp(u, min=0)
    if kind == "silu":
        return u * torch.sigmoid(u)
    if kind == "gelu":
        return 0.5 * u * (1 + torch.erf(u * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * u * (1 + torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3)))
    return u


def _act_slope(u, kind):
    if kind == "relu":
        return (u > 0).to(u.dtype)
    if kind == "silu":
        p = torch.sigmoid(u)
        return p * (1 + u * (1 - p))
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (u + 0.044715 * u ** 3))
        return 0.5 * (1 + t) + 0.5 * u * (1 - t * t) * c * (1 + 3 * 0.044715 * u * u)
    return torch.ones_like(u)


def _product(s):
    u = s["x"].float() @ s["w"].float()
    return u + s["bias"].float() if "bias" in s else u


def _run_linear(case, s):
    dtype, act, out = DTYPES[case["dtype"]], case["act"], {}
    if case["what"].startswith("forward"):
        u = _product(s)
        y = _act(u, act)
        out["y"] = (y + s["residual"].float() if "residual" in s else y).to(dtype)
        if case["save"]:
            out["u"] = u.to(dtype) if case["what"] == "forward" else _unpack(_pack(u, dtype)).to(dtype)
        return out
    x = _unpack(s["x8"]) if "x8" in s else s["x"].float()
    u = _unpack(s["u8"]) if "u8" in s else s["u"].float() if "u" in s else None
    du = s["dy"].float()
    if u is not None:
        du = du * _act_slope(u, act)
    out["dx"] = (du @ s["w"].float().t()).to(dtype)
    out["dw"] = (x.t() @ du).to(dtype)
    if case["bias"]:
        out["dbias"] = du.sum(dim=0)
    return out


def _gates(case, s):
    """The recurrence's inputs in the order of the scan: x, sigmoid(decay), sigmoid(gate) or None.  In 64 bits: products of
    thousands of decays near one, and sums of terms that cancel."""
    get = lambda n: _unpack(s[n + "8"]).double() if n + "8" in s else s[n].double() if n in s else None  # noqa: E731
    x, decay, gate = (get(n) for n in ("x", "decay", "gate"))
    g = dict(x=x, p=torch.sigmoid(decay), q=None if gate is None else torch.sigmoid(gate))
    g = {n: t.flip(1) if t is not None and case["reverse"] else t for n, t in g.items()}
    L = s["rate"] * g["p"]
    g["a"], g["e"] = torch.exp(-L), -torch.expm1(-L)
    g["v"] = g["x"] if g["q"] is None else g["q"] * g["x"]
    return g


def _scan(a, b, first):
    """h_t = a_t h_(t-1) + b_t along dim 1 from h_0 = first (or zero), by doubling the steps that are joined."""
    a, h = a.clone(), b.clone()
    if first is not None:
        h[:, 0] += a[:, 0] * first
    n = 1
    while n < h.shape[1]:
        h[:, n:] += a[:, n:] * h[:, :-n].clone()
        a[:, n:] = a[:, n:] * a[:, :-n].clone()
        n *= 2
    return h


def _forward(g, h0):
    return _scan(g["a"], g["e"] * g["v"], h0)


def _chunk_states(h, h0):
    """The states before tokens 0, 64, 128, ... of the scan."""
    first = torch.zeros_like(h[:, :1]) if h0 is None else h0.unsqueeze(1)
    return torch.cat([first, h[:, EVERY - 1:-1:EVERY]], dim=1).contiguous()


def _states_before(g, s):
    """h_(t-1) for every token: from the saved states each stretch of 64 tokens by itself, else by the whole scan."""
    if "state" not in s:
        h = _forward(g, s.get("h0"))
        first = torch.zeros_like(h[:, :1]) if "h0" not in s else s["h0"].unsqueeze(1)
        return torch.cat([first, h[:, :-1]], dim=1)
    B, N, C = g["a"].shape
    cut = lambda t: torch.nn.functional.pad(t, (0, 0, 0, -N % EVERY)).reshape(-1, EVERY, C)  # noqa: E731
    first = s["state"].reshape(-1, C)
    h = _scan(cut(g["a"]), cut(g["e"] * g["v"]), first)
    return torch.cat([first.unsqueeze(1), h[:, :-1]], dim=1).reshape(B, -1, C)[:, :N]


def _run_recurrence(case, s):
    dtype, turn = DTYPES[case["dtype"]], lambda t: t.flip(1) if case["reverse"] else t  # noqa: E731
    g = _gates(case, s)
    if case["what"] == "forward":
        h = _forward(g, s.get("h0"))
        out = {"h": turn(h).to(dtype), "last": h[:, -1].float()}
        if case["save"]:
            out["state"] = _chunk_states(h, s.get("h0")).float()
        return out
    before = _states_before(g, s)
    dh = turn(s["dh"].double())
    if "dlast" in s:
        dh = dh.clone()
        dh[:, -1] += s["dlast"]
    # G_t = dh_t + a_(t+1) G_(t+1)
    after = torch.cat([g["a"][:, 1:], torch.zeros_like(g["a"][:, :1])], dim=1)
    G = _scan(after.flip(1), dh.flip(1), None).flip(1)
    dv, dL = g["e"] * G, G * (g["v"] - before) * g["a"]
    out = {"x": dv if g["q"] is None else dv * g["q"], "decay": dL * s["rate"] * g["p"] * (1 - g["p"])}
    if g["q"] is not None:
        out["gate"] = dv * g["x"] * g["q"] * (1 - g["q"])
    out = {n: turn(t).to(dtype) for n, t in out.items()}
    out["rate"] = (dL * g["p"]).sum(dim=(0, 1)).float()
    if "h0" in s:
        out["h0"] = (g["a"][:, 0] * G[:, 0]).float()
    return out


def _run_pack8(case, s):
    dtype = DTYPES[case["dtype"]]
    return {"values": _unpack(_pack(s["x"].float(), dtype)).to(dtype)}


# -------------------------------------------------------------------------------------- one pass
def _own_linear(case, s):
    plan, given = s["plan"], {n: s[n] for n in ("bias", "residual") if n in s}
    need = ("x", "w", "bias") if case["bias"] else ("x", "w")
    if case["what"].startswith("forward"):
        save = ("full" if case["what"] == "forward" else "packed") if case["save"] else None
        y, u = plan.forward(s["x"], s["w"], save=save, **given)
        return {"y": y, "u": u.unpack() if save == "packed" else u} if save else {"y": y}
    from paper_2409_02097_b200 import layers
    get = lambda n: layers.Packed8(*s[n + "8"], case["dtype"]) if n + "8" in s else s.get(n)  # noqa: E731
    grads = plan.backward(s["dy"], get("x"), s["w"], u=get("u"), need=need)
    return {"d" + n: t for n, t in grads.items()}


def _own_recurrence(case, s):
    from paper_2409_02097_b200 import layers
    plan = s["plan"]
    get = lambda n: layers.Packed8(*s[n + "8"], case["dtype"]) if n + "8" in s else s.get(n)  # noqa: E731
    x, decay, gate = get("x"), get("decay"), get("gate")
    if case["what"] == "forward":
        h, last, state = plan.forward(x, decay, s["rate"], gate=gate, h0=s.get("h0"), save=case["save"])
        return {"h": h, "last": last, "state": state} if case["save"] else {"h": h, "last": last}
    return plan.backward(s["dh"], x, decay, s["rate"], gate=gate, h0=s.get("h0"), state=s.get("state"), dlast=s.get("dlast"))


def _own_pack8(case, s):
    from paper_2409_02097_b200 import layers
    return {"values": layers.pack8(s["x"]).unpack()}


def run(s):
    case = s["case"]
    if own:
        return {"linear": _own_linear, "recurrence": _own_recurrence, "pack8": _own_pack8}[case["op"]](case, s)
    return {"linear": _run_linear, "recurrence": _run_recurrence, "pack8": _run_pack8}[case["op"]](case, s)


# -------------------------------------------------------------------------------------- work
def work(case):
    packed = lambda rows, C: rows * (C + -(-C // GROUP))  # noqa: E731  bytes of codes and scales
    if case["op"] == "pack8":
        M, C = case["M"], case["C"]
        return {"bytes": 4 * M * C + 2 * packed(M, C), "flops": 6 * M * C}
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        if case["what"].startswith("forward"):
            values = M * K + K * N + M * N * (1 + case["residual"]) + N * case["bias"]
            kept = 0 if not case["save"] else 2 * M * N if case["what"] == "forward" else 2 * packed(M, N) + 2 * M * N
            return {"bytes": 2 * values + kept, "flops": 2 * M * K * N}
        # reads dY and W, and X and the pre-activation; writes dX and dW, and dbias in 32 bits
        kept = packed if case["what"] == "backward8" else lambda rows, C: 2 * rows * C  # noqa: E731
        read = kept(M, K) + (kept(M, N) if case["save"] else 0)
        return {"bytes": 2 * (M * N + 2 * K * N + M * K) + read + 4 * N * case["bias"], "flops": 4 * M * K * N}
    B, N, C = case["B"], case["N"], case["C"]
    inputs, states = 3 if case["gate"] else 2, 4 * B * C * -(-N // EVERY)
    ends = 4 * C + 4 * B * C * (1 + case["h0"])
    if case["what"] == "forward":
        return {"bytes": 2 * B * N * C * (inputs + 1) + states * case["save"] + ends, "flops": 20 * B * N * C}
    read = inputs * (packed(B * N, C) if case["what"] == "backward8" else 2 * B * N * C)
    return {"bytes": read + 2 * B * N * C * (1 + inputs) + states * case["saved"] + 2 * ends, "flops": 50 * B * N * C}


# -------------------------------------------------------------------------------------- 64 bits
def _exact_pack8(x, dtype):
    """The nearest of the 255 steps of each value's group, by the definition of the step."""
    x = x.double()
    lo, hi = EXPONENTS[dtype]
    out = torch.empty_like(x)
    for c in range(0, x.shape[-1], GROUP):
        group = x[..., c:c + GROUP]
        most = group.abs().amax(dim=-1, keepdim=True)
        e = torch.ceil(torch.log2(torch.clamp(most, min=1e-300) / 127))
        e = torch.where(most > 127 * torch.exp2(e), e + 1, e)
        e = torch.where(most <= 127 * torch.exp2(e - 1), e - 1, e)
        step = torch.exp2(e.clamp(lo, hi))
        out[..., c:c + GROUP] = torch.clamp(torch.round(group / step), -127, 127) * step
    return out


def _exact_values(packed):
    codes, scales = packed
    return codes.double() * torch.exp2(scales.double() - 127).repeat_interleave(GROUP, -1)[..., :codes.shape[-1]]


def _exact_act(u, kind):
    if kind == "relu":
        return torch.nn.functional.relu(u)
    if kind == "silu":
        return u / (1 + torch.exp(-u))
    if kind == "gelu":
        return u * torch.special.ndtr(u)
    if kind == "gelu_tanh":
        z = math.sqrt(2 / math.pi) * (u + 0.044715 * u * u * u)
        return u / (1 + torch.exp(-2 * z))
    return u


def _exact_linear(case, s):
    t = {n: x.double() for n, x in s.items() if torch.is_tensor(x)}
    out = {}
    if case["what"].startswith("forward"):
        u = torch.addmm(t["bias"], t["x"], t["w"]) if "bias" in t else torch.mm(t["x"], t["w"])
        out["y"] = _exact_act(u, case["act"]) + t.get("residual", 0.0)
        if case["save"]:
            out["u"] = u if case["what"] == "forward" else _exact_pack8(u, DTYPES[case["dtype"]])
        return out
    if case["what"] == "backward8":
        t.update({n: _exact_values(s[n + "8"]) for n in ("x", "u") if n + "8" in s})
    du = t["dy"]
    if case["act"] != "none":  # the slope by differentiation of the definition
        u = t["u"].requires_grad_(True)
        du, = torch.autograd.grad((_exact_act(u, case["act"]) * du).sum(), u)
    out["dx"], out["dw"] = torch.einsum("mn,kn->mk", du, t["w"]), torch.einsum("mk,mn->kn", t["x"], du)
    if case["bias"]:
        out["dbias"] = du.sum(0)
    return out


def _exact_recurrence(case, s):
    """Token by token, there and back."""
    back = slice(None, None, -1) if case["reverse"] else slice(None)
    B, N, C = case["B"], case["N"], case["C"]

    def get(n):
        return _exact_values(s[n + "8"]) if n + "8" in s else s[n].double() if n in s else None

    x, decay, gate = get("x"), get("decay"), get("gate")
    order = range(N)[back]
    rate = s["rate"].double()
    L = rate / (1 + torch.exp(-decay))
    a, e = torch.exp(-L), -torch.expm1(-L)
    q = None if gate is None else 1 / (1 + torch.exp(-gate))
    v = x if q is None else x * q
    h = s["h0"].double() if "h0" in s else torch.zeros(B, C, dtype=torch.float64, device="cuda")
    before = torch.empty_like(x)
    b = e * v
    states = []
    for i, t in enumerate(order):
        if i % EVERY == 0:
            if "state" in s:
                h = s["state"][:, i // EVERY].double()
            states.append(h)
        before[:, t] = h
        h = torch.addcmul(b[:, t], a[:, t], h)
    if case["what"] == "forward":
        out = {"h": a * before + b, "last": h}
        if case["save"]:
            out["state"] = torch.stack(states, dim=1)
        return out
    G = torch.empty_like(x)
    dh = s["dh"].double()
    carry = s["dlast"].double() if "dlast" in s else torch.zeros(B, C, dtype=torch.float64, device="cuda")
    for t in reversed(order):
        torch.add(dh[:, t], carry, out=carry)
        G[:, t] = carry
        carry = a[:, t] * carry
    dL = G * (v - before) * a
    out = {"x": G * e if q is None else G * e * q, "decay": dL * L / (1 + torch.exp(decay))}
    out["decay"] = torch.where(torch.isinf(decay), torch.zeros_like(L), out["decay"])
    if q is not None:
        out["gate"] = G * e * x * q / (1 + torch.exp(gate))
    out["rate"] = (dL / (1 + torch.exp(-decay))).sum(dim=(0, 1))
    if "h0" in s:
        out["h0"] = carry
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "pack8":
        return {"values": _exact_pack8(s["x"], DTYPES[case["dtype"]])}
    return {"linear": _exact_linear, "recurrence": _exact_recurrence}[case["op"]](case, s)
