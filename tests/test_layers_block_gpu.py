"""A transformer block of this framework's own parts: norms, projections, attention and feed-forward layers, forward and back, against 64 bits."""
import math

import pytest
import torch

import _block_ref as block_ref
import _layers_ref as ref

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
B, N, H, D = 2, 300, 2, 64
C, F = H * D, 4 * H * D


def _make(dtype, packed):
    from paper_2409_02097_b200 import attn, block, layers
    op = attn.LinFusionAttention(B, H, N, D, layout="token_major", dtype=dtype)
    norm = block.BlockNorm(C, pre="layer", post="none", dtype=dtype)
    proj, up, down = layers.Linear(C, C, dtype=dtype), layers.Linear(C, F, "gelu", dtype=dtype), layers.Linear(F, C, dtype=dtype)
    keep = layers.pack8 if packed else (lambda t: t)

    def run(s):
        heads = lambda t: t.view(B, N, H, D)  # noqa: E731
        _, n0 = norm.forward(s["x"])
        q, k, v = (heads(proj.forward(n0, s[w])[0]) for w in ("wq", "wk", "wv"))
        a = op.forward(q, k, v)
        state = op.save_state()
        y, _ = proj.forward(a.view(B, N, C), s["wo"], residual=s["x"])
        _, n1 = norm.forward(y)
        m, u = up.forward(n1, s["w1"], s["b1"], save="packed" if packed else "full")
        z, _ = down.forward(m, s["w2"], s["b2"], residual=y)
        kept = [keep(t) for t in (n0, a.view(B, N, C), n1, m)]
        g2 = down.backward(s["dz"], kept[3], s["w2"])
        g1 = up.backward(g2["x"], kept[2], s["w1"], u=u)
        dy = norm.backward(y, dn=g1["x"], dy=s["dz"])["x"]
        go = proj.backward(dy, kept[1], s["wo"], need=("x", "w"))
        dqkv = op.backward(q, k, v, heads(go["x"]), state=state)
        back = [proj.backward(t.view(B, N, C), kept[0], s[w], need=("x", "w")) for t, w in zip(dqkv, ("wq", "wk", "wv"))]
        dn0 = sum(b["x"].float() for b in back).to(TYPES[dtype])
        dx = norm.backward(s["x"], dn=dn0, dy=dy)["x"]
        return dict(z=z, x=dx, wq=back[0]["w"], wk=back[1]["w"], wv=back[2]["w"], wo=go["w"], w1=g1["w"], b1=g1["bias"], w2=g2["w"], b2=g2["bias"])

    return run, op


def _state(dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    shapes = dict(x=(B, N, C), dz=(B, N, C), wq=(C, C), wk=(C, C), wv=(C, C), wo=(C, C), w1=(C, F), b1=(F,), w2=(F, C), b2=(C,))
    s = {n: torch.randn(sh, generator=g, device="cuda") for n, sh in shapes.items()}
    return {n: (t / (math.sqrt(t.shape[0]) if n[0] == "w" else 1.0)).to(TYPES[dtype]) for n, t in s.items()}


def _exact(s):
    leaves = {n: t.double().requires_grad_(n != "dz") for n, t in s.items()}
    x = leaves["x"]
    n0 = block_ref.normed(x, "layer", 1e-6)
    q, k, v = ((n0 @ leaves[w]).view(B, N, H, D).transpose(1, 2) for w in ("wq", "wk", "wv"))
    fq, fk = (torch.nn.functional.elu(t) + 1 for t in (q, k))
    a = fq @ (fk.transpose(-1, -2) @ v) / (fq @ fk.sum(-2).unsqueeze(-1) + 1e-6)
    y = a.transpose(1, 2).reshape(B, N, C) @ leaves["wo"] + x
    z = torch.nn.functional.gelu(block_ref.normed(y, "layer", 1e-6) @ leaves["w1"] + leaves["b1"]) @ leaves["w2"] + leaves["b2"] + y
    names = [n for n in leaves if n != "dz"]
    return dict(zip(names, torch.autograd.grad((z * leaves["dz"]).sum(), [leaves[n] for n in names])), z=z.detach())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("packed", [False, True])
def test_a_block_of_all_parts(packed, dtype):
    from paper_2409_02097_b200 import attn, layers
    run, op = _make(dtype, packed)
    s = _state(dtype, 90)
    got, want = run(s), _exact(s)
    for n in want:
        rel = ((got[n].double() - want[n]).norm() / want[n].norm()).item()
        # at most sixteen roundings to 16 bits from the inputs to a gradient, each 0.6 of half a step in the 2-norm; the attention keeps its states in 16
        # bits as well (four more, forward and back).  Checkpoints add 0.8 % each, of which two or three meet
        most = 20 * 0.6 * ref.HALF_STEP[TYPES[dtype]] + (0.025 if packed and n != "z" else 0.0)
        assert rel <= most, (n, rel, most)
    assert layers.expired() == 0 and op.backward_status() == attn.OK
    op.close()


def test_a_block_captured_and_replayed():
    run, op = _make("bf16", True)
    s = _state("bf16", 91)
    want = {k: run(_state("bf16", k)) for k in (92, 93)}
    run(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(s)
    for k in (92, 93, 92):
        for n, v in _state("bf16", k).items():
            s[n].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[k][n]) for n in out)
    op.close()
