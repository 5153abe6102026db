"""The binding of the attention's backward pass, as far as no GPU is needed: stand-ins for the library and for device memory."""
import contextlib
import ctypes
import gc
import weakref

import pytest
import torch

from paper_2409_02097_b200 import attn


class _OnDevice(torch.Tensor):
    """A host tensor that says it is on device 0: the binding reads shapes and addresses, the stand-in library reads nothing."""
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", 0))

    def get_device(self):
        return 0


class _Library:
    """Every entry point answers OK after `during`, with the arguments that it was given."""

    def __init__(self, during):
        self.during, self.calls = during, []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            self.during(name, args)
            return attn.OK
        return call


B, H, N, D = 1, 2, 8, 64


@pytest.fixture
def made(monkeypatch):
    """Weak references to what the binding allocates, in order."""
    refs, empty, empty_like = [], torch.empty, torch.empty_like

    def note(t):
        t = t.as_subclass(_OnDevice)
        refs.append(weakref.ref(t))
        return t

    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: note(empty(*a, **kw)))
    monkeypatch.setattr(torch, "empty_like", lambda t, **kw: note(empty_like(t.as_subclass(torch.Tensor), **kw)))
    monkeypatch.setattr(attn, "allocating_on", lambda stream, index: contextlib.nullcontext())
    return refs


def _op(during=lambda name, args: None):
    op = object.__new__(attn.LinFusionAttention)
    op.desc, op.dtype, op.dk = attn.make_desc(B, H, N, D), "bf16", D
    op.shape = op.shape_qk = (B, H, N, D)
    op._lib, op._h, op._lent_ws, op._backward_bytes = _Library(during), None, None, 4096
    return op


def _inputs():
    return [torch.zeros(B, H, N, D, dtype=torch.bfloat16).as_subclass(_OnDevice) for _ in range(4)]


def _state():
    return torch.zeros(B * H, D * D + D).as_subclass(_OnDevice)


CALLS = {
    "linfusion_attn_backward": lambda op, q, k, v, dy: op.backward(q, k, v, dy, stream=1),
    "linfusion_attn_backward_state": lambda op, q, k, v, dy: op.backward_state(k, v, stream=1),
    "linfusion_attn_backward_q": lambda op, q, k, v, dy: op.backward_q(q, dy, _state(), stream=1),
    "linfusion_attn_backward_kv": lambda op, q, k, v, dy: op.backward_kv(k, v, _state(), stream=1),
}


@pytest.mark.parametrize("name", CALLS)
def test_what_a_call_allocates_lives_until_its_kernels_are_enqueued(made, name):
    # a thread that runs while the library is entered must not be handed the call's workspace or outputs
    alive = []

    def during(called, args):
        gc.collect()
        alive.append([r() is not None for r in made])

    op = _op(during)
    CALLS[name](op, *_inputs())
    assert op._lib.calls == [name]
    assert len(alive) == 1 and len(alive[0]) >= 2 and all(alive[0]), alive


def test_an_expired_wait_is_reported_without_a_workspace(monkeypatch):
    # the count of the device stands for the workspaces that calls made for themselves and dropped
    count = [0]

    def during(name, args):
        assert name == "linfusion_attn_backward_expired" and args[0] == 0
        args[1]._obj.value = count[0]

    lib = _Library(during)
    monkeypatch.setattr(attn, "load_library", lambda: lib)
    monkeypatch.setattr(attn, "_expired_known", {})
    op, other = _op(), _op()
    for o in (op, other):
        o._expired_seen = 0
    assert op.backward_status(stream=1) == attn.OK
    count[0] = 3
    assert op.backward_status(stream=1) == attn.ERR_TIMEOUT  # once
    assert op.backward_status(stream=1) == attn.OK
    assert other.backward_status(stream=1) == attn.ERR_TIMEOUT
    assert attn._expired_known == {0: 3}                      # where objects made from now on begin
    from paper_2409_02097_b200 import sharding
    shard = object.__new__(sharding.TokenShardedAttention)
    shard.op = type("Op", (), {"backward_status": lambda self: attn.ERR_TIMEOUT})()
    assert shard.backward_status() == attn.ERR_TIMEOUT


def test_the_count_of_expired_waits_refuses_bad_arguments():
    lib, n = attn.load_library(), ctypes.c_uint32(0)
    assert lib.linfusion_attn_backward_expired(0, None, None) == attn.ERR_INVALID_ARG
    assert lib.linfusion_attn_backward_expired(-1, ctypes.byref(n), None) == attn.ERR_INVALID_ARG
    desc = attn.make_desc(B, H, N, D)
    for ws in (0, 4096 + 16):
        assert lib.linfusion_attn_selftest_backward_wait(ctypes.byref(desc), ws, None) == attn.ERR_INVALID_ARG
    if not torch.cuda.is_available():
        assert lib.linfusion_attn_backward_expired(0, ctypes.byref(n), None) == attn.ERR_CUDA


def test_refusals_name_the_tensor(made):
    op = _op()
    q, k, v, dy = _inputs()
    for name, call in (("dy", lambda bad: op.backward(q, k, v, bad, stream=1)), ("dq", lambda bad: op.backward(q, k, v, dy, dq=bad, stream=1)),
                       ("dv", lambda bad: op.backward_kv(k, v, _state(), dv=bad, stream=1))):
        with pytest.raises(ValueError, match=rf"^{name}: "):
            call(q[:, :1])
