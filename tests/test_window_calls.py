"""The window heads' binding without a GPU: what reaches the library, call by call.  The library is
a stand-in that keeps the structs it is given; tensors say that they are on a GPU."""
import contextlib
import ctypes
import math
import types

import pytest
import torch

from paper_2505_00315_gb300 import _window as W


class OnGpu(torch.Tensor):
    """A tensor of the host that passes for one of the GPU."""
    is_cuda = True


class Library:
    """Keeps the struct of each call."""
    bytes = 256

    def __init__(self):
        self.seen = []

    def __getattr__(self, name):
        def call(ref, *args):
            if name.endswith("_bytes"):
                return self.bytes
            s = ref._obj
            self.seen.append((name, {n: getattr(s, n) for n, t in s._fields_
                                     if t in (ctypes.c_int32, ctypes.c_float)}, args))
            return 0
        return call

    def last(self, field):
        return self.seen[-1][1][field]


@pytest.fixture
def lib(monkeypatch):
    L = Library()
    monkeypatch.setattr(W._b, "load", lambda: L)
    monkeypatch.setattr(W._b, "_stream", lambda stream: 0)
    monkeypatch.setattr(W, "_plans", {})
    W._b._torch()
    return L


def t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


Q, K = t(2, 8, 4, 64), t(2, 8, 2, 64)
LSE, SPACE = t(2, 4, 8), t(256, dtype=torch.uint8)
CACHE, LENS = t(2, 8, 2, 64), t(2, dtype=torch.int32)
DG = {"dgamma_q": t(64), "dgamma_k": t(64)}


def forward(window=4, sinks=1, scale=0.0):
    return W.mosa_window_forward(Q, K, K, window, sinks, scale=scale, workspace=SPACE, out={"O": Q, "lse": LSE})


def backward(window=4, sinks=1, scale=0.0):
    return W.mosa_window_backward(Q, K, K, Q, LSE, Q, SPACE, window, sinks, scale=scale)


def norm(**kw):
    return W.mosa_qk_norm_rope(Q, K, **kw)


def norm_backward(**kw):
    return W.mosa_qk_norm_rope_backward(Q, K, None, None, Q, K, workspace=SPACE, out=DG, **kw)


def decode(window=4, sinks=1, **kw):
    return W.mosa_window_decode(Q[:, 0], K[:, 0], K[:, 0], CACHE, CACHE, LENS, window, sinks, workspace=SPACE,
                                out={"O": t(2, 4, 64)}, **kw)


FLOATS = [(forward, "scale"), (backward, "scale"), (decode, "scale")] + [
    (f, n) for f in (norm, norm_backward, decode) for n in ("theta", "eps")]
INTS = [(f, n) for f in (forward, backward, decode) for n in ("window", "sinks")] + [
    (f, "rotary") for f in (norm, norm_backward, decode)]


@pytest.mark.parametrize("call,name", FLOATS, ids=lambda x: getattr(x, "__name__", x))
def test_a_number_that_changes_in_place_counts_at_every_call(call, name, lib):
    """A learned scale, say: the optimizer writes to the same tensor."""
    x = torch.tensor(1.5)
    call(**{name: x})
    assert lib.last(name) == 1.5
    x.fill_(2.5)
    call(**{name: x})
    assert lib.last(name) == 2.5
    call(**{name: 3})
    assert lib.last(name) == 3.0


@pytest.mark.parametrize("call,name", INTS, ids=lambda x: getattr(x, "__name__", x))
def test_an_integer_that_changes_in_place_counts_at_every_call(call, name, lib):
    x = torch.tensor(2)
    call(**{name: x})
    assert lib.last(name) == 2
    x.fill_(4)
    call(**{name: x})
    assert lib.last(name) == 4


@pytest.mark.parametrize("call,name", INTS, ids=lambda x: getattr(x, "__name__", x))
def test_what_is_refused_is_refused_after_an_equal_integer_too(call, name, lib):
    call(**{name: 4})
    with pytest.raises(TypeError):
        call(**{name: 4.0})


@pytest.mark.parametrize("call,name", [(norm, "halves"), (norm_backward, "halves"), (decode, "halves"),
                                       (decode, "norm")], ids=lambda x: getattr(x, "__name__", x))
def test_a_truth_value_that_changes_in_place_counts_at_every_call(call, name, lib):
    x = torch.tensor(False)
    call(**{name: x})
    assert lib.last(name) == 0
    x.fill_(True)
    call(**{name: x})
    assert lib.last(name) == 1


def test_equal_calls_share_a_plan(lib):
    for _ in range(3):
        forward(scale=0.25), forward(scale=torch.tensor(0.25)), norm(theta=100), norm(theta=100.0)
    assert len(W._plans) == 2 and all(math.isclose(s["scale"], 0.25) for n, s, _ in lib.seen
                                      if n == "mosa_window_forward")


ON_A_STREAM = {
    "norm": lambda S: W.mosa_qk_norm_rope(Q, K, stream=S),
    "norm_backward": lambda S: W.mosa_qk_norm_rope_backward(Q, K, None, None, Q, K, stream=S),
    "forward": lambda S: W.mosa_window_forward(Q, K, K, 4, stream=S),
    "backward": lambda S: W.mosa_window_backward(Q, K, K, Q, LSE, Q, SPACE, 4, stream=S),
    "decode": lambda S: W.mosa_window_decode(Q[:, 0], K[:, 0], K[:, 0], CACHE, CACHE, LENS, 4, stream=S),
}


@pytest.mark.parametrize("call", ON_A_STREAM.values(), ids=ON_A_STREAM)
def test_results_and_workspaces_of_a_call_for_a_stream_are_of_that_stream(call, lib, monkeypatch):
    """Made, and zeroed, on another stream they could still be in use there, or be zeroed after the
    call's kernels have written them."""
    current, made = [0], []

    @contextlib.contextmanager
    def stream(x):
        current.append(x.cuda_stream)
        yield
        current.pop()

    def on(f):
        def make(*args, **kw):
            made.append(current[-1])
            return f(*args, **kw).as_subclass(OnGpu)
        return make

    S = types.SimpleNamespace(cuda_stream=77)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda n: types.SimpleNamespace(cuda_stream=n))
    monkeypatch.setattr(W._b, "_stream", lambda x: current[-1] if x is None else x.cuda_stream)
    for name in ("empty", "zeros", "empty_like"):
        monkeypatch.setattr(torch, name, on(getattr(torch, name)))
    call(S)
    assert lib.seen[-1][2][-1] == 77          # where the kernels go
    assert made and set(made) == {77}
    assert current == [0]


ALL = {
    "norm": lambda **kw: W.mosa_qk_norm_rope(Q, K, **kw),
    "norm_backward": lambda **kw: W.mosa_qk_norm_rope_backward(Q, K, None, None, Q, K, workspace=SPACE, **kw),
    "forward": lambda **kw: W.mosa_window_forward(Q, K, K, 4, workspace=SPACE, **kw),
    "backward": lambda **kw: W.mosa_window_backward(Q, K, K, Q, LSE, Q, SPACE, 4, **kw),
    "decode": lambda **kw: W.mosa_window_decode(Q[:, 0], K[:, 0], K[:, 0], CACHE, CACHE, LENS, 4, workspace=SPACE,
                                                **kw),
}


@pytest.fixture
def on_gpu(monkeypatch):
    """New tensors pass for ones of the GPU too."""
    for name in ("empty", "zeros", "empty_like"):
        f = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, _f=f, **kw: _f(*a, **kw).as_subclass(OnGpu))


@pytest.mark.parametrize("call", ALL.values(), ids=ALL)
def test_out_may_hold_nothing(call, lib, on_gpu):
    for out in ({}, None, {"unused": 1}):
        call(out=out)
    assert len(lib.seen) == 3


def test_the_librarys_own_refusal_is_what_a_call_raises(monkeypatch, on_gpu):
    """A head size that it does not support, and a rotation that is no even number, with and without a
    workspace."""
    monkeypatch.setattr(W._b, "_stream", lambda stream: 0)
    q, k, lse, kc = t(2, 8, 4, 48), t(2, 8, 2, 48), t(2, 4, 8), t(2, 8, 2, 48)
    for ws in (None, SPACE):
        for call in (lambda: W.mosa_qk_norm_rope(q, k),
                     lambda: W.mosa_qk_norm_rope_backward(q, k, None, None, q, k, workspace=ws),
                     lambda: W.mosa_window_forward(q, k, k, 4, workspace=ws),
                     lambda: W.mosa_window_backward(q, k, k, q, lse, q, SPACE, 4),
                     lambda: W.mosa_window_decode(q[:, 0], k[:, 0], k[:, 0], kc, kc, LENS, 4, workspace=ws)):
            with pytest.raises(W._b.MosaError) as e:
                call()
            assert e.value.code == W._b.MOSA_ERR_UNSUPPORTED
        for call in (lambda: W.mosa_qk_norm_rope(Q, K, rotary=7),
                     lambda: W.mosa_qk_norm_rope_backward(Q, K, None, None, Q, K, rotary=7, workspace=ws),
                     lambda: W.mosa_window_forward(Q, K, K, -4, workspace=ws),
                     lambda: W.mosa_window_decode(Q[:, 0], K[:, 0], K[:, 0], CACHE, CACHE, LENS, -4, workspace=ws)):
            with pytest.raises(W._b.MosaError) as e:
                call()
            assert e.value.code == W._b.MOSA_ERR_INVALID_ARG


def test_a_new_workspace_is_as_large_as_its_call_needs(lib, on_gpu, monkeypatch):
    """... and only its status word is zeroed: the rest may be large."""
    zeroed = []
    zero_ = torch.Tensor.zero_
    monkeypatch.setattr(torch.Tensor, "zero_", lambda x: (zeroed.append(x.numel()), zero_(x))[1])
    monkeypatch.setattr(torch, "zeros", lambda n, *a, **kw: zeroed.append(n) or torch.full((n,), 0, **kw))
    monkeypatch.setattr(Library, "bytes", 4096)
    O, lse, ws = W.mosa_window_forward(Q, K, K, 4)
    assert ws.numel() == 4096 and set(zeroed) == {4} and (ws[:4] == 0).all()
    O, lse, ws = W.mosa_window_forward(Q, K, K, 4, want_lse=False)
    assert lse is None and ws.numel() == 256 and set(zeroed) == {4}
    assert lib.seen[-1][2][-2] == 256
    zeroed.clear()
    _, ws = W.mosa_qk_norm_rope_backward(Q, K, None, None, Q, K)
    assert ws.numel() == 4096
    _, ws = W.mosa_window_decode(Q[:, 0], K[:, 0], K[:, 0], CACHE, CACHE, LENS, 4)
    assert ws.numel() == 4096 and not zeroed
