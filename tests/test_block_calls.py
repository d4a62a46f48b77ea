"""The block operators' binding and C ABI without a GPU: what reaches the library, and what is refused before it."""
import ctypes
import math

import pytest
import torch

import test_block_abi as abi
import test_window_calls as calls
from paper_2505_00315_gb300 import _binding as B
from paper_2505_00315_gb300 import _block as K
from paper_2505_00315_gb300 import _window as W


class Library(calls.Library):
    """Keeps the struct of each call, and its dropout."""

    def __getattr__(self, name):
        call = super().__getattr__(name)

        def with_dropout(ref, *args):
            rc = call(ref, *args)
            if not name.endswith("_bytes"):
                self.seen[-1] = (*self.seen[-1][:2], getattr(ref._obj, "dropout", None))
            return rc
        return with_dropout


def test_stats_is_a_truth_value():
    for bad in (2, -1):
        s = abi.logprob(stats=bad)
        assert abi.lp_fwd(s) == abi.INV and abi.lp_bwd(s) == abi.INV
        assert B.load().mosa_token_logprobs_workspace_bytes(ctypes.byref(s)) == 0
    p = [abi.FAKE] * 7
    p[4] = abi.OFF                  # lse, or stats
    assert abi.lp_fwd(abi.logprob(stats=1), p) == abi.INV


def test_stats_takes_no_other_place():
    """The struct is as long as before: the new field lies where alignment left room."""
    assert ctypes.sizeof(K.MosaLogprobShape) == 7 * 4 + 4 + 6 * 8
    assert K.MosaLogprobShape.z.offset == 32


class OnGpu(torch.Tensor):
    """A tensor of the host that passes for one of the first GPU."""
    is_cuda = True

    def get_device(self):
        return 0


@pytest.fixture
def lib(monkeypatch):
    L, plans = Library(), {}
    monkeypatch.setattr(B, "load", lambda: L)
    monkeypatch.setattr(B, "_lib", L)
    monkeypatch.setattr(W, "_plans", plans)
    monkeypatch.setattr(K, "_plans", plans)
    monkeypatch.setattr(K, "_structs", 0, raising=False)
    B._torch()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    L.plans = 0
    for name in ("_residual_plan", "_dropout_plan", "_logprob_plan"):
        def counted(*args, _plan=getattr(K, name), **kw):
            L.plans += 1
            return _plan(*args, **kw)
        monkeypatch.setattr(K, name, counted)
    return L


def t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


X, STATS, ROW = t(2, 8, 64), t(2, 2, 8), t(2, 8)
SPACE, RNG, GAMMA = t(256, dtype=torch.uint8), t(2, dtype=torch.int64), t(64)
OUT = {"x": X, "h": X, "stats": STATS, "dx": X, "dy": X, "dgamma_post": GAMMA, "dgamma_pre": GAMMA, "y": X, "dlogits": X}
LP = {"entropy": ROW, "lse": ROW}


def step(**kw):
    return K.mosa_residual_forward(X, X, rng=RNG, out=OUT, **kw)


def step_back(**kw):
    return K.mosa_residual_backward(X, X, STATS, X, X, rng=RNG, workspace=SPACE, out=OUT, **kw)


def drop(dropout=0.5, site=0):
    return K.mosa_dropout(X, dropout, RNG, site=site, out=OUT)


def logp(scale=1.0):
    return K.mosa_token_logprobs(X, scale=scale, workspace=SPACE, out=LP)


def logp_back(scale=1.0):
    return K.mosa_token_logprobs_backward(X, None, ROW, dlse=ROW, scale=scale, out=OUT)


def test_layers_that_differ_in_numbers_share_plans(lib):
    """Two training steps of 200 layers with two residual steps each: a plan for each call's shapes, and the window
    heads' plan stays."""
    q, k, o, lse = t(2, 8, 4, 64), t(2, 8, 2, 64), t(2, 8, 4, 64), t(2, 4, 8)
    W.mosa_window_forward(q, k, k, 4, 1, workspace=SPACE, out={"O": o, "lse": lse})
    window = list(W._plans)
    for _ in range(2):
        for i in range(400):
            numbers = dict(scale=1.0 / (i + 1), eps=1e-6 * (1 + i % 2), dropout=0.1 + 0.001 * (i % 3), site=i)
            for call in (step, step_back):
                call(**numbers)
                assert all(math.isclose(lib.last(n), v, rel_tol=1e-6) for n, v in numbers.items() if n != "dropout")
                assert lib.seen[-1][2] == numbers["dropout"]
            drop(numbers["dropout"], i), logp(numbers["scale"]), logp_back(numbers["scale"])
    assert lib.plans == 5 and len(W._plans) == 6 and window[0] in W._plans


def test_numbers_without_end_do_not_fill_memory(lib):
    for i in range(20000):
        drop(site=i)
        assert lib.last("site") == i
    assert lib.plans == 1 and sum(len(p[0]) for p in K._plans.values()) <= 8192


@pytest.mark.parametrize("call,name", [(f, n) for f in (step, step_back) for n in ("scale", "eps", "dropout")]
                         + [(drop, "dropout"), (logp, "scale"), (logp_back, "scale")],
                         ids=lambda x: getattr(x, "__name__", x))
def test_a_number_that_changes_in_place_counts_at_every_call(call, name, lib):
    x = torch.tensor(0.5)
    for value in (0.5, 0.25):
        x.fill_(value)
        call(**{name: x})
        assert (lib.seen[-1][2] if name == "dropout" else lib.last(name)) == value
    call(**{name: 1})
    assert (lib.seen[-1][2] if name == "dropout" else lib.last(name)) == 1.0


def test_numbers_are_refused_after_others_were_taken(lib):
    step(site=1, dropout=0.5), drop(site=1)
    for call in (step, step_back, drop):
        with pytest.raises(ValueError, match="32 bits"):
            call(site=2**31)
        with pytest.raises(TypeError):
            call(site=1.0)
    K.mosa_residual_forward(X, X, out=OUT)
    with pytest.raises(ValueError, match="rng"):
        K.mosa_residual_forward(X, X, out=OUT, dropout=0.5)
    K.mosa_dropout(X, 0.0, None, out=OUT)
    with pytest.raises(ValueError, match="rng"):
        K.mosa_dropout(X, 0.5, None, out=OUT)
