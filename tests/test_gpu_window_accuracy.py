"""Errors of bf16 window attention against 64 bits, next to those of a form that rounds nothing but what it
stores: the ratio of the two.

Bounds, from the roundings beside the stored one, each about as large and independent of it:
  few terms   (a query sees at most 128 tokens) and CUDA cores: P and dS lose 2^-17: 1.0; 1.1 with room
              for chance.
  many terms  O and dv: P's, sqrt(2) = 1.41: 1.5.  dk: dS's, and P's in the forward through D, sqrt(3) = 1.73:
              1.75.  dq: P's in the forward through D only, a part of a rounding: 1.3 (with dS in one
              part it would be 1.41 and more)."""
import pytest
import torch

import _window_ref as ref
from test_gpu_window import inputs, run

pytestmark = pytest.mark.gpu

FEW = {n: 1.1 for n in ("O", "dq", "dk", "dv")}
MANY = {"O": 1.5, "dq": 1.3, "dk": 1.75, "dv": 1.5}


def draw(kind, *shape, sinks=0, seed=0):
    q, k, v, dO = inputs(*shape, "bf16", seed=seed, layout="plain")
    if kind == "peaked":       # scores of standard deviation 3
        q, k = (x * 1.7 for x in (q, k))
    elif kind == "sinks":      # most weight on the first tokens
        u = torch.randn(shape[5], generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
        q, k = q + (0.7 * u).to(q.dtype), k.clone()
        k[:, :max(1, sinks)] += (0.7 * u).to(k.dtype)
    return q, k, v, dO


def ratios(q, k, v, dO, window, sinks):
    got, want = run(q, k, v, dO, window, sinks), ref.attention(q, k, v, window, sinks, dO=dO)
    out = {}
    for n in FEW:
        stored = (want[n].bfloat16().double() - want[n]).norm()
        out[n] = float((got[n].double() - want[n]).norm() / stored)
    return out


def check(got, bounds):
    assert all(got[n] < bounds[n] for n in bounds), {n: round(x, 3) for n, x in got.items()}


@pytest.mark.parametrize("kind", ["plain", "peaked", "sinks"])
@pytest.mark.parametrize("hp", [32, 64, 128])
@pytest.mark.parametrize("B,T,H,Hkv,window,sinks", [
    (16, 2, 8, 8, 0, 0), (16, 17, 8, 4, 5, 1), (4, 91, 4, 4, 0, 0), (4, 128, 4, 1, 64, 4),   # short texts
    (2, 129, 4, 4, 128, 0), (2, 600, 4, 2, 2, 1), (2, 600, 4, 4, 16, 4), (2, 1000, 4, 1, 124, 4),   # short windows
    (2, 700, 2, 2, 1, 127),
])
def test_few_terms_lose_nothing_but_what_is_stored(B, T, H, Hkv, window, sinks, hp, kind):
    check(ratios(*draw(kind, B, T, T, H, Hkv, hp, sinks=sinks, seed=T), window, sinks), FEW)


@pytest.mark.parametrize("hp", [64, 128])
@pytest.mark.parametrize("T,H,Hkv,window,sinks", [(300, 4, 4, 0, 0), (900, 4, 2, 256, 4), (900, 4, 4, 128, 1)])
def test_many_terms_lose_one_rounding_of_weights(T, H, Hkv, window, sinks, hp):
    check(ratios(*draw("plain", 2, T, T, H, Hkv, hp, seed=T), window, sinks), MANY)


@pytest.mark.parametrize("kind", ["plain", "peaked", "sinks"])
def test_cuda_cores_lose_nothing_but_what_is_stored(kind, monkeypatch):
    monkeypatch.setenv("MOSA_FORCE_SIMT", "1")
    check(ratios(*draw(kind, 2, 400, 400, 4, 2, 64, sinks=4, seed=9), 200, 4), FEW)
