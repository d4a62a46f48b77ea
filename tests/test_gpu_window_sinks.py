"""Gradients of sink rows, whose far queries go to CTAs of their own or to the tile's, by how many sink tiles
there are."""
import pytest
import torch

import _window_ref as ref
from test_gpu_window import DT, check, inputs, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,force", [("bf16", "0"), ("bf16", "1"), ("f32", "0")])
@pytest.mark.parametrize("B,T,H,Hkv,hp,window,sinks", [
    (1, 1500, 2, 1, 64, 100, 512), (1, 1500, 2, 1, 64, 100, 513), (1, 1300, 1, 1, 128, 1, 1000),
    (8, 300, 32, 32, 32, 40, 3),     # as many sink tiles as fill the GPU
    (40, 300, 4, 4, 64, 20, 140),
])
def test_many_sinks_and_many_sink_tiles(B, T, H, Hkv, hp, window, sinks, dtype, force, monkeypatch):
    monkeypatch.setenv("MOSA_FORCE_SIMT", force)
    q, k, v, dO = inputs(B, T, T, H, Hkv, hp, dtype, seed=sinks)
    lens = torch.randint(T // 2, T + 1, (B,), device="cuda", dtype=torch.int32,
                         generator=torch.Generator("cuda").manual_seed(1))
    got = run(q, k, v, dO, window, sinks, lens)
    check(got, ref.attention(q, k, v, window, sinks, lens, dO=dO), DT[dtype])
    again = run(q, k, v, dO, window, sinks, lens)
    for n in got:
        assert torch.equal(got[n], again[n]), n
