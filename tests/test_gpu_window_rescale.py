"""The tensor-core forward's running maximum where it has to move: scores that rise, fall or jump from block
to block by more than the 2^8 that pass without rescaling O and its sum.

O's tolerance: its own rounding and P's, 2^-9 of each term, 8e-3 with room as for other bf16 outputs; a
rescaling missed or done twice is off by 2^8 and more.  lse is the maximum and a logarithm in fp32 of
scores up to 2^8: 2^-24 * 2^8 / (a mean lse of 10 and more): 2e-6 relative."""
import pytest
import torch

import _window_ref as ref
import paper_2505_00315_gb300 as mosa
from test_gpu_window import inputs, rel

pytestmark = pytest.mark.gpu


def moving(kind, T):
    """The scores' mean (in units of the natural logarithm) of each key."""
    t = torch.arange(T, device="cuda", dtype=torch.float32)
    if kind == "rising":          # 13 a block of 128: each block's maximum exceeds the last by 2^19
        return t * 0.1
    if kind == "falling":
        return (T - t) * 0.1
    if kind == "steps":           # jumps at every third block, some within a block's first keys
        return (t // 389) * 40.0
    return torch.where((t // 64) % 3 == 1, 30.0, -30.0) + t * 0.02   # "waves"


@pytest.mark.parametrize("hp", [32, 64, 128])
@pytest.mark.parametrize("kind", ["rising", "falling", "steps", "waves"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (500, 3), (100, 0)])
def test_scores_that_move_from_block_to_block(window, sinks, kind, hp):
    T = 1200
    q, k, v, _ = inputs(2, T, T, 4, 2, hp, "bf16", seed=61, layout="plain")
    # a dimension of its own carries the mean; every fourth query sees little of it, so that rows of a warp
    # rescale at different blocks
    q[..., 0], k[..., 0] = 1.0, (moving(kind, T) * hp ** 0.5)[None, :, None].to(k.dtype)
    q[:, ::4, :, 0] = 0.03
    want = ref.attention(q, k, v, window, sinks)
    O, lse, _ = mosa.mosa_window_forward(q, k, v, window, sinks)
    assert rel(O, want["O"]) < 8e-3
    assert rel(lse, want["lse"]) < 2e-6
