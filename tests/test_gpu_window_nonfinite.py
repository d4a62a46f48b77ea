"""Window heads on NaN and infinities: where they reach, and where not."""
import math

import pytest
import torch

import paper_2505_00315_gb300 as mosa
from test_gpu_window import norm_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,layout", [("bf16", "packed"), ("bf16", "unaligned"), ("f32", "packed")])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("where", ["k", "dyk", "q", "dyq"])
def test_the_norms_gradients_of_queries_and_keys_stay_apart(where, bad, dtype, layout):
    """A bad value of a key is in no sum over queries, nor the other way round, and other rows'
    gradients are as without it."""
    for B, T in ((1, 3), (2, 300)):
        q, k, gq, gk, dyq, dyk, pos = norm_inputs(B, T, 4, 2, 64, dtype, layout, seed=T)
        x = {"q": q, "k": k, "dyq": dyq, "dyk": dyk}
        clean, _ = mosa.mosa_qk_norm_rope_backward(q, k, gq, gk, dyq, dyk, positions=pos)
        x[where][B - 1, T // 2, 1, 5] = bad
        got, _ = mosa.mosa_qk_norm_rope_backward(q, k, gq, gk, dyq, dyk, positions=pos)
        mine, other = ("q", "k") if "q" in where else ("k", "q")
        for n in ("d", "dgamma_"):
            assert torch.equal(got[n + other], clean[n + other]), n + other
        assert not torch.isfinite(got["dgamma_" + mine]).all()
        keep = torch.ones(got["d" + mine].shape[:3], dtype=torch.bool, device="cuda")
        keep[B - 1, T // 2, 1] = False
        assert torch.equal(got["d" + mine][keep], clean["d" + mine][keep])
