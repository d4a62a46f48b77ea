"""Window heads on NaN and infinities: where they reach, and where not."""
import math

import pytest
import torch

import paper_2505_00315_gb300 as mosa
from test_gpu_window import inputs, norm_inputs, run

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


KERNELS = [("bf16", "0"), ("bf16", "1"), ("f32", "0")]   # tensor cores, CUDA cores with either storage


@pytest.mark.parametrize("dtype,force", KERNELS)
@pytest.mark.parametrize("hp", [64, 128])
def test_a_visible_nan_counts_where_its_weight_underflows(hp, dtype, force, monkeypatch):
    """A token with a score so low that its weight is 0 (2^-900), and a NaN in its value: the queries
    that see it have NaN there, and it has NaN gradients, in tiles seen whole or in part."""
    monkeypatch.setenv("MOSA_FORCE_SIMT", force)
    T, j, w = 400, 150, 130
    q, k, v, dO = inputs(1, T, T, 2, 1, hp, dtype, seed=41, layout="plain")
    q.fill_(2.0)
    k[0, j] = -640.0 * hp ** -0.5 / 2
    clean = run(q, k, v, dO, w, 0)
    assert torch.isfinite(clean["O"]).all()
    v[0, j, 0, 3] = math.nan
    got = run(q, k, v, dO, w, 0)
    sees = torch.zeros(T, dtype=torch.bool, device="cuda")
    sees[j:j + w] = True
    assert torch.isnan(got["O"][0, sees][..., 3]).all()
    assert not torch.isfinite(got["dq"][0, sees].float()).any()
    assert not torch.isfinite(got["dk"][0, j].float()).any()
    for n in ("O", "dq"):
        assert torch.equal(got[n][0, ~sees], clean[n][0, ~sees]), n


@pytest.mark.parametrize("dtype,force", KERNELS)
@pytest.mark.parametrize("T,window", [(1, 0), (3, 1), (200, 1)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["q", "k", "v", "dO"])
def test_a_query_that_sees_one_token_passes_a_nan_on(where, bad, T, window, dtype, force, monkeypatch):
    """Its scores have no gradient (P = 1), unless what it meets is no number."""
    monkeypatch.setenv("MOSA_FORCE_SIMT", force)
    q, k, v, dO = inputs(1, T, T, 1, 1, 64, dtype, seed=42, layout="plain")
    clean = run(q, k, v, dO, window, 0)
    for n in ("dq", "dk"):
        assert (clean[n] == 0).all()
    j = T // 2
    {"q": q, "k": k, "v": v, "dO": dO}[where][0, j] = bad
    got = run(q, k, v, dO, window, 0)
    reached = {"q": ("O", "dq", "dk", "dv"), "k": ("O", "dq", "dk", "dv"), "v": ("O", "dq", "dk"),
               "dO": ("dq", "dk", "dv")}[where]
    for n in reached:
        assert not torch.isfinite(got[n][0, j].float()).any(), n
    keep = torch.arange(T, device="cuda") != j
    for n in ("O", "dq", "dk", "dv"):
        assert torch.equal(got[n][0, keep], clean[n][0, keep]), n


@pytest.mark.parametrize("dtype,force", KERNELS)
def test_scores_of_minus_infinity_are_no_empty_row(dtype, force, monkeypatch):
    """A query all of whose scores are -inf sees tokens: O is NaN (0 / 0), not the zeros of a query
    past its sequence's end; beside others such a token has no weight."""
    monkeypatch.setenv("MOSA_FORCE_SIMT", force)
    q, k, v, dO = inputs(1, 200, 200, 2, 1, 64, dtype, seed=43, layout="plain")
    q[0, 90].fill_(-math.inf)
    k.abs_().add_(0.1)
    lens = torch.tensor([150], device="cuda", dtype=torch.int32)
    O, lse, _ = mosa.mosa_window_forward(q, k, v, 40, 2, lens=lens)
    assert torch.isnan(O[0, 90].float()).all() and not torch.isfinite(lse[0, :, 90]).any()
    keep = torch.arange(200, device="cuda") != 90
    assert torch.isfinite(O[0, keep].float()).all()
    assert (O[0, 150:] == 0).all() and (lse[0, :, 150:] == -math.inf).all()
