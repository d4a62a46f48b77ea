"""The block operators where inputs, gradients or places are not the usual ones, against their definitions in 64 bits."""
import pytest
import torch

import paper_2505_00315_gb300 as mosa
from _block_ref import keep_mask, logprobs, near, residual
from test_gpu_block import BF, F32, INF, NAN, check_logprobs, gen, inputs, logits_of, state, targets_of

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------ residual step

# Kernels of 8, 16 and 32 columns a thread, in both types, and those of rows that are not whole pieces.
WIDTHS = [(BF, BF, 30, 320), (BF, F32, 30, 1500), (F32, F32, 30, 768), (BF, F32, 4000, 1024), (F32, F32, 30, 6000),
          (F32, F32, 30, 8192), (BF, BF, 30, 1001)]


@pytest.mark.parametrize("dt,xt,T,d", WIDTHS)
@pytest.mark.parametrize("pre", [True, False])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate", ["none", "token"])
def test_without_a_gradient_of_h_dx_is_dx_out_whatever_the_inputs_hold(dt, xt, T, d, pre, post, gate):
    s, dx_out, _ = inputs(2, T, d, dt, xt=xt, gate=gate, seed=31)
    kw = dict(post_norm=post, pre_norm=pre, scale=0.5)

    def backward(v):
        stats = mosa.mosa_residual_forward(**v, **kw)[2]
        return mosa.mosa_residual_backward(stats=stats, dx_out=dx_out, dh=None, **v, **kw)[0]

    clean = backward(s)
    y, x = s["y"].clone(), s["x"].clone()
    y[0, 3], y[1, 4, 5], y[1, 29, d - 1] = NAN, INF, -INF
    x[0, 7], x[1, 9, 2] = NAN, INF
    got = backward({**s, "x": x, "y": y, "gamma_pre": torch.full_like(s["gamma_pre"], NAN)})
    assert torch.equal(got["dx"], dx_out) and torch.equal(clean["dx"], dx_out)
    others = torch.ones(2, T, dtype=torch.bool, device="cuda")
    others[0, 3] = others[1, 4] = others[1, 29] = False
    for n in ("dy", "dgate"):
        assert n not in got or torch.equal(got[n][others], clean[n][others]), n
    if pre:
        assert not got["dgamma_pre"].any()


@pytest.mark.parametrize("dt,xt,T,d", WIDTHS)
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
def test_without_a_norm_dy_does_not_see_y(dt, xt, T, d, gate):
    """dy = scale g dx_out, also where y is infinite or no number."""
    s, dx_out, _ = inputs(2, T, d, dt, xt=xt, gate=gate, seed=32)
    kw = dict(post_norm=False, pre_norm=False, scale=0.5)

    def backward(v):
        stats = mosa.mosa_residual_forward(**v, **kw)[2]
        return mosa.mosa_residual_backward(stats=stats, dx_out=dx_out, dh=None, **v, **kw)[0]

    clean = backward(s)
    y = s["y"].clone()
    y[0, 3], y[1, 4, 5], y[1, 29, d - 1] = NAN, INF, -INF
    got = backward({**s, "y": y})
    assert torch.equal(got["dy"], clean["dy"])
    g = 1.0 if gate == "none" else s["gate"].double()
    want = 0.5 * g * dx_out.double()
    near("dy", got["dy"], want, 2.0 ** -22 * want.abs())   # three products


@pytest.mark.parametrize("dt,xt,T,d", WIDTHS)
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
def test_a_dropped_infinity_of_a_normed_row_does_not_count(dt, xt, T, d, gate):
    """1 / sqrt(mean(y^2)) is 0 there, and the row that of a block that gave zeros, but for dy, which is 0 with r_y."""
    p, rng = 0.5, state(9)
    s, dx_out, dh = inputs(2, T, d, dt, xt=xt, gate=gate, seed=33)
    keep = keep_mask(rng, 0, s["x"].shape, p, "cuda")
    y, zero = s["y"].clone(), s["y"].clone()
    rows = ((0, 3), (1, 4), (1, 29))
    for i, (b, t) in enumerate(rows):
        gone = (~keep[b, t]).nonzero()[:, 0]
        y[b, t, gone[:1 + 3 * i]] = -INF if i == 1 else INF
        zero[b, t] = 0
    y[1, 29, (~keep[1, 29]).nonzero()[-1, 0]] = -INF
    s["y"] = y
    kw = dict(dropout=p, rng=rng, scale=0.5)
    x, h, stats = mosa.mosa_residual_forward(**s, **kw)
    g, _ = mosa.mosa_residual_backward(stats=stats, dx_out=dx_out, dh=dh, **s, **kw)
    want = residual(**{**s, "y": zero}, dx_out=dx_out, dh=dh, backward=True, **kw)
    for b, t in rows:
        want["dy"][0][b, t] = want["dy"][1][b, t] = 0
    for n, t in {"x": x, "h": h, **g}.items():
        near(n, t, *want[n])


@pytest.mark.parametrize("dt,xt,T,d", WIDTHS)
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
def test_a_block_that_is_dropped_whole_does_not_count(dt, xt, T, d, gate):
    """Rows of NaN, of infinities, and of zeros whose norm has no eps: gradients know nothing of them."""
    s, dx_out, dh = inputs(2, T, d, dt, xt=xt, gate=gate, seed=44)
    kw = dict(dropout=1.0, rng=state(10), scale=0.5, eps=0.0)
    want = residual(**s, dx_out=dx_out, dh=dh, backward=True, **kw)
    s["y"][0, ::3], s["y"][0, 1::3], s["y"][1, ::2, 0] = 0.0, NAN, INF
    x, h, stats = mosa.mosa_residual_forward(**s, **kw)
    g, _ = mosa.mosa_residual_backward(stats=stats, dx_out=dx_out, dh=dh, **s, **kw)
    for n, t in {"x": x, "h": h, **g}.items():
        near(n, t, *want[n])


@pytest.mark.parametrize("dt,xt,T,d", WIDTHS)
@pytest.mark.parametrize("gate", ["channel", "token"])
def test_gradient_of_a_saturated_gate(dt, xt, T, d, gate):
    """Through a sigmoid s of gates far from 0, where 1 - s is not what fp32 keeps of s.  The gradient is that of the
    gate s itself times s (1 - s), and its bound that one's, with u = 2^-24: s (1 - s) = e r^2 of e = e^-|x| (off by 1.3 u |x|
    from the exponent, 4 u from the power), 1 + e (u), r (2 u) twice and two products is off by (4 + 2 (1 + 2) + 2 + 1.3 |x|) u
    = (12 + 1.3 |x|) u relative, a share of (12 + 1.3 |x|) / 256 of the bound's 2^-16."""
    s, dx_out, dh = inputs(2, T, d, dt, xt=xt, gate=gate, seed=35)
    some = torch.tensor([0.0, 1.0, -1.0, 8.0, -8.0, 12.0, -12.0, 16.0, -16.0, 30.0, -30.0, -60.0], device="cuda")
    s["gate"] = some[torch.randint(0, 12, s["gate"].shape, generator=gen(36), device="cuda")].to(dt)
    kw = dict(scale=0.5, dropout=0.1, rng=state())
    x, h, stats = mosa.mosa_residual_forward(**s, sigmoid=True, **kw)
    g, _ = mosa.mosa_residual_backward(stats=stats, dx_out=dx_out, dh=dh, **s, sigmoid=True, **kw)
    z = s["gate"].double()
    want = residual(**{**s, "gate": torch.sigmoid(z)}, dx_out=dx_out, dh=dh, backward=True, **kw)
    slope = torch.sigmoid(z) * torch.sigmoid(-z)
    ref, bound = want["dgate"]
    want["dgate"] = ref * slope, bound * slope * (1 + (12 + 1.3 * z.abs()) / 256)
    for n, t in {"x": x, "h": h, **g}.items():
        near(n, t, *want[n])


@pytest.mark.parametrize("dt,xt,T,d", [*WIDTHS, (BF, F32, 40, 5000), (F32, F32, 3300, 1024), (BF, F32, 3300, 2048)])
@pytest.mark.parametrize("gate", ["channel", "token"])
def test_cut_sequences_without_a_gradient_of_h(dt, xt, T, d, gate):
    """Tokens 2 to T + 1 of T + 5, in and out, and what lies around them as it was; without dx_out too."""
    B = 3
    s, dx_out, _ = inputs(B, T + 5, d, dt, xt, xt, gate=gate, seed=39)
    cut = lambda t: t[:, 2:2 + T]   # noqa: E731
    s = {n: cut(v) if v is not None and v.dim() == 3 else v for n, v in s.items()}
    kw = dict(scale=0.5, dropout=0.2, rng=state(), sigmoid=gate == "token")
    types = {"dx": xt, "dy": dt, **({"dgate": dt} if gate == "token" else {})}
    for up in (cut(dx_out), None):
        room = {n: torch.full((B, T + 5, d), 7.0, device="cuda", dtype=v) for n, v in types.items()}
        stats = mosa.mosa_residual_forward(**s, **kw)[2]
        g, _ = mosa.mosa_residual_backward(stats=stats, dx_out=up, dh=None, out={n: cut(v) for n, v in room.items()}, **s, **kw)
        want = residual(**s, dx_out=up, dh=None, backward=True, **kw)
        for n in g:
            near(n, g[n], *want[n])
        for n, v in room.items():
            assert (v[:, :2] == 7).all() and (v[:, 2 + T:] == 7).all(), n


@pytest.mark.parametrize("B,T", [(1, 3), (3, 1), (2, 2)])
@pytest.mark.parametrize("with_dh", [True, False])
def test_backward_of_rows_past_32_bits(B, T, with_dh):
    """A stream and its gradient whose rows, or sequences, lie further than 2^32 bytes apart; dx takes dx_out's place."""
    d, far = 1024, 2**31 + 512
    room = torch.zeros(2 * far + 8192, device="cuda", dtype=BF)
    s, dx_out, dh = inputs(B, T, d, gate="channel", seed=40)
    stride = (far, 4096, 1) if T == 2 else (far, far, 1)
    x, up = (room.as_strided((B, T, d), stride, i * 2048) for i in range(2))
    x.copy_(s["x"]), up.copy_(dx_out)
    dh = dh if with_dh else None
    kw = dict(dropout=0.1, rng=state(), scale=0.5)
    want = residual(**s, dx_out=dx_out, dh=dh, backward=True, **kw)
    stats = mosa.mosa_residual_forward(**{**s, "x": x}, **kw)[2]
    g, _ = mosa.mosa_residual_backward(stats=stats, dx_out=up, dh=dh, out={"dx": up}, **{**s, "x": x}, **kw)
    assert g["dx"] is up and torch.equal(x, s["x"])
    for n in g:
        near(n, g[n], *want[n])


# -------------------------------------------------------- log probabilities

@pytest.mark.parametrize("V", [40, 3001, 40000])
@pytest.mark.parametrize("dt", [BF, F32])
def test_rows_that_are_no_numbers_are_so_where_entries_are_ruled_out(V, dt):
    """A NaN or an entry above 2^90 beside ruled-out ones, which are targets and alternatives."""
    z = logits_of(1, 6, V, dt, seed=34)
    z[0, :, V // 2:] = -INF
    z[0, 0], z[0, 0, 1] = -INF, NAN
    z[0, 1, 3] = INF
    z[0, 2], z[0, 2, V - 1] = torch.finfo(dt).min, 1e30
    z[0, 3, 0] = NAN
    t = torch.tensor([[V - 1, V - 1, 0, V // 2, V - 1, 2]], device="cuda")
    r = check_logprobs(z, t, 5)
    assert torch.isnan(r["dlogits"][0, :4]).all() and torch.isfinite(r["dlogits"][0, 4:]).all()
    idx = torch.tensor([[[V - 1, 7, V - 2]]], dtype=torch.int32, device="cuda").expand(1, 6, 3).contiguous()
    up = torch.ones(1, 6, 3, device="cuda")
    dz = mosa.mosa_token_logprobs_backward(z, t, r["lse"], top=idx, dtop_logp=up)
    assert torch.isnan(dz[0, :4]).all() and torch.isfinite(dz[0, 4:]).all()


def gradients(z, t, top, scale, seed=0, stats=True):
    """The forward's results, upstream gradients of all of them, and the logits' gradient."""
    B, T, V = z.shape
    r, _ = mosa.mosa_token_logprobs(z, t, top=top, scale=scale, stats=stats)
    up = {n: torch.randn((B, T) + (top,) * (n == "dtop_logp"), generator=gen(seed + i), device="cuda")
          for i, n in enumerate(("dlogp", "dentropy", "dlse", "dtop_logp")) if top or n != "dtop_logp"}
    dz = mosa.mosa_token_logprobs_backward(z, t, r["stats" if stats else "lse"], r["entropy"], top=r.get("top"), scale=scale,
                                           **up)
    return r, up, dz


@pytest.mark.parametrize("B,T,V,top", [(2, 13, 2000, 3), (1, 9, 1001, 0), (1, 2, 131072, 20), (1, 5, 40001, 4),
                                       (1, 3000, 1500, 2)])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("scale", [1.0, 0.8])
@pytest.mark.parametrize("far", [0.0, 30.0, -1000.0, 1e5])
def test_gradient_of_logits_far_from_zero(far, scale, dt, B, T, V, top):
    """From stats, within a bound that knows how far a logit lies from its row's largest, not from 0.  With u = 2^-24 and
    k = (a_max - a_j): the exponent c (z - m) is off by 3 u of itself (difference, c, product) and its power by 4 u, so a term
    by (3 k + 4) u; a sum adds up V / 64 of them one after another at most, and 16 in a tree; its inverse and two products are
    6 u more: e_j = (V / 64 + 32 + 3 k) u relative for p_j, beside the terms' own errors in the sum, on average
    (3 E[k] + 4) u with E[k] <= H.  ln s and t / s, of which H and log p + H are made, carry the same relative errors: of
    quantities of at most 2 + H and 2 + H + k."""
    u = 2.0 ** -24
    z = (logits_of(B, T, V, F32, seed=37) + far).to(dt)
    t = targets_of(B, T, V)
    r, up, dz = gradients(z, t, top, scale, seed=60)
    a = z.double() * float(torch.tensor(scale))
    logp = torch.log_softmax(a, -1)
    p = logp.exp()
    H = -(p * logp).sum(-1, keepdim=True)
    k = a.amax(-1, keepdim=True) - a
    row = (V / 64 + 36 + 3 * H) * u
    e = row + (V / 64 + 32 + 3 * k) * u
    gl = torch.where(t < 0, 0.0, up["dlogp"].double())[..., None]
    own = torch.zeros_like(p).scatter_add_(-1, t.clamp(min=0)[..., None], gl)
    G, Ga = gl, gl.abs()
    if top:
        g = up["dtop_logp"].double()
        own.scatter_add_(-1, r["top"].long(), g)
        G, Ga = G + g.sum(-1, keepdim=True), Ga + g.abs().sum(-1, keepdim=True)
    dH, dL = up["dentropy"].double()[..., None], up["dlse"].double()[..., None]
    s = float(torch.tensor(scale))
    want = s * (own + p * (dL - G - dH * (logp + H)))
    # (the factor of p is a sum of some terms, each off by some u: 24 for up to 20 alternatives and the rest)
    size = p * (dL.abs() + Ga + dH.abs() * (logp.abs() + H))
    bound = s * (own.abs() * 24 * u + (e + 24 * u) * size + p * dH.abs() * (e + row) * (4 + 2 * H + k))
    near("dlogits", dz, want, bound + 2.0 ** -126 * s * (dL.abs() + Ga + dH.abs() * 210 + 1))
    if dt is F32:   # p of a row sums to 1
        one = torch.ones(B, T, device="cuda")
        p1 = mosa.mosa_token_logprobs_backward(z, None, r["stats"], dlse=one, scale=scale).double() / s
        assert ((p1.sum(-1, keepdim=True) - 1).abs() <= (p * e).sum(-1, keepdim=True) + 2 * u).all()


@pytest.mark.parametrize("dt", [BF, F32])
def test_stats_are_for_all_rows(dt):
    """Masked rows, rows that are no numbers, large and few entries: results as without stats, and gradients within the
    bounds of those."""
    V = 3001
    z = logits_of(2, 8, V, dt, seed=38)
    low = torch.finfo(dt).min
    z[0, 0], z[0, 1], z[0, 2, 1:], z[0, 3, :-1], z[0, 4, ::2] = -INF, low, -INF, low, -INF
    z[0, 5, 5], z[0, 6, 7], z[1, 0, 3], z[1, 1] = NAN, INF, 1e30, NAN
    z[1, 2], z[1, 3] = z[1, 2] * 1e20, z[1, 3] - 1e20
    z[1, 4, :-3] = -INF
    t = targets_of(2, 8, V)
    t[1, 5], t[1, 6] = V, 2**40
    for top in (0, 7):
        for scale in (1.0, 0.5, 2.0 ** -20):
            plain = mosa.mosa_token_logprobs(z, t, top=top, scale=scale)[0]
            r, up, dz = gradients(z, t, top, scale, seed=70)
            assert set(r) == set(plain) | {"stats"} and r["lse"].data_ptr() == r["stats"].data_ptr()
            for n in plain:
                assert torch.equal(torch.nan_to_num(r[n].double(), 7e77), torch.nan_to_num(plain[n].double(), 7e77)), n
            up["dtop"] = up.pop("dtop_logp", None)
            near("dlogits", dz, *logprobs(z, t, top, scale, **up)["dlogits"])
            again = mosa.mosa_token_logprobs(z, t, top=top, scale=scale, stats=True, out=r)[0]
            assert all(again[n] is r[n] for n in r)
    with pytest.raises(ValueError, match="planes"):
        mosa.mosa_token_logprobs(z, t, stats=True, out={"lse": plain["lse"]})
    with pytest.raises(ValueError, match="stats"):
        mosa.mosa_token_logprobs_backward(z, t, r["stats"][:2].contiguous(), dlse=plain["lse"])


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("stats", [False, True])
def test_gradient_in_place_where_warps_share_a_row(dt, stats):
    """Each warp reads the target and the alternatives in its own columns before it writes any: rows of 40001 entries, with
    alternatives on both sides of every step's border (1024 columns of bf16, 512 of fp32) and the target at it.  Bit for bit
    what the call gives elsewhere, and that within the bounds."""
    V, K = 40001, 1024 if dt is BF else 512
    T = V // K
    z = logits_of(1, T, V, dt, seed=41)
    border = torch.arange(1, T + 1, device="cuda") * K
    t = border[None].contiguous()
    idx = (border[:, None] + torch.arange(-16, 16, device="cuda")).clamp(max=V - 1).int()[None].contiguous()
    r, _ = mosa.mosa_token_logprobs(z, t, scale=0.7, stats=stats)
    up, up_top = torch.randn(1, T, generator=gen(42), device="cuda"), torch.randn(1, T, 32, generator=gen(43), device="cuda")
    kw = dict(entropy=r["entropy"], dlogp=up, dentropy=up, top=idx, dtop_logp=up_top, scale=0.7)
    lse = r["stats" if stats else "lse"]
    want = mosa.mosa_token_logprobs_backward(z, t, lse, **kw)
    p = torch.softmax(z.double() * float(torch.tensor(0.7)), -1)
    own = torch.zeros_like(p).scatter_add_(-1, t[..., None], up.double()[..., None])
    own.scatter_add_(-1, idx.long(), up_top.double())
    G, H = own.sum(-1, keepdim=True), -(p * p.log()).sum(-1, keepdim=True)
    dz = 0.7 * (own - p * (G + up.double()[..., None] * (p.log() + H)))
    # (logits below 20, so that lse's rounding is 2^-19; sums of V / 64 = 626 terms 2^-14; some 40 additions of upstream values)
    size = own.abs() + p * (own.abs().sum(-1, keepdim=True) + up.abs().double()[..., None] * (p.log().abs() + H))
    near("dlogits", want, dz, 2.0 ** -13 * size)
    got = mosa.mosa_token_logprobs_backward(z, t, lse, out={"dlogits": z}, **kw)
    assert got is z and torch.equal(got, want)
