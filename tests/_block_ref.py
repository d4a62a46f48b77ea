"""The block operators in 64 bits, from their definitions, each with a bound on what 32-bit arithmetic
may be off by.

Bounds.  u = 2^-24 is half a step of fp32.  A norm's sum of d <= 8192 squares is added up on one
thread over at most 16 values and then in a tree of at most 9 levels, so that r = 1/sqrt(..) is off by at most
(16 + 9 + 6) u < 2^-19 relative; what is computed from r in a few more steps is off by less than
2^-18 of the sum of its terms' magnitudes, and a value that has gone through two means by less
than 2^-16.  Magnitudes are carried along (names in _abs): x' = x + scale u has |x| + |scale u|, however much
of it cancels.  A result in bf16 is rounded once more, by at most eps/2 = 2^-8 relative."""
import numpy as np
import torch

F64 = torch.float64


def philox(seed, offset, rows, d):
    """One 32-bit word for each column of each row, as NumPy uint64 [rows, d]."""
    u = np.uint64
    q = (d + 3) // 4
    low, half = u(0xFFFFFFFF), u(32)
    o = offset % 2 ** 64
    x = [np.tile(np.arange(q, dtype=u), (rows, 1)), np.repeat(np.arange(rows, dtype=u)[:, None], q, 1),
         np.full((rows, q), o % 2 ** 32, u), np.full((rows, q), o // 2 ** 32, u)]
    return np.stack(philox_words(x, seed % 2 ** 64), -1).reshape(rows, 4 * q)[:, :d]


def philox_words(x, seed, rounds=7):
    u = np.uint64
    low, half = u(0xFFFFFFFF), u(32)
    for r in range(rounds):
        k0, k1 = u((seed % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32), u((seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32)
        a, b = x[0] * u(0xD2511F53), x[2] * u(0xCD9E8D57)
        x = [(b >> half) ^ x[1] ^ k0, b & low, (a >> half) ^ x[3] ^ k1, a & low]
    return x


def keep_mask(rng, site, shape, p, device):
    """Which values are kept (bool tensor)."""
    seed, offset = (int(v) for v in rng.tolist())
    w = philox(seed, offset + site, int(np.prod(shape[:-1])), shape[-1])
    return torch.from_numpy(w >= np.uint64(round(p * 2 ** 32))).to(device).reshape(shape)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def near(name, got, ref, bound, extra=0.0):
    """|got - ref| <= bound + the rounding to got's type, wherever ref is finite; else the same kind."""
    got64 = got.to(F64)
    assert torch.equal(torch.isnan(got64), torch.isnan(ref)), f"{name}: NaN elsewhere"
    inf = torch.isinf(ref)
    assert torch.equal(got64[inf], ref[inf]), f"{name}: infinities elsewhere"
    ok = torch.isfinite(ref)
    tol = bound + half_step(got.dtype) * (ref.abs() + bound) + extra
    far = (got64 - ref).abs()
    tol = tol.expand_as(far) if torch.is_tensor(tol) else torch.full_like(far, tol)
    bad = ok & ~(far <= tol)
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{name}{list(i)}: {got64[i].item()!r} for {ref[i].item()!r}, off by {far[i].item():.3e}, "
                             f"may be {tol[i].item():.3e}; {int(bad.sum())} of {bad.numel()}")


def residual(x, y, gate=None, gamma_post=None, gamma_pre=None, post_norm=True, pre_norm=True, sigmoid=False,
             scale=1.0, eps=1e-6, dropout=0.0, rng=None, site=0, dx_out=None, dh=None, backward=False):
    """{name: (value, bound)}."""
    scale, eps = float(np.float32(scale)), float(np.float32(eps))   # as the library's fields hold them
    f = lambda t: t.to(F64)   # noqa: E731
    x, y = f(x), f(y)
    d = x.shape[-1]
    one = torch.ones(d, dtype=F64, device=x.device)
    gp = one if gamma_post is None else f(gamma_post)
    gr = one if gamma_pre is None else f(gamma_pre)
    g = one if gate is None else f(gate)
    if sigmoid and gate is not None:
        g = 1 / (1 + torch.exp(-g))
    keep = torch.ones_like(x, dtype=torch.bool)
    if dropout > 0:
        keep = keep_mask(rng, site, x.shape, dropout, x.device)
    unit = torch.where(keep, scale / (1 - dropout) if dropout < 1 else 0.0, 0.0)
    ry = 1 / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) if post_norm else torch.ones_like(y[..., :1])
    yh = y * ry
    n = yh * (gp if post_norm else 1)
    u = torch.where(keep, unit * g * n, 0.0)
    x1, x1_abs = x + u, x.abs() + u.abs()
    out = {"x": (x1, 2 ** -18 * x1_abs)}
    rx = 1 / torch.sqrt((x1 * x1).mean(-1, keepdim=True) + eps)
    # (an error of x' that cancels shows in r_x too: by its share of the row's squares)
    rel = 2 ** -18 * (1 + ((x1_abs * x1.abs()).mean(-1, keepdim=True) * rx * rx))
    if pre_norm:
        out["h"] = (x1 * rx * gr, (gr * rx).abs() * (2 ** -18 * x1_abs + rel * x1.abs()))
    if not backward:
        return out
    xh, xa = x1 * rx, rx * x1_abs
    zero = torch.zeros_like(x)
    do = zero if dx_out is None else f(dx_out)
    dhv = zero if dh is None or not pre_norm else f(dh)
    e = dhv * gr
    mean = lambda t: t.mean(-1, keepdim=True)   # noqa: E731
    t = do + rx * (e - xh * mean(e * xh))
    ta = do.abs() + rx * (e.abs() + xa * mean(e.abs() * xa))
    c = unit * t
    ca = unit.abs() * ta
    yn, ya = torch.where(keep, n, 0.0), torch.where(keep, n.abs(), 0.0)
    gk = torch.where(keep, g.expand_as(x), 0.0)
    w = c * gk * (gp if post_norm else 1)
    wa = ca * (gk * (gp if post_norm else 1)).abs()
    dy, dya = w, wa
    if post_norm:
        dy = ry * (w - yh * mean(w * yh))
        dya = ry * (wa + yh.abs() * mean(wa * yh.abs()))
    # sums over tokens: some hundred additions one after another at most, of terms as above
    many = 2 ** -16 + 2 ** -24 * (x.shape[0] * x.shape[1] / 152 + 200)
    out["dx"], out["dy"] = (t, 2 ** -16 * ta), (dy, 2 ** -16 * dya)
    slope = g * (1 - g) if sigmoid else torch.ones_like(g)
    # (g is off by some 2^-21 where it comes from a sigmoid, 1 - g by as much, not relative to itself)
    dg, dga = c * yn * slope, ca * ya * (slope + (2 ** -4 if sigmoid else 0))
    if gate is not None:
        out["dgate"] = (dg, 2 ** -16 * dga) if gate.dim() == 3 else (dg.sum((0, 1)), many * dga.sum((0, 1)))
    if post_norm:
        out["dgamma_post"] = ((c * gk * yh).sum((0, 1)), many * (ca * gk.abs() * yh.abs()).sum((0, 1)))
    if pre_norm:
        out["dgamma_pre"] = ((dhv * xh).sum((0, 1)), many * (dhv.abs() * xa).sum((0, 1)))
    return out


LEAST = -2.0 ** 90


def logprobs(logits, targets=None, top=0, scale=1.0, dlogp=None, dentropy=None, dlse=None, dtop=None):
    """{name: (value, bound)}; "top" has no bound.

    A weight 2^(c z - c m) is off by u (|c z| + 2 |c z - c m|) + 2^-22 (the power), a sum of V of them over
    at most V / 32 additions on a lane and a tree by (V / 32 + 16) u: the bound of lse below."""
    scale = float(np.float32(scale))
    z = logits.to(F64)
    V = z.shape[-1]
    ruled = z <= LEAST
    a = torch.where(ruled, -torch.inf, z * scale)
    bad = (torch.isnan(z) | (z > -LEAST)).any(-1)
    none = ruled.all(-1)
    lse = torch.logsumexp(a, -1)
    logp = torch.where(ruled, -torch.inf, a - lse[..., None])
    p = torch.where(ruled, 0.0, torch.exp(logp))
    H = -torch.where(p > 0, p * logp, 0.0).sum(-1)
    big = torch.where(ruled | torch.isnan(z), 0.0, a.abs()).amax(-1)
    e_lse = 2.0 ** -24 * (V / 32 + 32) + 2.0 ** -22 * (big + 2)
    e_H = e_lse * (4 + 2 * H) + 2.0 ** -22 * big
    nan = torch.full_like(lse, torch.nan)
    fix = lambda t, v: torch.where(bad, nan, torch.where(none, torch.full_like(t, v), t))   # noqa: E731
    lse, H = fix(lse, -torch.inf), fix(H, 0.0)
    zero = torch.zeros_like(lse)
    ok = lambda t: torch.where(torch.isfinite(t), t, 0.0)   # noqa: E731
    out = {"lse": (lse, ok(e_lse)), "entropy": (H, ok(e_H))}
    if targets is not None:
        t64 = targets.long()
        at = t64.clamp(0, V - 1)[..., None]
        lt = fix(logp.gather(-1, at)[..., 0], -torch.inf)
        lt = torch.where(t64 < 0, 0.0, torch.where(t64 >= V, torch.nan, lt))
        out["logp"] = (lt, ok(torch.where(t64 < 0, zero, e_lse + 2.0 ** -23 * (big + ok(lse).abs()))))
    if top:
        idx = torch.sort(logits.to(F64), dim=-1, descending=True, stable=True).indices[..., :top]
        tl = torch.where(bad[..., None], torch.nan, logp.gather(-1, idx))
        tl = torch.where(none[..., None] & ~bad[..., None], -torch.inf, tl)
        out["top"] = (idx.int(), None)
        out["top_logp"] = (tl, ok(e_lse + 2.0 ** -23 * (big + ok(lse).abs()))[..., None].expand_as(tl))
    if dlogp is None and dentropy is None and dlse is None and dtop is None:
        return out
    val = lambda t: zero if t is None else t.to(F64)   # noqa: E731
    gl = zero
    if dlogp is not None:
        gl = torch.where((targets >= 0) & (targets < V), val(dlogp), 0.0)
    dH, dL = val(dentropy), val(dlse)
    G, Ga = gl, gl.abs()
    own = torch.zeros_like(z)
    if dlogp is not None:
        own.scatter_add_(-1, at, gl[..., None])
    if dtop is not None:
        G, Ga = G + val(dtop).sum(-1), Ga + val(dtop).abs().sum(-1)
        own.scatter_add_(-1, idx, val(dtop))
    lp = torch.where(p > 0, logp, 0.0)
    dz = scale * (own + p * ((dL - G)[..., None] - dH[..., None] * (lp + H[..., None])))
    mag = scale * (own.abs() + p * ((dL.abs() + Ga)[..., None] + dH.abs()[..., None] * (lp.abs() + H[..., None])))
    bound = (2 * e_lse + 2.0 ** -21 * big + 2.0 ** -19)[..., None] * mag + scale * p * (dH.abs() * (e_H + e_lse))[..., None]
    # A power below 2^-126, the least normal number of fp32, may be 0: off by at most 2^-126 of what it is
    # multiplied by (beyond 200 below lse, p |log p| itself is less than 200 2^-126).
    bound = bound + 2.0 ** -126 * scale * (dL.abs() + Ga + dH.abs() * (200 + H) + 1)[..., None]
    still = none | ((gl == 0) & (dH == 0) & (dL == 0) & (True if dtop is None else (val(dtop) == 0).all(-1)))
    dz = torch.where(still[..., None], 0.0, torch.where(bad[..., None], torch.nan, torch.where(ruled, 0.0, dz)))
    out["dlogits"] = (dz, ok(torch.where(still[..., None], 0.0, bound)))
    return out
