"""Plain 64-bit implementations of the window heads' operators, from their
definitions (test infrastructure; no code of the library)."""
import math

import torch


def visible(Tq, Tk, window, sinks, length, device):
    """[Tq, Tk] truth values: which tokens each of the last Tq of Tk tokens sees."""
    p = torch.arange(Tk - Tq, Tk, device=device)[:, None]
    t = torch.arange(Tk, device=device)[None]
    see = (t <= p) & (t < length) & (p < length)
    return see & ((p - t < (window or Tk)) | (t < sinks))


def attention(q, k, v, window, sinks=0, lens=None, scale=0.0, dO=None):
    """O, lse and with dO also dq, dk, dv, in 64 bits; masked places are never touched."""
    B, Tq, H, hp = q.shape
    Tk, Hkv = k.shape[1], k.shape[2]
    scale = scale or 1 / math.sqrt(hp)
    f64 = dict(dtype=torch.float64, device=q.device)
    out = {"O": torch.zeros(q.shape, **f64), "lse": torch.full((B, H, Tq), -math.inf, **f64)}
    if dO is not None:
        out.update(dq=torch.zeros(q.shape, **f64), dk=torch.zeros(k.shape, **f64),
                   dv=torch.zeros(k.shape, **f64))
    for b in range(B):
        n = Tk if lens is None else min(max(int(lens[b]), 0), Tk)
        see = visible(Tq, Tk, window, sinks, n, q.device)
        rows = see.any(1).nonzero()[:, 0]
        cols = see.any(0).nonzero()[:, 0]
        if not len(rows):
            continue
        see = see[rows][:, cols]
        for h in range(H):
            hk = h // (H // Hkv)
            qq, kk, vv = (x.double() for x in (q[b, rows, h], k[b, cols, hk], v[b, cols, hk]))
            S = (qq @ kk.T * scale).masked_fill(~see, -math.inf)
            lse = torch.logsumexp(S, 1)
            P = torch.exp(S - lse[:, None])
            P = torch.where(see, P, torch.zeros_like(P))
            clean = torch.nan_to_num(vv, 0.0, 0.0, 0.0)
            o = P @ clean
            bad = ~torch.isfinite(vv).all(1)
            if bad.any():   # a token with NaN or infinities makes the rows that see it NaN
                o[(see & bad[None]).any(1)] = math.nan
            out["O"][b, rows, h] = o
            out["lse"][b, h, rows] = lse
            if dO is None:
                continue
            g = dO[b, rows, h].double()
            dP = g @ vv.T
            D = torch.where(see, P * dP, torch.zeros_like(P)).sum(1, keepdim=True)
            dS = torch.where(see, P * (dP - D), torch.zeros_like(P)) * scale
            kf, qf, gf = (torch.nan_to_num(x, 0.0, 0.0, 0.0) for x in (kk, qq, g))
            out["dq"][b, rows, h] = dS @ kf
            out["dk"][b, cols, hk] += dS.T @ qf
            out["dv"][b, cols, hk] += P.T @ gf
    return out


def turned(x, pos, rotary, theta, halves):
    """x [..., heads, hp] turned by positions pos [...], in 64 bits."""
    x = x.clone()
    for p in range(rotary // 2):
        a = pos.double() * theta ** (-2.0 * p / rotary)
        c, s = torch.cos(a)[..., None], torch.sin(a)[..., None]
        i, j = (p, p + rotary // 2) if halves else (2 * p, 2 * p + 1)
        x0, x1 = x[..., i].clone(), x[..., j].clone()
        x[..., i], x[..., j] = x0 * c - x1 * s, x0 * s + x1 * c
    return x


def norm_rope(x, gamma, pos, rotary, theta=10000.0, eps=1e-6, halves=False, norm=True):
    x = x.double()
    if norm:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if gamma is not None:
            x = x * gamma.double()
    return turned(x, pos, rotary, theta, halves)


def norm_rope_grad(x, gamma, pos, dy, rotary, theta=10000.0, eps=1e-6, halves=False):
    """dx and dgamma from the formula: dx = r (u - n mean(u n)), u = g gamma, g turned back."""
    x = x.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n = x * r
    g = turned(dy.double(), -pos.double(), rotary, theta, halves)
    u = g * (gamma.double() if gamma is not None else 1.0)
    dx = r * (u - n * (u * n).mean(-1, keepdim=True))
    return dx, (g * n).reshape(-1, x.shape[-1]).sum(0)


def slot_of(t, sinks, C):
    return t if t < sinks else sinks + (t - sinks) % (C - sinks)


def decode(q, k, v, Kc, Vc, lens, window, sinks, gamma_q, gamma_k, norm, rotary, theta, eps, halves,
           scale=0.0):
    """O and the caches after the step, in 64 bits but for the cache's own rounding of k."""
    B, H, hp = q.shape
    C, Hkv = Kc.shape[1], k.shape[1]
    scale = scale or 1 / math.sqrt(hp)
    Kn, Vn = Kc.double().clone(), Vc.double().clone()
    O = torch.zeros(B, H, hp, dtype=torch.float64, device=q.device)
    for b in range(B):
        n = int(lens[b])
        if n <= 0:
            continue
        at = n - 1
        pos = torch.tensor(at, device=q.device)
        qn = norm_rope(q[b], gamma_q, pos, rotary, theta, eps, halves, norm)
        kn = norm_rope(k[b], gamma_k, pos, rotary, theta, eps, halves, norm)
        s = slot_of(at, sinks, C)
        Kn[b, s], Vn[b, s] = kn.to(Kc.dtype).double(), v[b].double()
        w = min(window or C, C - sinks)
        seen = [t for t in range(n) if t < sinks or at - t < w]
        at_slots = torch.tensor([slot_of(t, sinks, C) for t in seen], device=q.device)
        for h in range(H):
            hk = h // (H // Hkv)
            P = torch.softmax(Kn[b, at_slots, hk] @ qn[h] * scale, 0)
            O[b, h] = P @ Vn[b, at_slots, hk]
    return O, Kn, Vn
