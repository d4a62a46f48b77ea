"""The cases that the window-attention operators are timed on: the per-head norm and rotation of
queries and keys, attention with a sliding window and sink tokens, and the decoding step over a
ring cache, each beside a plain form in elementary torch operations.

A case is a dict of plain values:
  op        "norm"        the norm and rotation alone (forward)
            "norm_train"  forward and backward of it
            "attn"        window attention, forward (a prompt)
            "attn_train"  forward and backward of it
            "decode"      one decoding step: norm, rotation, append to the cache, attention
  dtype     "bf16" or "f32" storage
  B         sequences
  Tq, Tk    queries and keys of a sequence (queries are its last Tq tokens); "decode": Tk is the
            number of slots of the cache
  H, Hkv    query heads and key / value heads
  hp        head size
  window    tokens that a query sees, itself included (0: all before it)
  sinks     first tokens that stay visible
  ragged    sequences end at lengths of their own
  halves    rotation pairs (p, p + rotary/2) instead of (2p, 2p+1)

Queries, keys and values come as a projection leaves them, q | k | v of one token side by side,
where all tokens have queries; caches are [B, Hkv, C, hp].
"""
import math

import torch

own = False

THETA, EPS = 10000.0, 1e-6
FIELDS = ("op", "dtype", "B", "Tq", "Tk", "H", "Hkv", "hp", "window", "sinks", "ragged", "halves")


def _case(name, *values):
    c = dict(zip(FIELDS, values))
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # serving: the new tokens of eight sequences, before they go to a cache; launch latency
        _case("norm_B8_T1_H16", "norm", "bf16", 8, 1, 1, 16, 4, 128, 0, 0, False, False),
        # a prompt of the long-sequence models (T = 8192), heads of 64
        _case("norm_B2_T8192_H16_hp64", "norm", "bf16", 2, 8192, 8192, 16, 16, 64, 0, 0, False, False),
        # a training step at the benchmark's B4 T4096, shared key heads
        _case("norm_train_B4_T4096_H32", "norm_train", "bf16", 4, 4096, 4096, 32, 8, 128, 0, 0, False, True),
        # fp32 training at a ragged length (T = 1000)
        _case("norm_train_f32_B4_T1000_H12", "norm_train", "f32", 4, 1000, 1000, 12, 12, 64, 0, 0, False, False),
        # the smallest call: two short prompts, little more than a tile
        _case("attn_B2_T77_H4", "attn", "bf16", 2, 77, 77, 4, 4, 64, 32, 4, False, False),
        # one long prompt with shared key heads: the most work of a prompt
        _case("attn_B1_T16384_H32_w2048", "attn", "bf16", 1, 16384, 16384, 32, 8, 128, 2048, 4, False, False),
        # a late chunk of a long prompt, sequences of their own lengths, odd sizes
        _case("attn_chunk_B2_T1000_of_8191", "attn", "bf16", 2, 1000, 8191, 16, 4, 64, 1500, 16, True, False),
        # training at the benchmark's B4 T4096: the largest step
        _case("attn_train_B4_T4096_H16_w1024", "attn_train", "bf16", 4, 4096, 4096, 16, 4, 128, 1024, 4, False, False),
        # the four local heads beside the MoSA heads of the long-sequence hybrid (window 512),
        # the first token kept
        _case("attn_train_B2_T8192_H4_w512", "attn_train", "bf16", 2, 8192, 8192, 4, 4, 64, 512, 1, False, False),
        # fp32 training, ragged lengths
        _case("attn_train_f32_B2_T1000_H12", "attn_train", "f32", 2, 1000, 1000, 12, 12, 64, 125, 4, True, False),
        # one sequence being decoded: latency
        _case("decode_B1_C1028_H16", "decode", "bf16", 1, 1, 1028, 16, 4, 128, 1024, 4, False, False),
        # a serving batch at lengths of their own, some past the ring's end: the caches' bytes count
        _case("decode_B48_C4100_H32", "decode", "bf16", 48, 1, 4100, 32, 8, 128, 4096, 4, True, False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op)
            for op in ("norm", "norm_train", "attn", "attn_train", "decode")}
    while True:
        op = rng.choice(("norm", "norm_train", "attn", "attn_train", "attn_train", "decode"))
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        hp = rng.choice((32, 64, 64, 128, 128))
        Hkv = rng.choice((1, 2, 3, 4, 8))
        H = Hkv * rng.choice((1, 2, 3, 4, 8))
        B = _log_int(rng, 1, 64 if op == "decode" else 8)
        window, sinks = _log_int(rng, 16, 4096), rng.choice((0, 1, 4, 4, 16, 130))
        ragged, halves = rng.random() < 0.4, rng.random() < 0.3
        if op == "decode":
            Tq, Tk = 1, sinks + window + rng.choice((0, 0, 5))
        else:
            Tk = _log_int(rng, 1, 16384)
            Tq = Tk
            if op == "attn" and rng.random() < 0.3:
                Tq = rng.randint(1, Tk)
            if op.startswith("norm"):
                window, sinks, ragged = 0, 0, False
            else:
                halves = False
                if rng.random() < 0.15 and Tk <= 4096:
                    window = 0
        c = _case(None, op, dtype, B, Tq, Tk, H, Hkv, hp, window, sinks, ragged, halves)
        f32_most = max(_cost(x) for x in listed() if x["op"] == "attn_train" and x["dtype"] == "f32")
        slow = dtype == "f32" and op.startswith("attn")
        if _cost(c) <= (4 * f32_most if slow else most[op]):
            return c


# ------------------------------------------------------------------ inputs

def _lens(c, gen):
    """Lengths of the sequences on the GPU, or None."""
    B, Tk = c["B"], c["Tk"]
    if c["op"] == "decode":
        if c["ragged"]:   # from one token to well past the ring's end
            return torch.randint(1, 3 * Tk, (B,), generator=gen, device="cuda", dtype=torch.int32)
        return torch.full((B,), Tk, device="cuda", dtype=torch.int32)
    if c["ragged"]:   # the first one whole, the others end somewhere among the queries
        n = torch.randint(Tk - c["Tq"], Tk + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
        n[0] = Tk
        return n
    return None


def prepare(case, seed):
    c = {k: case[k] for k in FIELDS}
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    B, Tq, Tk, H, Hkv, hp, op = (c[n] for n in ("B", "Tq", "Tk", "H", "Hkv", "hp", "op"))

    def rand(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    s = {"case": c, "lens": _lens(c, gen)}
    # a direction that queries share and the first tokens' keys answer to, as sinks do
    u = rand(hp)
    if op == "decode" or Tq == Tk:
        T = 1 if op == "decode" else Tk
        x = rand(B, T, H + 2 * Hkv, hp)
        x[:, :, :H] += 0.5 * u
        if op != "decode":
            x[:, :c["sinks"], H:H + Hkv] += 0.5 * u
        x = x.to(dt)
        q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
        if op == "decode":
            q, k, v = q[:, 0], k[:, 0], v[:, 0]
    else:
        q = (rand(B, Tq, H, hp) + 0.5 * u).to(dt)
        k = rand(B, Tk, Hkv, hp)
        k[:, :c["sinks"]] += 0.5 * u
        k, v = k.to(dt), rand(B, Tk, Hkv, hp).to(dt)
    s.update(q=q, k=k, v=v)
    if op in ("norm", "norm_train", "decode"):
        s["gq"] = (1 + 0.2 * rand(hp)).to(dt)
        s["gk"] = (1 + 0.2 * rand(hp)).to(dt)
    if op in ("norm", "norm_train"):
        # prompts that start anywhere in their text
        start = torch.randint(0, 50000, (B, 1), generator=gen, device="cuda", dtype=torch.int32)
        s["positions"] = (start + torch.arange(Tk, device="cuda", dtype=torch.int32)).contiguous()
    if op == "norm_train":
        s["dq"], s["dk"] = rand(B, Tk, H, hp).to(dt), rand(B, Tk, Hkv, hp).to(dt)
    if op == "attn_train":
        s["dO"] = rand(B, Tq, H, hp).to(dt)
    if op == "decode":
        # keys as an earlier step left them (normalised), values as projected
        kc = torch.empty(B, Hkv, Tk, hp, device="cuda", dtype=dt)
        vc = torch.empty(B, Hkv, Tk, hp, device="cuda", dtype=dt)
        for b in range(B):   # by sequence, so that the fp32 draws stay small
            kc[b] = rand(Hkv, Tk, hp).to(dt)
            vc[b] = rand(Hkv, Tk, hp).to(dt)
        s["K_cache"], s["V_cache"] = kc.transpose(1, 2), vc.transpose(1, 2)   # [B, C, Hkv, hp]
    return s


# -------------------------------------------------------------- plain forms

def _cos_sin(positions, hp):
    """cos and sin of every pair's angle; the angle itself in 64 bits (in 32 it would be off by
    4e-3 at position 65535)."""
    rotary = hp // 2
    p = torch.arange(rotary // 2, device=positions.device, dtype=torch.float64)
    a = positions.double()[..., None] * THETA ** (-2 * p / rotary)
    return torch.cos(a).float(), torch.sin(a).float()


def _turn(x, cos, sin, halves):
    """x [..., heads, hp] with its first hp/2 dimensions turned; cos, sin [..., hp/4]."""
    r = x.shape[-1] // 2
    cos, sin = cos[..., None, :], sin[..., None, :]
    y = x.clone()
    if halves:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * cos - b * sin, a * sin + b * cos
    return y


def _plain_norm(x, gamma, cos, sin, halves):
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return _turn(x * r * gamma.float(), cos, sin, halves)


def _plain_norm_grad(x, gamma, cos, sin, halves, dy):
    x, gamma = x.float(), gamma.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    n = x * r
    g = _turn(dy.float(), cos, -sin, halves)
    u = g * gamma
    dx = r * (u - n * (u * n).mean(-1, keepdim=True))
    return dx, (g * n).sum((0, 1, 2))


def _blocks(x, first, length, size, step):
    """Rows [first, first + length) of x [B, Hkv, T, hp] (zeros outside) as blocks
    [B, Hkv, n, size, hp] that start `step` apart."""
    T = x.shape[2]
    lo, hi = max(0, first), min(T, first + length)
    x = torch.nn.functional.pad(x[:, :, lo:hi], (0, 0, lo - first, first + length - hi))
    return x.unfold(2, size, step).transpose(-1, -2)


def _plain_attention(q, k, v, window, sinks, lens, dO=None):
    """Scores of a block of queries against the keys within its window, and against the sinks."""
    dt, dev = q.dtype, q.device
    B, Tq, H, hp = q.shape
    Tk, Hkv = k.shape[1], k.shape[2]
    G, scale = H // Hkv, 1 / math.sqrt(hp)
    w = min(window or Tk, Tk)
    off = Tk - Tq
    step = min(Tq, max(128, w))
    n = -(-Tq // step)
    size, s = step + w, min(sinks, Tk)

    def rows(x):   # [B, Tq, H, hp] -> [B, Hkv, G, n, step, hp]
        x = x.float().reshape(B, Tq, Hkv, G, hp).permute(0, 2, 3, 1, 4)
        return torch.nn.functional.pad(x, (0, 0, 0, n * step - Tq)).reshape(B, Hkv, G, n, step, hp)

    qf = rows(q)
    kf, vf = k.float().transpose(1, 2), v.float().transpose(1, 2)
    kb, vb = (_blocks(x, off - w, w + n * step, size, step) for x in (kf, vf))
    ks, vs = kf[:, :, :s], vf[:, :, :s]
    at = off + torch.arange(n * step, device=dev).view(n, step, 1)
    tl = (off - w + step * torch.arange(n, device=dev)[:, None] + torch.arange(size, device=dev))[:, None]
    ts = torch.arange(s, device=dev)
    end = torch.full((B,), Tk, device=dev) if lens is None else lens.clamp(0, Tk).long()
    end = end.view(B, 1, 1, 1)
    near = (tl >= 0) & (tl <= at) & (tl > at - w) & (tl < end) & (at < end)
    far = (ts <= at - w) & (ts < end) & (at < end)
    S = torch.cat([torch.einsum("bhgnid,bhnjd->bhgnij", qf, kb),
                   torch.einsum("bhgnid,bhjd->bhgnij", qf, ks)], -1) * scale
    S.masked_fill_(~torch.cat([near, far], -1)[:, None, None], -math.inf)
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = torch.exp(S - m)
    l = P.sum(-1, keepdim=True)
    lse = (m + torch.log(l))[..., 0]
    P = P / torch.where(l == 0, torch.ones_like(l), l)
    O = torch.einsum("bhgnij,bhnjd->bhgnid", P[..., :size], vb) + \
        torch.einsum("bhgnij,bhjd->bhgnid", P[..., size:], vs)

    def back(x):   # [B, Hkv, G, n, step, ..] -> [B, Tq, H, ..]
        x = x.reshape(B, H, n * step, *x.shape[5:])[:, :, :Tq]
        return x.transpose(1, 2)

    out = {"O": back(O).to(dt).contiguous(), "lse": lse.reshape(B, H, n * step)[:, :, :Tq].contiguous()}
    if dO is None:
        return out
    g = rows(dO)
    dP = torch.cat([torch.einsum("bhgnid,bhnjd->bhgnij", g, vb),
                    torch.einsum("bhgnid,bhjd->bhgnij", g, vs)], -1)
    dS = P * (dP - (P * dP).sum(-1, keepdim=True)) * scale
    dq = torch.einsum("bhgnij,bhnjd->bhgnid", dS[..., :size], kb) + \
        torch.einsum("bhgnij,bhjd->bhgnid", dS[..., size:], ks)

    def to_keys(A, x):
        """sum over queries of A^T x, put back from the blocks to the keys."""
        blk = torch.einsum("bhgnij,bhgnid->bhnjd", A[..., :size], x)
        full = torch.zeros(B, Hkv, w + n * step, hp, device=dev)
        idx = (step * torch.arange(n, device=dev)[:, None] + torch.arange(size, device=dev)).reshape(-1)
        full.index_add_(2, idx, blk.reshape(B, Hkv, n * size, hp))
        got = torch.zeros(B, Hkv, Tk, hp, device=dev)
        lo = max(0, off - w)
        got[:, :, lo:] = full[:, :, lo - (off - w):lo - (off - w) + Tk - lo]
        got[:, :, :s] += torch.einsum("bhgnij,bhgnid->bhjd", A[..., size:], x)
        return got.transpose(1, 2).to(dt).contiguous()

    out.update(dq=back(dq).to(dt).contiguous(), dk=to_keys(dS, qf), dv=to_keys(P, g))
    return out


def _plain_decode(s, c):
    dt = s["q"].dtype
    B, C, H, Hkv, hp, w, n = (c[x] for x in ("B", "Tk", "H", "Hkv", "hp", "window", "sinks"))
    Kc, Vc, lens = s["K_cache"], s["V_cache"], s["lens"].long()
    at, ring = lens - 1, C - n
    cos, sin = _cos_sin(at, hp)
    qn = _plain_norm(s["q"], s["gq"], cos, sin, c["halves"])
    kn = _plain_norm(s["k"], s["gk"], cos, sin, c["halves"])
    slot = torch.where(at < n, at, n + (at - n) % ring)
    rows = torch.arange(B, device=lens.device)
    Kc[rows, slot] = kn.to(dt)
    Vc[rows, slot] = s["v"]
    # the token that each slot holds: the last one not after `at` that goes there
    i = torch.arange(C, device=lens.device)
    t = torch.where(i < n, i, at[:, None] - (at[:, None] - i) % ring)
    held = (t <= at[:, None]) & ((i < n) | (t >= n))
    seen = held & ((t < n) | (t > at[:, None] - w))
    q = qn.view(B, Hkv, H // Hkv, hp)
    S = torch.einsum("bhgd,bchd->bhgc", q, Kc.float()) / math.sqrt(hp)
    S = S.masked_fill(~seen[:, None, None], -math.inf)
    P = torch.exp(S - S.amax(-1, keepdim=True))
    P = P / P.sum(-1, keepdim=True)
    O = torch.einsum("bhgc,bchd->bhgd", P, Vc.float()).reshape(B, H, hp)
    return {"O": O.to(dt), "K_cache": Kc, "V_cache": Vc}


def _plain(s, c):
    op, dt = c["op"], s["q"].dtype
    if op == "decode":
        return _plain_decode(s, c)
    if op in ("attn", "attn_train"):
        return _plain_attention(s["q"], s["k"], s["v"], c["window"], c["sinks"], s["lens"],
                                s.get("dO"))
    cos, sin = _cos_sin(s["positions"], c["hp"])
    out = {}
    for x in "qk":
        out[x] = _plain_norm(s[x], s["g" + x], cos, sin, c["halves"]).to(dt)
        if op == "norm_train":
            dx, dg = _plain_norm_grad(s[x], s["g" + x], cos, sin, c["halves"], s["d" + x])
            out["d" + x], out["dgamma_" + x] = dx.to(dt), dg
    return out


# ------------------------------------------------- the framework's operators

def _own(s, c):
    import paper_2505_00315_gb300 as mosa
    op = c["op"]
    if op == "decode":
        O, s["ws"] = mosa.mosa_window_decode(
            s["q"], s["k"], s["v"], s["K_cache"], s["V_cache"], s["lens"], c["window"], c["sinks"],
            gamma_q=s["gq"], gamma_k=s["gk"], theta=THETA, eps=EPS, halves=c["halves"],
            workspace=s.get("ws"))
        return {"O": O, "K_cache": s["K_cache"], "V_cache": s["V_cache"]}
    if op in ("attn", "attn_train"):
        O, lse, s["ws"] = mosa.mosa_window_forward(s["q"], s["k"], s["v"], c["window"], c["sinks"],
                                                   lens=s["lens"], workspace=s.get("ws"))
        out = {"O": O, "lse": lse}
        if op == "attn_train":
            out.update(mosa.mosa_window_backward(s["q"], s["k"], s["v"], O, lse, s["dO"], s["ws"],
                                                 c["window"], c["sinks"], lens=s["lens"]))
        return out
    kw = dict(positions=s["positions"], theta=THETA, eps=EPS, halves=c["halves"])
    q, k = mosa.mosa_qk_norm_rope(s["q"], s["k"], s["gq"], s["gk"], **kw)
    out = {"q": q, "k": k}
    if op == "norm_train":
        g, s["ws"] = mosa.mosa_qk_norm_rope_backward(s["q"], s["k"], s["gq"], s["gk"], s["dq"],
                                                     s["dk"], workspace=s.get("ws"), **kw)
        out.update(g)
    return out


def run(s):
    return _own(s, s["case"]) if own else _plain(s, s["case"])


# ------------------------------------------------------------- work, 64 bits

def _pairs(c):
    """Visible (query, key) pairs of one head of one sequence at its full length."""
    off, w = c["Tk"] - c["Tq"], c["window"] or c["Tk"]
    n = 0
    for p in range(off, c["Tk"]):
        near = min(p + 1, w)
        n += near + min(c["sinks"], p + 1 - near)
    return n


def work(case):
    c = {k: case[k] for k in FIELDS}
    B, Tq, Tk, H, Hkv, hp, op = (c[n] for n in ("B", "Tq", "Tk", "H", "Hkv", "hp", "op"))
    e = 2 if c["dtype"] == "bf16" else 4
    if op in ("norm", "norm_train"):
        n = B * Tk * (H + Hkv) * hp
        passes = 2 if op == "norm" else 5   # x and y; then x, dy and dx
        return {"bytes": passes * n * e + 4 * B * Tk, "flops": (10 if op == "norm" else 30) * n}
    part = (B + 1) / (2 * B) if c["ragged"] else 1.0   # lengths but the first are drawn evenly
    if op == "decode":
        rows = min(Tk, c["sinks"] + c["window"]) * (0.8 if c["ragged"] else 1.0)
        return {"bytes": B * (2 * Hkv * rows + 2 * H + 4 * Hkv) * hp * e,
                "flops": 4 * B * H * rows * hp}
    qb, kb, rows = B * Tq * H * hp * e, B * Tk * Hkv * hp * e, 4 * B * H * Tq
    pairs = _pairs(c) * B * H * part
    if op == "attn":
        return {"bytes": 2 * qb + 2 * kb + rows, "flops": 4 * pairs * hp}
    return {"bytes": 6 * qb + 6 * kb + 2 * rows, "flops": 14 * pairs * hp}


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 100)


def _exact_norm(s, c):
    """Each token's heads turned by complex multiplication, gradients by autograd."""
    hp, r = c["hp"], c["hp"] // 2
    pos = s["positions"].double()
    ang = pos[..., None] * torch.tensor([THETA ** (-2.0 * p / r) for p in range(r // 2)],
                                        dtype=torch.float64, device=pos.device)
    z = torch.polar(torch.ones_like(ang), ang)[:, :, None]

    def f(x, gamma):
        n = x / torch.sqrt((x * x).sum(-1, keepdim=True) / hp + EPS) * gamma
        a, b = (n[..., :r // 2], n[..., r // 2:r]) if c["halves"] else (n[..., 0:r:2], n[..., 1:r:2])
        t = torch.complex(a.contiguous(), b.contiguous()) * z
        t = torch.cat([t.real, t.imag], -1) if c["halves"] else torch.view_as_real(t).flatten(-2)
        return torch.cat([t, n[..., r:]], -1)

    out = {}
    for x in "qk":
        v, g = s[x].double().requires_grad_(), s["g" + x].double().requires_grad_()
        y = f(v, g)
        out[x] = y.detach()
        if c["op"] == "norm_train":
            out["d" + x], out["dgamma_" + x] = torch.autograd.grad(y, (v, g), s["d" + x].double())
    return out


def _exact_attention(s, c):
    """Each key head's queries a few at a time, over the keys that one of them sees."""
    q, k, v, dO = (s.get(n) for n in ("q", "k", "v", "dO"))
    B, Tq, Tk, H, Hkv, hp = (c[n] for n in ("B", "Tq", "Tk", "H", "Hkv", "hp"))
    G, off, dev = H // Hkv, Tk - Tq, q.device
    f64 = dict(dtype=torch.float64, device=dev)
    out = {"O": torch.zeros(B, Tq, H, hp, **f64), "lse": torch.full((B, H, Tq), -math.inf, **f64)}
    if dO is not None:
        out.update(dq=torch.zeros(B, Tq, H, hp, **f64), dk=torch.zeros(B, Tk, Hkv, hp, **f64),
                   dv=torch.zeros(B, Tk, Hkv, hp, **f64))
    for b in range(B):
        n = Tk if s["lens"] is None else max(0, min(Tk, int(s["lens"][b])))
        for i in range(0, max(0, min(Tq, n - off)), 512):
            p = torch.arange(i, min(i + 512, n - off), device=dev)[:, None] + off
            t = torch.arange(n, device=dev)[None]
            see = (t <= p) & ((t < c["sinks"]) | (t > p - (c["window"] or Tk)))
            idx = see.any(0).nonzero()[:, 0]
            see = see[:, idx]
            sl = slice(i, i + p.shape[0])
            for h in range(Hkv):
                hs = slice(h * G, h * G + G)
                qq = q[b, sl, hs].double().transpose(0, 1)
                kk, vv = k[b, idx, h].double(), v[b, idx, h].double()
                S = (qq @ kk.T / math.sqrt(hp)).masked_fill(~see, -math.inf)
                lse = torch.logsumexp(S, -1)
                P = torch.exp(S - lse[..., None])
                o = P @ vv
                out["O"][b, sl, hs] = o.transpose(0, 1)
                out["lse"][b, hs, sl] = lse
                if dO is not None:
                    g = dO[b, sl, hs].double().transpose(0, 1)
                    dS = P * (g @ vv.T - (g * o).sum(-1, keepdim=True)) / math.sqrt(hp)
                    out["dq"][b, sl, hs] = (dS @ kk).transpose(0, 1)
                    out["dk"][b, idx, h] += (dS.transpose(1, 2) @ qq).sum(0)
                    out["dv"][b, idx, h] += (P.transpose(1, 2) @ g).sum(0)
    return out


def _exact_decode(s, c):
    """Sequence by sequence, over the list of the tokens that it sees."""
    hp, n, C = c["hp"], c["sinks"], c["Tk"]
    G, r = c["H"] // c["Hkv"], hp // 2
    Kc, Vc = s["K_cache"].double(), s["V_cache"].double()
    out = torch.zeros(c["B"], c["H"], hp, dtype=torch.float64, device=Kc.device)

    def f(x, gamma, at):
        x = x.double()
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / hp + EPS) * gamma.double()
        for p in range(r // 2):
            a = at * THETA ** (-2.0 * p / r)
            i, j = (p, p + r // 2) if c["halves"] else (2 * p, 2 * p + 1)
            x0, x1 = x[:, i].clone(), x[:, j].clone()
            x[:, i], x[:, j] = x0 * math.cos(a) - x1 * math.sin(a), x0 * math.sin(a) + x1 * math.cos(a)
        return x

    for b, length in enumerate(s["lens"].tolist()):
        at = length - 1
        seen = [t for t in range(max(0, at - C), length) if t > at - c["window"] and t >= n]
        seen = torch.tensor([t for t in range(n) if t <= at] + [n + (t - n) % (C - n) for t in seen],
                            device=Kc.device)
        slot = at if at < n else n + (at - n) % (C - n)
        Kc[b, slot] = f(s["k"][b], s["gk"], at)
        Vc[b, slot] = s["v"][b].double()
        q = f(s["q"][b], s["gq"], at).view(c["Hkv"], G, hp)
        kk, vv = Kc[b, seen].transpose(0, 1), Vc[b, seen].transpose(0, 1)
        out[b] = (torch.softmax(q @ kk.transpose(1, 2) / math.sqrt(hp), -1) @ vv).reshape(-1, hp)
    return {"O": out, "K_cache": Kc, "V_cache": Vc}


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "decode":
        return _exact_decode(s, c)
    return _exact_norm(s, c) if c["op"].startswith("norm") else _exact_attention(s, c)
