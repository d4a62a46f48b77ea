"""The cases that the operators around a model's heads are timed on, each beside a plain form in
elementary torch operations: the residual step after a block (norm of its output, gate, dropout,
scaled sum with the stream, norm before the next block), dropout alone, and log probabilities of
given tokens with entropy and top alternatives.

A case is a dict of plain values:
  op        "residual"        the residual step, forward
            "residual_train"  forward and backward of it
            "dropout"         dropout alone
            "logprob"         log probabilities, entropies and top alternatives
            "logprob_train"   the same and the gradient of the logits
  dtype     "bf16" or "f32" storage
  layer     the block's output and the gradient of the next one's input are fp32, as the
            layer's Y and dX are
  x32       the residual stream is fp32
  B, T, d   sequences, tokens of a sequence, width of the stream
  gate      "none", "channel" (a learned vector) or "token" (sigmoid of a value per element)
  p         dropout's probability
  V, top    entries of the vocabulary, alternatives asked for
  masked    part of the vocabulary is ruled out (-inf), as for constrained output
"""
import math

import numpy as np
import torch

own = False

SCALE, EPS, SITE, TEMPERATURE = 0.5, 1e-6, 3, 0.8
FIELDS = ("op", "dtype", "layer", "x32", "B", "T", "d", "gate", "p", "V", "top", "masked")


def _case(name, *values):
    c = dict(zip(FIELDS, values))
    if name is not None:
        c["name"] = name
    return c


def _residual(name, op, dtype, layer, x32, B, T, d, gate, p):
    return _case(name, op, dtype, layer, x32, B, T, d, gate, p, 0, 0, False)


def _logprob(name, op, dtype, B, T, V, top, masked):
    return _case(name, op, dtype, False, False, B, T, 0, "none", 0.0, V, top, masked)


def listed():
    return [
        # serving: the new tokens of eight sequences between two blocks; launch latency
        _residual("residual_B8_T1_d1024", "residual", "bf16", False, False, 8, 1, 1024, "none", 0.0),
        # a prompt at the benchmark's B4 T4096 d1024, after the layer's fp32 Y
        _residual("residual_B4_T4096_d1024", "residual", "bf16", True, False, 4, 4096, 1024, "none", 0.0),
        # training at the benchmark's sizes: a learned vector as gate, dropout
        _residual("residual_train_B4_T4096_d1024", "residual_train", "bf16", True, False, 4, 4096, 1024,
                  "channel", 0.1),
        # a wide model with gated outputs and an fp32 stream, long sequences: the largest step
        _residual("residual_train_B2_T8192_d4096", "residual_train", "bf16", False, True, 2, 8192, 4096,
                  "token", 0.1),
        # fp32 training at a ragged length (T = 1000)
        _residual("residual_train_f32_B4_T1000_d768", "residual_train", "f32", False, False, 4, 1000, 768,
                  "none", 0.0),
        # odd sizes: rows that no 16-byte piece starts with
        _residual("residual_train_B3_T333_d1001", "residual_train", "bf16", False, False, 3, 333, 1001,
                  "channel", 0.2),
        # activations of the small models in training
        _residual("dropout_B8_T1024_d512", "dropout", "bf16", False, False, 8, 1024, 512, "none", 0.1),
        # fp32 activations at the benchmark's sizes
        _residual("dropout_f32_B4_T4096_d1024", "dropout", "f32", False, False, 4, 4096, 1024, "none", 0.25),
        # serving: the next tokens of eight sequences with their alternatives, constrained output
        _logprob("logprob_B8_T1_V131072_top20", "logprob", "bf16", 8, 1, 131072, 20, True),
        # scoring prompts, a vocabulary of odd size
        _logprob("logprob_B4_T1024_V50001_top5", "logprob", "bf16", 4, 1024, 50001, 5, False),
        # the loss of a training step at the benchmark's B4 T4096: the most work
        _logprob("logprob_train_B4_T4096_V32768", "logprob_train", "bf16", 4, 4096, 32768, 0, False),
        # fp32 logits, odd sizes, gradients through the alternatives too (distillation)
        _logprob("logprob_train_f32_B2_T500_V32003_top8", "logprob_train", "f32", 2, 500, 32003, 8, False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), _cost(c))
    while True:
        op = rng.choice(("residual", "residual_train", "residual_train", "dropout", "logprob", "logprob_train"))
        dtype = "f32" if rng.random() < 0.3 else "bf16"
        B, T = _log_int(rng, 1, 16), _log_int(rng, 1, 8192)
        if op.startswith("logprob"):
            V = _log_int(rng, 40, 200000)
            V = V if rng.random() < 0.5 else -(-V // 64) * 64
            top = rng.choice((0, 0, 1, 3, 5, 10, 20, 32))
            c = _logprob(None, op, dtype, B, T, V, top, op == "logprob" and rng.random() < 0.3)
        else:
            d = _log_int(rng, 8, 8192)
            d = rng.choice((d, -(-d // 8) * 8, -(-d // 64) * 64, -(-d // 64) * 64))
            gate, p = rng.choice(("none", "channel", "token")), rng.choice((0.0, 0.1, 0.1, 0.25))
            layer, x32 = rng.random() < 0.4, rng.random() < 0.3
            if op == "dropout":
                gate, p, layer, x32 = "none", p or 0.5, False, False
            c = _residual(None, op, dtype, layer, x32, B, T, d, gate, p)
        if _cost(c) <= most[op]:
            return c


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    c = {k: case[k] for k in FIELDS}
    gen = torch.Generator(device="cuda").manual_seed(seed)
    f32 = torch.float32
    dt = torch.bfloat16 if c["dtype"] == "bf16" else f32
    B, T, d, V, op = (c[n] for n in ("B", "T", "d", "V", "op"))

    def rand(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    s = {"case": c}
    if op.startswith("logprob"):
        z = torch.empty(B, T, V, device="cuda", dtype=dt)
        targets = torch.empty(B, T, device="cuda", dtype=torch.int64)
        # words differ in how common they are, and each place prefers some of them
        common = -1.5 * torch.log1p(torch.rand(V, generator=gen, device="cuda") * V)
        for b in range(B):   # by sequence, so that the fp32 draws stay small
            zb = 2.0 * rand(T, V) + common
            if c["masked"]:
                zb[torch.rand(T, V, generator=gen, device="cuda") < 0.6] = -math.inf
                zb[:, 17] = 1.0
            z[b] = zb.to(dt)
            best = zb.argmax(-1)
            other = torch.randint(0, V, (T,), generator=gen, device="cuda")
            pick = torch.rand(T, generator=gen, device="cuda")
            targets[b] = torch.where(pick < 0.6, best, torch.full_like(other, 17) if c["masked"] else other)
            if op == "logprob_train":   # padding carries no target
                targets[b][pick > 0.9] = -1
        s.update(logits=z, targets=targets)
        if op == "logprob_train":
            n = B * T
            # a policy's advantages, an entropy bonus, and weights on the alternatives
            s["dlogp"] = rand(B, T) / n
            s["dentropy"] = torch.full((B, T), -0.01 / n, device="cuda")
            s["dtop"] = rand(B, T, c["top"]).abs() / -n if c["top"] else None
        return s
    s["rng"] = torch.randint(0, 2 ** 62, (2,), generator=gen, device="cuda", dtype=torch.int64)
    if op == "dropout":
        s["x"] = rand(B, T, d).to(dt)
        return s
    xt, yt = f32 if c["x32"] else dt, f32 if c["layer"] else dt
    # a stream that grew over earlier blocks, with a few strong channels; a block's output
    strong = 1 + 4 * (torch.rand(d, generator=gen, device="cuda") < 0.02)
    s["x"] = (2 * rand(B, T, d) * strong).to(xt)
    s["y"] = (0.3 * rand(B, T, d)).to(yt)
    s["gamma_post"], s["gamma_pre"] = ((1 + 0.2 * rand(d)).to(dt) for _ in range(2))
    s["gate"] = {"none": None, "channel": (0.5 + 0.2 * rand(d)).to(dt),
                 "token": rand(B, T, d).to(dt) if c["gate"] == "token" else None}[c["gate"]]
    if op == "residual_train":
        s["dx_out"] = rand(B, T, d).to(xt)
        s["dh"] = rand(B, T, d).to(yt)
    return s


# -------------------------------------------------------------- plain forms

def _words(rng, site, rows, d):
    """One 32-bit word for each of d places of each row (int64 tensor): counter-based, four
    words from each counter (place // 4, row, offset + site), seven rounds of Philox 4x32 (Salmon et
    al., "Parallel random numbers: as easy as 1, 2, 3", 2011) under the seed as key."""
    low, dev = 0xFFFFFFFF, rng.device
    c0 = torch.arange(-(-d // 4), device=dev).expand(rows, -1)
    c1 = torch.arange(rows, device=dev)[:, None].expand_as(c0)
    off = rng[1] + site
    c2, c3 = (off & low).expand_as(c0), (off >> 32 & low).expand_as(c0)
    k0, k1 = rng[0] & low, rng[0] >> 32 & low
    for _ in range(7):
        a, b = 0xD2511F53 * c0, 0xCD9E8D57 * c2   # (mod 2^64: the shift's sign bits are cut off)
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    return torch.stack((c0, c1, c2, c3), -1).reshape(rows, -1)[:, :d]


def _kept(rng, shape, p):
    """1/(1-p) where a value is kept, else 0."""
    rows, d = math.prod(shape[:-1]), shape[-1]
    keep = _words(rng, SITE, rows, d) >= round(p * 2 ** 32)
    return torch.where(keep, 1 / (1 - p), 0.0).float().reshape(shape)


def _plain_dropout(s, c):
    x = s["x"]
    m = _kept(s["rng"], x.shape, c["p"])
    return {"y": torch.where(m == 0, 0.0, x.float() * m).to(x.dtype)}


def _plain_residual(s, c):
    x, y, post, pre = (s[n].float() for n in ("x", "y", "gamma_post", "gamma_pre"))
    xt, dt = s["x"].dtype, s["gamma_pre"].dtype
    m = _kept(s["rng"], x.shape, c["p"]) if c["p"] else 1.0
    g = 1.0
    if c["gate"] != "none":
        g = s["gate"].float()
        g = torch.sigmoid(g) if c["gate"] == "token" else g
    ry = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
    n = y * ry * post
    x1 = x + SCALE * (m * (g * n))
    rx = torch.rsqrt(x1.square().mean(-1, keepdim=True) + EPS)
    xh = x1 * rx
    out = {"x": x1.to(xt), "h": (xh * pre).to(dt)}
    if c["op"] == "residual":
        return out
    dh = s["dh"].float()
    e = dh * pre
    t = s["dx_out"].float() + rx * (e - xh * (e * xh).mean(-1, keepdim=True))
    u = SCALE * m * t
    f, yh = u * g, y * ry
    w = f * post
    out.update(dx=t.to(xt), dy=(ry * (w - yh * (w * yh).mean(-1, keepdim=True))).to(dt),
               dgamma_pre=(dh * xh).sum((0, 1)), dgamma_post=(f * yh).sum((0, 1)))
    if c["gate"] == "channel":
        out["dgate"] = (u * n).sum((0, 1))
    elif c["gate"] == "token":
        out["dgate"] = (u * n * g * (1 - g)).to(dt)
    return out


def _top(z, k):
    """Places of the k largest of each row, ties by the lower index."""
    bits = (z.float() + 0.0).view(torch.int32)
    order = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF).long()
    key = order * 2 ** 32 + (2 ** 32 - 1 - torch.arange(z.shape[-1], device=z.device))
    return 2 ** 32 - 1 - (key.topk(k, -1).values & 0xFFFFFFFF)


def _plain_logprob(s, c):
    z, targets, k = s["logits"], s["targets"], c["top"]
    a = z.float() * TEMPERATURE
    m = a.amax(-1, keepdim=True)
    e = torch.exp(a - m)
    S = e.sum(-1, keepdim=True)
    lse = m + torch.log(S)
    p = e / S
    entropy = torch.log(S) - torch.where(p > 0, p * (a - m), 0.0).sum(-1, keepdim=True)
    at = targets.clamp(min=0)[..., None]
    logp = torch.where(targets < 0, 0.0, (a.gather(-1, at) - lse)[..., 0])
    out = {"logp": logp, "entropy": entropy[..., 0], "lse": lse[..., 0]}
    if k:
        top = _top(z, k)
        out["top"], out["top_logp"] = top.int(), a.gather(-1, top) - lse
    if c["op"] == "logprob":
        return out
    g = torch.where(targets < 0, 0.0, s["dlogp"])[..., None]
    G = g
    if k:
        G = G + s["dtop"].sum(-1, keepdim=True)
    dz = -p * (G + s["dentropy"][..., None] * (a - lse + entropy))
    dz.scatter_add_(-1, at, g)
    if k:
        dz.scatter_add_(-1, top, s["dtop"])
    out["dlogits"] = (dz * TEMPERATURE).to(z.dtype)
    return out


def _plain(s, c):
    if c["op"] == "dropout":
        return _plain_dropout(s, c)
    return _plain_logprob(s, c) if c["op"].startswith("logprob") else _plain_residual(s, c)


# ------------------------------------------------- the framework's operators

def _own(s, c):
    import paper_2505_00315_gb300 as mosa
    if c["op"] == "dropout":
        return {"y": mosa.mosa_dropout(s["x"], c["p"], s["rng"], site=SITE)}
    if c["op"].startswith("logprob"):
        out, s["ws"] = mosa.mosa_token_logprobs(s["logits"], s["targets"], top=c["top"], scale=TEMPERATURE,
                                                workspace=s.get("ws"))
        if c["op"] == "logprob_train":
            out["dlogits"] = mosa.mosa_token_logprobs_backward(
                s["logits"], s["targets"], out["lse"], out["entropy"], dlogp=s["dlogp"],
                dentropy=s["dentropy"], top=out.get("top"), dtop_logp=s["dtop"], scale=TEMPERATURE)
        return out
    kw = dict(gate=s["gate"], gamma_post=s["gamma_post"], gamma_pre=s["gamma_pre"],
              sigmoid=c["gate"] == "token", scale=SCALE, eps=EPS, dropout=c["p"], rng=s["rng"], site=SITE)
    x, h, stats = mosa.mosa_residual_forward(s["x"], s["y"], **kw)
    out = {"x": x, "h": h}
    if c["op"] == "residual_train":
        g, s["ws"] = mosa.mosa_residual_backward(s["x"], s["y"], stats, s["dx_out"], s["dh"],
                                                 workspace=s.get("ws"), **kw)
        out.update(g)
    return out


def run(s):
    return _own(s, s["case"]) if own else _plain(s, s["case"])


# ------------------------------------------------------------- work, 64 bits

def work(case):
    c = {k: case[k] for k in FIELDS}
    e = 2 if c["dtype"] == "bf16" else 4
    rows, d, op = c["B"] * c["T"], c["d"], c["op"]
    if op == "dropout":
        return {"bytes": 2 * rows * d * e, "flops": 2 * rows * d}
    if op.startswith("logprob"):
        n = rows * c["V"]
        if op == "logprob":
            return {"bytes": n * e + rows * (20 + 8 * c["top"]), "flops": 6 * n}
        return {"bytes": 3 * n * e + rows * (28 + 12 * c["top"]), "flops": 12 * n}
    n, x, y = rows * d, 4 if c["x32"] else e, 4 if c["layer"] else e
    token = e if c["gate"] == "token" else 0
    if op == "residual":
        return {"bytes": n * (2 * x + y + e + token) + 2 * d * e, "flops": 12 * n}
    # x, y, gate, dx_out and dh come in, x, h, dx, dy and the gate's gradient go out; the
    # backward cannot begin before the forward has ended, and reads x, y and the gate again
    return {"bytes": n * (5 * x + 3 * y + 2 * e + 3 * token) + 5 * d * e, "flops": 40 * n}


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 10)


def _exact_mask(s, c, shape):
    """The same words by NumPy's unsigned integers."""
    seed, offset = (int(v) for v in s["rng"].tolist())
    rows, d = math.prod(shape[:-1]), shape[-1]
    u = np.uint64
    q = (d + 3) // 4
    low, half = u(0xFFFFFFFF), u(32)
    x = [np.broadcast_to(np.arange(q, dtype=u)[None], (rows, q)),
         np.broadcast_to(np.arange(rows, dtype=u)[:, None], (rows, q)),
         np.full((rows, q), (offset + SITE) % 2 ** 32, u), np.full((rows, q), (offset + SITE) // 2 ** 32, u)]
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for r in range(7):
        k0 = u((key[0] + r * 0x9E3779B9) % 2 ** 32)
        k1 = u((key[1] + r * 0xBB67AE85) % 2 ** 32)
        a, b = x[0] * u(0xD2511F53), x[2] * u(0xCD9E8D57)
        x = [(b >> half) ^ x[1] ^ k0, b & low, (a >> half) ^ x[3] ^ k1, a & low]
    words = np.stack(x, -1).reshape(rows, 4 * q)[:, :d]
    keep = torch.from_numpy(words >= u(round(c["p"] * 2 ** 32))).to(s["rng"].device)
    return keep.reshape(shape).double() / (1 - c["p"])


def _exact_residual(s, c):
    """Gradients by autograd."""
    v = {n: s[n].double().requires_grad_() for n in ("x", "y", "gamma_post", "gamma_pre")}
    if s["gate"] is not None:
        v["gate"] = s["gate"].double().requires_grad_()

    def norm(t, gamma):
        return t / torch.sqrt((t * t).sum(-1, keepdim=True) / c["d"] + EPS) * gamma

    u = norm(v["y"], v["gamma_post"])
    if c["gate"] == "token":
        u = u / (1 + torch.exp(-v["gate"]))
    elif c["gate"] == "channel":
        u = u * v["gate"]
    if c["p"]:
        u = u * _exact_mask(s, c, u.shape)
    x = v["x"] + SCALE * u
    h = norm(x, v["gamma_pre"])
    out = {"x": x.detach(), "h": h.detach()}
    if c["op"] == "residual_train":
        g = torch.autograd.grad((x, h), list(v.values()), (s["dx_out"].double(), s["dh"].double()))
        out.update(zip(("d" + n for n in v), g))
    return out


def _exact_logprob(s, c):
    """A few rows at a time."""
    V, k, rows = c["V"], c["top"], c["B"] * c["T"]
    z, targets = s["logits"].view(rows, V), s["targets"].view(rows)
    f64 = dict(dtype=torch.float64, device=z.device)
    out = {n: torch.zeros(rows, **f64) for n in ("logp", "entropy", "lse")}
    if k:
        out["top"] = torch.zeros(rows, k, dtype=torch.int32, device=z.device)
        out["top_logp"] = torch.zeros(rows, k, **f64)
    train = c["op"] == "logprob_train"
    if train:
        out["dlogits"] = torch.zeros(rows, V, **f64)
    step = max(1, (1 << 25) // V)
    for i in range(0, rows, step):
        a = z[i:i + step].double().mul(TEMPERATURE)
        if train:
            a.requires_grad_()
        logp = torch.log_softmax(a, -1)
        p = logp.exp()
        H = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(-1)
        t = targets[i:i + step]
        own_logp = torch.where(t < 0, torch.zeros_like(H), logp.gather(1, t.clamp(min=0)[:, None])[:, 0])
        sl = slice(i, i + a.shape[0])
        out["logp"][sl], out["entropy"][sl] = own_logp.detach(), H.detach()
        out["lse"][sl] = torch.logsumexp(a.detach(), -1)
        loss = 0.0
        if k:
            idx = torch.sort(z[i:i + step].float(), dim=-1, descending=True, stable=True).indices[:, :k]
            top = logp.gather(1, idx)
            out["top"][sl], out["top_logp"][sl] = idx.int(), top.detach()
            if train:
                loss = (top * s["dtop"].view(rows, k)[sl].double()).sum()
        if train:
            loss = loss + (own_logp * s["dlogp"].view(-1)[sl].double()).sum() + \
                (H * s["dentropy"].view(-1)[sl].double()).sum()
            out["dlogits"][sl] = torch.autograd.grad(loss, a)[0] * TEMPERATURE
    return {n: t.view(*s["targets"].shape, *t.shape[1:]) for n, t in out.items()}


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "dropout":
        return {"y": s["x"].double() * _exact_mask(s, c, s["x"].shape)}
    return _exact_logprob(s, c) if c["op"].startswith("logprob") else _exact_residual(s, c)
