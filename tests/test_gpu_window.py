"""The window heads against plain 64-bit implementations: norm and rotation of queries and
keys, sliding-window attention with sinks (forward and backward), the decoding step.

Tolerances (relative L2 of each output), from the roundings a result goes through:
  fp32  sums of up to a few thousand products, each within 2^-24 of itself and adding up
        at random, the exponentials within 2 ulp of arguments up to 2^5: under 2^-24 * 2^6
        = 4e-6; 1e-5 with room for the gradients' cancellation.
  bf16  the output's own rounding (2^-9 at most) and, for the attention, that of the
        weights or score gradients (another 2^-9 of each term, adding up at random): 2^-8 = 4e-3,
        and 8e-3 for the gradients of shared heads, which add up cancelling terms.
  lse   fp32 whatever the storage: its bf16 inputs are exact."""
import math

import pytest
import torch

import _window_ref as ref
import paper_2505_00315_gb300 as mosa

pytestmark = pytest.mark.gpu

TOL = {torch.float32: 1e-5, torch.bfloat16: 8e-3}
LSE_TOL = 2e-6
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def rel(got, want):
    got, want = got.double(), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), "finite places differ"
    assert torch.equal(torch.isnan(want), torch.isnan(got)), "NaN places differ"
    off = (got[fine] - want[fine]).norm()
    den = want[fine].norm()
    return float(off / den) if den > 0 else float(off)


def rand(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def inputs(B, Tq, Tk, H, Hkv, hp, dtype, seed=0, layout="packed"):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[dtype]
    if layout == "packed" and Tq == Tk:   # q | k | v of one token side by side
        x = rand(gen, B, Tk, H + 2 * Hkv, hp, dtype=dt)
        q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    elif layout == "heads":               # [B, heads, T, hp] storage
        q = rand(gen, B, H, Tq, hp, dtype=dt).transpose(1, 2)
        k, v = (rand(gen, B, Hkv, Tk, hp, dtype=dt).transpose(1, 2) for _ in range(2))
    elif layout == "unaligned":           # rows that start off 16 bytes
        q = rand(gen, B, Tq, H, hp + 1, dtype=dt)[..., 1:]
        k, v = (rand(gen, B, Tk, Hkv, hp + 3, dtype=dt)[..., :hp] for _ in range(2))
    elif layout == "repeated":            # one key / value head repeated by stride 0
        q = rand(gen, B, Tq, H, hp, dtype=dt)
        k, v = (rand(gen, B, Tk, 1, hp, dtype=dt).expand(B, Tk, Hkv, hp) for _ in range(2))
    else:
        q = rand(gen, B, Tq, H, hp, dtype=dt)
        k, v = (rand(gen, B, Tk, Hkv, hp, dtype=dt) for _ in range(2))
    return q, k, v, rand(gen, B, Tq, H, hp, dtype=dt)


def run(q, k, v, dO, window, sinks, lens=None, scale=0.0):
    O, lse, ws = mosa.mosa_window_forward(q, k, v, window, sinks, lens=lens, scale=scale)
    g = mosa.mosa_window_backward(q, k, v, O, lse, dO, ws, window, sinks, lens=lens, scale=scale)
    assert mosa.mosa_window_check_status(ws) == 0
    return {"O": O, "lse": lse, **g}


def check(got, want, dtype):
    for name, w in want.items():
        e = rel(got[name], w)
        assert e < (LSE_TOL if name == "lse" else TOL[dtype]), f"{name}: {e:.3e}"


CASES = [
    # B, Tq, Tk, H, Hkv, hp, window, sinks, lens
    (1, 1, 1, 1, 1, 64, 1, 0, None),
    (2, 1, 1, 4, 2, 128, 0, 3, None),
    (1, 2, 2, 2, 1, 64, 1, 0, None),
    (2, 7, 7, 3, 3, 16, 3, 1, None),
    (2, 77, 77, 4, 4, 64, 32, 4, None),
    (1, 128, 128, 2, 1, 128, 64, 0, None),
    (1, 129, 129, 2, 1, 64, 128, 1, None),
    (1, 255, 255, 2, 2, 32, 127, 5, None),
    (2, 300, 300, 4, 1, 128, 100, 130, None),     # sinks past a tile
    (1, 500, 500, 8, 1, 64, 0, 0, None),          # no window
    (1, 640, 640, 3, 3, 128, 1, 1, None),         # itself and the first token
    (1, 700, 700, 2, 1, 64, 257, 300, None),      # sinks past the window
    (3, 333, 333, 6, 2, 64, 50, 2, (0, 333, 100)),
    (4, 260, 260, 2, 2, 128, 64, 4, (-3, 1, 1000, 129)),   # clamped, one token, a tile and one
    (2, 1, 1000, 4, 2, 64, 300, 4, None),         # one query of a long text
    (2, 100, 1000, 4, 2, 128, 300, 4, (1000, 950)),
    (2, 129, 700, 4, 4, 64, 0, 0, (400, 600)),    # the first sequence ends before its queries
    (1, 1100, 1200, 2, 1, 64, 256, 17, None),
    (1, 1500, 1500, 5, 5, 128, 129, 1, None),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "_".join(map(str, c[:8])))
def test_attention_against_64_bits(case, dtype):
    B, Tq, Tk, H, Hkv, hp, window, sinks, lens = case
    q, k, v, dO = inputs(B, Tq, Tk, H, Hkv, hp, dtype, seed=Tk + hp)
    lens = None if lens is None else torch.tensor(lens, device="cuda", dtype=torch.int32)
    check(run(q, k, v, dO, window, sinks, lens), ref.attention(q, k, v, window, sinks, lens, dO=dO),
          DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["heads", "unaligned", "repeated", "plain"])
def test_attention_on_other_layouts(layout, dtype):
    q, k, v, dO = inputs(2, 200, 200, 6, 3, 64, dtype, seed=3, layout=layout)
    check(run(q, k, v, dO, 70, 4), ref.attention(q, k, v, 70, 4, dO=dO), DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cuda_core_kernels_give_the_same(dtype, monkeypatch):
    monkeypatch.setenv("MOSA_FORCE_SIMT", "1")
    for hp in (16, 32, 64, 128):
        q, k, v, dO = inputs(2, 200, 200, 4, 2, hp, dtype, seed=5)
        check(run(q, k, v, dO, 70, 4), ref.attention(q, k, v, 70, 4, dO=dO), DT[dtype])


def test_gradients_into_a_packed_buffer_and_a_given_scale():
    q, k, v, dO = inputs(2, 300, 300, 4, 2, 64, "bf16", seed=8)
    want = ref.attention(q, k, v, 90, 2, scale=0.2, dO=dO)
    O, lse, ws = mosa.mosa_window_forward(q, k, v, 90, 2, scale=0.2)
    buf = torch.full((2, 300, 9, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    out = {"dq": buf[:, :, :4], "dk": buf[:, :, 4:6], "dv": buf[:, :, 6:8]}
    g = mosa.mosa_window_backward(q, k, v, O, lse, dO, ws, 90, 2, scale=0.2, out=out)
    check({"O": O, "lse": lse, **g}, want, torch.bfloat16)
    assert (buf[:, :, 8] == 7.0).all()   # beside the outputs nothing is written


@pytest.mark.parametrize("dtype,hp", [("bf16", 64), ("bf16", 128), ("f32", 64), ("bf16", 32)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_the_mask_hides_reaches_nothing(dtype, hp, bad):
    """Tokens past the length hold NaN or infinities, and so does one token within it: rows
    that see neither are as without them."""
    B, T, H, Hkv, w, s = 2, 400, 4, 2, 60, 2
    q, k, v, dO = inputs(B, T, T, H, Hkv, hp, dtype, seed=11, layout="plain")
    lens = torch.tensor([350, 400], device="cuda", dtype=torch.int32)
    want = ref.attention(q, k, v, w, s, lens, dO=dO)
    for x in (q, k, v, dO):
        x[0, 350:] = bad
    got = run(q, k, v, dO, w, s, lens)
    check(got, want, DT[dtype])          # padding: nothing changes at all
    clean = {n: x.clone() for n, x in got.items()}
    j = 200                              # a token that positions j .. j + w - 1 see
    for x in (k, v):
        x[1, j] = bad
    got = run(q, k, v, dO, w, s, lens)
    for n in ("O", "dq"):
        for rows in (slice(0, j), slice(j + w, T)):
            assert torch.equal(got[n][1, rows], clean[n][1, rows]), n
        assert torch.equal(got[n][0], clean[n][0])
    assert not torch.isfinite(got["O"][1, j:j + w].float()).any(-1).any()
    # keys that only rows without the bad token see keep their gradients (not the sinks)
    for n in ("dk", "dv"):
        for rows in (slice(s, j - w + 1), slice(j + w, T)):
            assert torch.equal(got[n][1, rows], clean[n][1, rows]), n


def test_infinite_scores_of_a_query_stay_in_its_row():
    q, k, v, dO = inputs(1, 300, 300, 2, 2, 64, "bf16", seed=12, layout="plain")
    clean = run(q, k, v, dO, 50, 0)
    q[0, 130] = math.nan
    got = run(q, k, v, dO, 50, 0)
    for n in ("O", "dq"):
        keep = torch.arange(300, device="cuda") != 130
        assert torch.equal(got[n][0, keep], clean[n][0, keep])
        assert torch.isnan(got[n][0, 130].float()).all()
    for n in ("dk", "dv"):
        assert torch.equal(got[n][0, :81], clean[n][0, :81])
        assert torch.equal(got[n][0, 131:], clean[n][0, 131:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_same_bits_every_time(dtype):
    q, k, v, dO = inputs(2, 900, 900, 6, 2, 64, dtype, seed=13)
    a, b = run(q, k, v, dO, 130, 3), run(q, k, v, dO, 130, 3)
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_gradients_against_differences():
    """Central differences of <O, dO> in fp32 storage along random directions: the step's own
    error is third order (1e-6 at 1e-2 of unit directions), the outputs' rounding 1e-5."""
    q, k, v, dO = inputs(1, 150, 150, 2, 1, 32, "f32", seed=14, layout="plain")
    g = run(q, k, v, dO, 40, 2)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        d = torch.randn(x.shape, generator=gen, device="cuda")
        h = 1e-2
        f = []
        for sign in (1, -1):
            args = {"dq": (q, k, v), "dk": (q, k, v), "dv": (q, k, v)}[name]
            args = [y + sign * h * d if y is x else y for y in args]
            O = mosa.mosa_window_forward(*args, 40, 2)[0]
            f.append((O.double() * dO.double()).sum())
        want = (f[0] - f[1]) / (2 * h)
        got = (g[name].double() * d.double()).sum()
        scale = g[name].double().norm()
        assert abs(float(got - want)) < 5e-3 * float(scale), name


def test_attention_on_another_stream():
    q, k, v, dO = inputs(2, 500, 500, 4, 2, 128, "bf16", seed=15)
    want = run(q, k, v, dO, 100, 4)
    s = torch.cuda.Stream()
    q2, k2, v2, dO2 = (torch.zeros_like(x) for x in (q, k, v, dO))
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)    # the inputs are written late, on this stream
        for x, y in ((q2, q), (k2, k), (v2, v), (dO2, dO)):
            x.copy_(y)
        got = run(q2, k2, v2, dO2, 100, 4)
    s.synchronize()
    for n in want:
        assert torch.equal(got[n], want[n]), n


# ------------------------------------------------------- norm and rotation

def norm_inputs(B, T, H, Hkv, hp, dtype, layout="packed", seed=0):
    q, k, _, dyq = inputs(B, T, T, H, Hkv, hp, dtype, seed=seed, layout=layout)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    dt = DT[dtype]
    gq, gk = ((1 + 0.3 * rand(gen, hp, dtype=torch.float32)).to(dt) for _ in range(2))
    pos = torch.randint(0, 1 << 20, (B, T), generator=gen, device="cuda", dtype=torch.int32)
    return q, k, gq, gk, dyq, rand(gen, B, T, Hkv, hp, dtype=dt), pos


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,H,Hkv,hp,rotary,halves,layout", [
    (1, 1, 1, 1, 128, None, False, "packed"), (8, 1, 16, 4, 128, None, True, "packed"),
    (2, 77, 5, 1, 64, 64, False, "packed"), (2, 77, 5, 1, 64, 64, True, "packed"),
    (1, 33, 4, 4, 32, 6, False, "plain"), (3, 50, 3, 3, 16, None, True, "plain"),
    (2, 40, 4, 2, 16, 16, True, "plain"), (2, 64, 3, 1, 128, 96, True, "heads"),
    (2, 64, 3, 1, 128, 0, True, "heads"), (2, 31, 6, 2, 64, None, False, "unaligned"),
    (2, 1500, 7, 2, 64, None, False, "packed"), (1, 2500, 12, 12, 128, None, True, "packed"),
])
def test_norm_and_rotation_against_64_bits(B, T, H, Hkv, hp, rotary, halves, layout, dtype):
    q, k, gq, gk, dyq, dyk, pos = norm_inputs(B, T, H, Hkv, hp, dtype, layout, seed=T)
    kw = dict(positions=pos, rotary=rotary, halves=halves)
    yq, yk = mosa.mosa_qk_norm_rope(q, k, gq, gk, **kw)
    g, _ = mosa.mosa_qk_norm_rope_backward(q, k, gq, gk, dyq, dyk, **kw)
    rotary = hp // 2 if rotary is None else rotary
    tol = 2 ** -8 if dtype == "bf16" else 2e-6
    for x, gm, y, dy, dx, dg in ((q, gq, yq, dyq, g["dq"], g["dgamma_q"]),
                                 (k, gk, yk, dyk, g["dk"], g["dgamma_k"])):
        assert rel(y, ref.norm_rope(x, gm, pos, rotary, halves=halves)) < tol
        want, wg = ref.norm_rope_grad(x, gm, pos, dy, rotary, halves=halves)
        assert rel(dx, want) < tol
        # fp32 sums of products that cancel: against the sum of their sizes
        assert float((dg.double() - wg).abs().max()) < 1e-6 * math.sqrt(dy.numel()) * 8


def test_norm_defaults_in_place_and_without_weights():
    q, k, _, _, _, _, _ = norm_inputs(2, 40, 4, 2, 64, "bf16", seed=2)
    pos = torch.arange(40, device="cuda").expand(2, 40)
    wq, wk = (ref.norm_rope(x, None, pos, 32) for x in (q, k))
    mosa.mosa_qk_norm_rope(q, k, out={"q": q, "k": k})
    assert rel(q, wq) < 2 ** -8 and rel(k, wk) < 2 ** -8


def test_norm_gradient_against_differences():
    q, k, gq, gk, dyq, dyk, pos = norm_inputs(1, 20, 2, 1, 32, "f32", "plain", seed=4)
    g, _ = mosa.mosa_qk_norm_rope_backward(q, k, gq, gk, dyq, dyk, positions=pos)
    gen = torch.Generator(device="cuda").manual_seed(3)
    d, h = torch.randn(q.shape, generator=gen, device="cuda"), 1e-2
    f = [(mosa.mosa_qk_norm_rope(q + s * h * d, k, gq, gk, positions=pos)[0].double()
          * dyq.double()).sum() for s in (1, -1)]
    got = float((g["dq"].double() * d.double()).sum())
    assert abs(got - float(f[0] - f[1]) / (2 * h)) < 5e-3 * float(g["dq"].norm())
    dg = torch.randn(32, generator=gen, device="cuda")
    f = [(mosa.mosa_qk_norm_rope(q, k, gq + s * h * dg, gk, positions=pos)[0].double()
          * dyq.double()).sum() for s in (1, -1)]
    got = float((g["dgamma_q"].double() * dg.double()).sum())
    assert abs(got - float(f[0] - f[1]) / (2 * h)) < 5e-3 * float(g["dgamma_q"].norm())


def test_norm_gradient_in_place_and_the_same_bits():
    q, k, gq, gk, dyq, dyk, pos = norm_inputs(2, 3000, 8, 2, 64, "bf16", seed=6)
    a, ws = mosa.mosa_qk_norm_rope_backward(q, k, gq, gk, dyq, dyk, positions=pos)
    ws.fill_(0xFF)   # whatever the workspace held before
    b, _ = mosa.mosa_qk_norm_rope_backward(q, k, gq, gk, dyq, dyk, positions=pos, workspace=ws,
                                           out={"dq": dyq, "dk": dyk})
    for n in a:
        assert torch.equal(a[n], b[n]), n


# ------------------------------------------------------------------ decode

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,C,H,Hkv,hp,window,sinks,lens,cache", [
    (1, 2, 1, 1, 16, 1, 1, (1,), "tokens"), (3, 9, 2, 1, 32, 0, 1, (0, 1, 40), "tokens"),
    (4, 133, 8, 2, 64, 128, 4, (3, 133, 134, 1000), "heads"),
    (2, 700, 12, 4, 128, 300, 4, (650, 5000), "heads"),
    (1, 3000, 16, 1, 128, 0, 0, (9001,), "tokens"), (2, 1029, 9, 3, 64, 1024, 4, (1, 100000), "tokens"),
    (2, 64, 32, 1, 64, 64, 0, (64, 65), "unaligned"), (1, 40, 11, 1, 128, 5, 30, (29,), "tokens"),
    (40, 260, 8, 8, 128, 256, 4, None, "heads"),
])
@pytest.mark.parametrize("norm,halves", [(True, False), (False, True)])
def test_decode_against_64_bits(B, C, H, Hkv, hp, window, sinks, lens, cache, norm, halves, dtype):
    gen = torch.Generator(device="cuda").manual_seed(C)
    dt = DT[dtype]
    x = rand(gen, B, H + 2 * Hkv, hp, dtype=dt)
    q, k, v = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
    gq, gk = ((1 + 0.3 * rand(gen, hp, dtype=torch.float32)).to(dt) for _ in range(2))
    if cache == "heads":
        Kc, Vc = (rand(gen, B, Hkv, C, hp, dtype=dt).transpose(1, 2) for _ in range(2))
    elif cache == "unaligned":
        Kc, Vc = (rand(gen, B, C, Hkv, hp + 1, dtype=dt)[..., 1:] for _ in range(2))
    else:
        Kc, Vc = (rand(gen, B, C, Hkv, hp, dtype=dt) for _ in range(2))
    lens = torch.randint(0, 3 * C, (B,), generator=gen, device="cuda", dtype=torch.int32) \
        if lens is None else torch.tensor(lens, device="cuda", dtype=torch.int32)
    for b in range(B):   # slots that no token was written to yet
        n = int(lens[b])
        if n < C:
            Kc[b, max(n, 0):], Vc[b, max(n, 0):] = math.nan, math.inf
    O, Kw, Vw = ref.decode(q, k, v, Kc, Vc, lens, window, sinks, gq, gk, norm, hp // 2, 10000.0,
                           1e-6, halves)
    got, ws = mosa.mosa_window_decode(q, k, v, Kc, Vc, lens, window, sinks, gamma_q=gq, gamma_k=gk,
                                      norm=norm, halves=halves)
    # (the key is rounded from an fp32 value: one that lies between two may go either way)
    assert rel(Kc, Kw) < (1e-4 if dtype == "bf16" else 1e-6) and torch.equal(
        torch.nan_to_num(Vc.double()), torch.nan_to_num(Vw))
    assert rel(got, O) < (4e-3 if dtype == "bf16" else 5e-6)


def test_decoding_token_by_token_is_the_prompt():
    """Every token of a text, one at a time through the ring, gives what the whole text does."""
    B, T, H, Hkv, hp, window, sinks = 2, 150, 4, 2, 64, 40, 3
    q, k, v, _ = inputs(B, T, T, H, Hkv, hp, "f32", seed=21)
    gen = torch.Generator(device="cuda").manual_seed(22)
    gq, gk = (1 + 0.3 * rand(gen, hp, dtype=torch.float32) for _ in range(2))
    yq, yk = mosa.mosa_qk_norm_rope(q, k, gq, gk)
    want = mosa.mosa_window_forward(yq, yk, v, window, sinks)[0]
    Kc, Vc = (torch.full((B, window + sinks, Hkv, hp), math.nan, device="cuda") for _ in range(2))
    ws = None
    for t in range(T):
        lens = torch.full((B,), t + 1, device="cuda", dtype=torch.int32)
        O, ws = mosa.mosa_window_decode(q[:, t], k[:, t], v[:, t], Kc, Vc, lens, window, sinks,
                                        gamma_q=gq, gamma_k=gk, workspace=ws)
        assert rel(O, want[:, t]) < 1e-5, t


def test_decode_in_a_cache_past_32_bits():
    """A cache whose last rows lie beyond 2^31 elements (and 2^32 bytes)."""
    B, C, Hkv, hp = 2, 70000, 128, 128
    Kc, Vc = (torch.zeros(B, C, Hkv, hp, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    assert Kc.numel() > 2 ** 31
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (rand(gen, B, Hkv, hp) for _ in range(3))
    for x in (Kc, Vc):
        x[:, -60:] = rand(gen, B, 60, Hkv, hp)
    lens = torch.full((B,), C, device="cuda", dtype=torch.int32)
    O, _ = mosa.mosa_window_decode(q, k, v, Kc, Vc, lens, 50, 0, norm=False, rotary=0)
    small = [x[:, -60:].float().clone() for x in (Kc, Vc)]
    assert torch.equal(small[0][:, -1], k.float()) and torch.equal(small[1][:, -1], v.float())
    S = torch.einsum("bhd,bthd->bht", q.double(), small[0][:, -50:].double()) / math.sqrt(hp)
    want = torch.einsum("bht,bthd->bhd", torch.softmax(S, -1), small[1][:, -50:].double())
    assert rel(O, want) < 4e-3


@pytest.mark.parametrize("hp", [64, 128])
@pytest.mark.parametrize("force", ["0", "1"])
def test_gradients_where_the_weight_lies_on_one_token(hp, force, monkeypatch):
    """A strong sink: dP - D cancels there, so D must not carry O's rounding (with it these
    gradients are off by 2e-2 and more).  The scores' gradients are rounded once, 2^-9 of each."""
    monkeypatch.setenv("MOSA_FORCE_SIMT", force)
    q, k, v, dO = inputs(2, 300, 300, 4, 2, hp, "bf16", seed=31, layout="plain")
    u = torch.randn(hp, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    q += (0.7 * u).to(q.dtype)
    k[:, :1] += (0.7 * u).to(k.dtype)
    want = ref.attention(q, k, v, 24, 1, dO=dO)
    check(run(q, k, v, dO, 24, 1), want, torch.bfloat16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T", [(1, 237), (3, 101), (1, 461), (2, 299), (1, 911), (7, 131)])
def test_norm_and_rotation_at_lengths_between(B, T, dtype):
    """Blocks take 1, 2, 4 or 8 tokens a step by the number of tokens, the last step fewer."""
    test_norm_and_rotation_against_64_bits(B, T, 5, 2, 64, None, False, "packed", dtype)


@pytest.mark.parametrize("dtype,hp", [("bf16", 64), ("bf16", 128), ("f32", 32)])
@pytest.mark.parametrize("Hkv,window,sinks", [(8, 100, 2), (4, 300, 0), (8, 1, 130)])
def test_attention_where_blocks_take_several_tiles(Hkv, window, sinks, dtype, hp):
    """More tiles than SMs, among them ones with nothing to see, and NaN in all that is hidden."""
    B, T, H = 8, 900, 8
    lens = [900, 0, 130, 899, 5, 700, 257, 128]
    q, k, v, dO = inputs(B, T, T, H, Hkv, hp, dtype, seed=window, layout="plain")
    dl = torch.tensor(lens, device="cuda", dtype=torch.int32)
    want = ref.attention(q, k, v, window, sinks, dl, dO=dO)
    for x in (q, k, v, dO):
        for b, n in enumerate(lens):
            x[b, n:] = math.nan
    got = run(q, k, v, dO, window, sinks, dl)
    check(got, want, DT[dtype])
    for b, n in enumerate(lens):
        for name in ("O", "dq", "dk", "dv"):
            assert (got[name][b, n:] == 0).all(), name


@pytest.mark.parametrize("force", ["0", "1"])
def test_attention_on_tensors_past_32_bits(force, monkeypatch):
    """Tokens 9 million elements apart, 2.7 * 10^9 from the first to the last: the same bits as packed."""
    monkeypatch.setenv("MOSA_FORCE_SIMT", force)
    q, k, v, dO = inputs(1, 300, 300, 2, 2, 64, "bf16", seed=21, layout="plain")
    want = run(q, k, v, dO, 100, 2)
    st = 9_000_000
    far = torch.empty(299 * st + 8 * 128, device="cuda", dtype=torch.bfloat16)
    at = [far.as_strided(q.shape, (0, st, 64, 1), 128 * n) for n in range(7)]
    for to, x in zip(at, (q, k, v, dO)):
        to.copy_(x)
    O, lse, ws = mosa.mosa_window_forward(*at[:3], 100, 2)
    g = mosa.mosa_window_backward(*at[:3], O, lse, at[3], ws, 100, 2,
                                  out={"dq": at[4], "dk": at[5], "dv": at[6]})
    for name, x in {"O": O, "lse": lse, **g}.items():
        assert torch.equal(x, want[name]), name


def test_the_calls_can_be_captured():
    """A training step and a decoding step in one graph, replayed on other inputs."""
    q, k, v, dO = inputs(2, 200, 200, 4, 2, 64, "bf16", seed=22, layout="plain")
    gq, gk = (torch.rand(64, device="cuda", generator=torch.Generator("cuda").manual_seed(n)).bfloat16()
              for n in (1, 2))
    lens = torch.tensor([200, 150], device="cuda", dtype=torch.int32)
    caches = [torch.zeros(2, 64, 2, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    spaces = {}

    def step():
        yq, yk = mosa.mosa_qk_norm_rope(q, k, gq, gk)
        O, lse, spaces["a"] = mosa.mosa_window_forward(yq, yk, v, 70, 4, lens=lens,
                                                       workspace=spaces.get("a"))
        g = mosa.mosa_window_backward(yq, yk, v, O, lse, dO, spaces["a"], 70, 4, lens=lens)
        gn, spaces["n"] = mosa.mosa_qk_norm_rope_backward(q, k, gq, gk, g["dq"], g["dk"],
                                                          workspace=spaces.get("n"))
        o, spaces["d"] = mosa.mosa_window_decode(q[:, 0], k[:, 0], v[:, 0], *caches, lens, 60, 4,
                                                 gamma_q=gq, gamma_k=gk, workspace=spaces.get("d"))
        return [O, lse, g["dv"], *gn.values(), o]

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for x in (q, k, v, dO):
        x.copy_(torch.randn(x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(9)))
    for c in caches:
        c.zero_()
    graph.replay()
    got = [x.clone() for x in got]
    for c in caches:
        c.zero_()
    for a, b in zip(got, step()):
        assert torch.equal(a, b)
