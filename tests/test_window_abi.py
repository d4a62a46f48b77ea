"""The window heads' C ABI and binding without a GPU: what they refuse, before anything is
launched and before any CUDA call."""
import ctypes

import pytest
import torch

from paper_2505_00315_gb300 import _binding as B
from paper_2505_00315_gb300 import _window as W

FAKE = ctypes.c_void_p(0x100000)   # never dereferenced: validation fails first
OFF = ctypes.c_void_p(0x100001)    # not at a multiple of any element's size
INV, UNS, WS = B.MOSA_ERR_INVALID_ARG, B.MOSA_ERR_UNSUPPORTED, B.MOSA_ERR_WORKSPACE


def dense(T, H, hp):
    return W.MosaStrides(T * H * hp, H * hp, hp)


def qk(**kw):
    f = dict(B=2, T=10, H=4, Hkv=2, hp=64, dtype=B.MOSA_BF16, rotary=32, halves=0, theta=1e4,
             eps=1e-6)
    f.update({k: v for k, v in kw.items() if k in f})
    s = W.MosaQkShape(**f)
    for n, h in (("q", f["H"]), ("k", f["Hkv"]), ("yq", f["H"]), ("yk", f["Hkv"]), ("dq", f["H"]),
                 ("dk", f["Hkv"])):
        setattr(s, n, kw.get("s_" + n, dense(f["T"], h, f["hp"])))
    return s


def window(**kw):
    f = dict(B=2, Tq=10, Tk=10, H=4, Hkv=2, hp=64, dtype=B.MOSA_BF16, window=4, sinks=1, scale=0.0)
    f.update({k: v for k, v in kw.items() if k in f})
    s = W.MosaWindowShape(**f)
    for n, t, h in (("q", "Tq", "H"), ("k", "Tk", "Hkv"), ("v", "Tk", "Hkv"), ("o", "Tq", "H"),
                    ("go", "Tq", "H"), ("dq", "Tq", "H"), ("dk", "Tk", "Hkv"), ("dv", "Tk", "Hkv")):
        setattr(s, n, kw.get("s_" + n, dense(f[t], f[h], f["hp"])))
    return s


def decode(**kw):
    f = dict(B=2, C=20, H=4, Hkv=2, hp=64, dtype=B.MOSA_BF16, window=16, sinks=4, norm=1, rotary=32,
             halves=0, scale=0.0, theta=1e4, eps=1e-6)
    f.update({k: v for k, v in kw.items() if k in f})
    s = W.MosaDecodeShape(**f)
    for n, t, h in (("q", 1, "H"), ("k", 1, "Hkv"), ("v", 1, "Hkv"), ("o", 1, "H"),
                    ("kc", f["C"], "Hkv"), ("vc", f["C"], "Hkv")):
        setattr(s, n, kw.get("s_" + n, dense(t, f[h], f["hp"])))
    return s


def norm_fwd(s, ptrs=None):
    return B.load().mosa_qk_norm_rope(ctypes.byref(s), *(ptrs or [FAKE] * 7), None)


def norm_bwd(s, ptrs=None, ws=FAKE, n=1 << 40):
    return B.load().mosa_qk_norm_rope_backward(ctypes.byref(s), *(ptrs or [FAKE] * 11), ws, n, None)


def win_fwd(s, ptrs=None, ws=FAKE, n=1 << 40):
    return B.load().mosa_window_forward(ctypes.byref(s), *(ptrs or [FAKE] * 6), ws, n, None)


def win_bwd(s, ptrs=None, ws=FAKE, n=1 << 40):
    return B.load().mosa_window_backward(ctypes.byref(s), *(ptrs or [FAKE] * 10), ws, n, None)


def win_dec(s, ptrs=None, ws=FAKE, n=1 << 40):
    return B.load().mosa_window_decode(ctypes.byref(s), *(ptrs or [FAKE] * 9), ws, n, None)


S = W.MosaStrides


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), INV), (dict(T=0), INV), (dict(H=-1), INV), (dict(dtype=5), INV), (dict(hp=48), UNS),
    (dict(rotary=3), INV), (dict(rotary=66), INV), (dict(rotary=-2), INV), (dict(halves=2), INV),
    (dict(halves=1, rotary=20), UNS), (dict(theta=0.5), INV), (dict(theta=float("inf")), INV),
    (dict(eps=-1.0), INV), (dict(eps=float("nan")), INV), (dict(B=70000), UNS), (dict(T=1 << 30), UNS),
    (dict(B=60000, T=60000), UNS), (dict(s_q=S(-1, 64, 64)), INV), (dict(s_yq=S(0, 256, 64)), INV),
    (dict(s_yk=S(1280, 32, 64)), INV), (dict(s_q=S(1 << 61, 64, 64)), INV),
])
def test_norm_refuses(kw, code):
    assert norm_fwd(qk(**kw)) == code


def test_norm_refuses_pointers_and_workspaces():
    L = B.load()
    for i in (0, 1, 5, 6):       # q, k, yq, yk
        for bad in (None, OFF):
            p = [FAKE] * 7
            p[i] = bad
            assert norm_fwd(qk(), p) == INV, i
    for i in (2, 3, 4):          # gammas and positions may be NULL, not misplaced
        p = [FAKE] * 7
        p[i] = OFF
        assert norm_fwd(qk(), p) == INV, i
    for i in (0, 1, 5, 6, 7, 8):
        p = [FAKE] * 11
        p[i] = None
        assert norm_bwd(qk(), p) == INV, i
    assert norm_bwd(qk(s_dq=S(0, 0, 0))) == INV
    need = L.mosa_qk_norm_rope_workspace_bytes(ctypes.byref(qk()))
    assert need > 0
    assert norm_bwd(qk(), ws=None) == WS
    assert norm_bwd(qk(), ws=ctypes.c_void_p(0x100010)) == WS
    assert norm_bwd(qk(), n=need - 1) == WS
    assert L.mosa_qk_norm_rope(None, *[FAKE] * 7, None) == INV


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), INV), (dict(Tq=0), INV), (dict(Tq=11), INV), (dict(H=3), INV), (dict(Hkv=0), INV),
    (dict(window=-1), INV), (dict(sinks=-1), INV), (dict(scale=-0.1), INV),
    (dict(scale=float("inf")), INV), (dict(scale=float("nan")), INV), (dict(hp=80), UNS),
    (dict(dtype=-1), INV), (dict(H=70000, Hkv=70000), UNS), (dict(Tk=1 << 30), UNS),
    (dict(s_k=S(1, -1, 1)), INV), (dict(s_o=S(2560, 0, 64)), INV),
])
def test_attention_refuses(kw, code):
    s = window(**kw)
    assert win_fwd(s) == code
    assert win_bwd(s) == code or "s_o" in kw
    if "s_o" not in kw:
        assert B.load().mosa_window_workspace_bytes(ctypes.byref(s)) == 0


def test_attention_refuses_pointers_and_workspaces():
    L = B.load()
    for i in (0, 1, 2, 4):
        for bad in (None, OFF):
            p = [FAKE] * 6
            p[i] = bad
            assert win_fwd(window(), p) == INV, i
    for i in (0, 1, 2, 4, 5, 6, 7, 8, 9):
        for bad in (None, OFF):
            p = [FAKE] * 10
            p[i] = bad
            assert win_bwd(window(), p) == INV, i
    for n in ("s_dq", "s_dk", "s_dv"):
        assert win_bwd(window(**{n: S(0, 64, 64)})) == INV
    need = L.mosa_window_workspace_bytes(ctypes.byref(window()))
    for call in (win_fwd, win_bwd):
        assert call(window(), ws=None) == WS
        assert call(window(), ws=ctypes.c_void_p(0x100080)) == WS
        assert call(window(), n=need - 1) == WS
    assert L.mosa_window_check_status(None, None) == WS
    assert L.mosa_window_check_status(ctypes.c_void_p(0x100080), None) == WS


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), INV), (dict(C=4), INV), (dict(C=0, sinks=0), INV), (dict(window=-2), INV),
    (dict(sinks=-1), INV), (dict(norm=2), INV), (dict(rotary=65), INV), (dict(H=5), INV),
    (dict(halves=1, rotary=36), UNS), (dict(C=1 << 30), UNS), (dict(hp=8), UNS),
    (dict(scale=-1.0), INV), (dict(s_kc=S(0, 128, 64)), INV), (dict(s_vc=S(2560, 128, 0)), INV),
])
def test_decode_refuses(kw, code):
    assert win_dec(decode(**kw)) == code


def test_decode_refuses_pointers_and_workspaces():
    for i in (0, 1, 2, 5, 6, 7, 8):
        for bad in (None, OFF):
            p = [FAKE] * 9
            p[i] = bad
            assert win_dec(decode(), p) == INV, i
    need = B.load().mosa_window_decode_workspace_bytes(ctypes.byref(decode()))
    assert need > 0 and win_dec(decode(), ws=None) == WS and win_dec(decode(), n=need - 1) == WS


def test_binding_refuses():
    """Shapes, types and devices, before the library is called."""
    q, k = torch.zeros(2, 8, 4, 64), torch.zeros(2, 8, 2, 64)
    with pytest.raises(ValueError, match="CUDA tensor"):
        W.mosa_window_forward(q, k, k, 4)
    with pytest.raises(ValueError, match="dimensions"):
        W.mosa_window_forward(q[0], k, k, 4)
    with pytest.raises(ValueError, match="k must be"):
        W.mosa_window_forward(q, k[:1], k, 4)
    with pytest.raises(ValueError, match="v must have shape"):
        W.mosa_window_forward(q, k, k[:, :4], 4)
    with pytest.raises(TypeError, match="storage dtype"):
        W.mosa_window_forward(q, k.bfloat16(), k, 4)
    with pytest.raises(TypeError, match="unsupported"):
        W.mosa_window_forward(q.half(), k.half(), k.half(), 4)
    with pytest.raises(ValueError, match="contiguous"):
        W.mosa_window_forward(q.transpose(2, 3).contiguous().transpose(2, 3), k, k, 4)
    with pytest.raises(ValueError, match="lens"):
        W.mosa_window_forward(q, k, k, 4, lens=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="O must have shape"):
        W.mosa_window_forward(q, k, k, 4, out={"O": k})
    with pytest.raises(TypeError):
        W.mosa_window_forward(q, k, k, 4.5)
    with pytest.raises(ValueError, match="32 bits"):
        W.mosa_window_forward(q, k, k, 2**32 + 4)
    with pytest.raises(ValueError, match="gamma_q"):
        W.mosa_qk_norm_rope(q, k, torch.zeros(32))
    with pytest.raises(ValueError, match="positions"):
        W.mosa_qk_norm_rope(q, k, positions=torch.zeros(8, dtype=torch.int32))
    with pytest.raises(ValueError, match="dyk must have shape"):
        W.mosa_qk_norm_rope_backward(q, k, None, None, q, q)
    with pytest.raises(ValueError, match="V_cache"):
        W.mosa_window_decode(q[:, 0], k[:, 0], k[:, 0], k, k[:, :4], torch.ones(2), 4)
    with pytest.raises(ValueError, match="lens"):
        W.mosa_window_decode(q[:, 0], k[:, 0], k[:, 0], k, k, torch.ones(3), 4)
