"""ctypes binding of the window heads (include/mosa.h): norm and rotation of queries
and keys, sliding-window attention with sinks, and the decoding step over a ring
cache.  Argument marshalling only, as in ``_binding``; tensors are [B, T, heads, hp]
with any strides whose last is 1."""
from __future__ import annotations

import ctypes
import functools

from . import _binding as _b

_i32, _i64, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class MosaStrides(ctypes.Structure):
    """mosa_strides: elements between sequences, tokens and heads."""
    _fields_ = [("b", _i64), ("t", _i64), ("h", _i64)]


class MosaQkShape(ctypes.Structure):
    """mosa_qk_shape: sizes, rotation and strides of mosa_qk_norm_rope and its backward."""
    _fields_ = ([(n, _i32) for n in ("B", "T", "H", "Hkv", "hp", "dtype", "rotary", "halves")]
                + [("theta", _f32), ("eps", _f32)]
                + [(n, MosaStrides) for n in ("q", "k", "yq", "yk", "dq", "dk")])


class MosaWindowShape(ctypes.Structure):
    """mosa_window_shape: sizes, window and strides of mosa_window_forward and its backward."""
    _fields_ = ([(n, _i32) for n in ("B", "Tq", "Tk", "H", "Hkv", "hp", "dtype", "window", "sinks")]
                + [("scale", _f32)]
                + [(n, MosaStrides) for n in ("q", "k", "v", "o", "go", "dq", "dk", "dv")])


class MosaDecodeShape(ctypes.Structure):
    """mosa_decode_shape: sizes, window, rotation and strides of mosa_window_decode."""
    _fields_ = ([(n, _i32) for n in ("B", "C", "H", "Hkv", "hp", "dtype", "window", "sinks",
                                     "norm", "rotary", "halves")]
                + [("scale", _f32), ("theta", _f32), ("eps", _f32)]
                + [(n, MosaStrides) for n in ("q", "k", "v", "o", "kc", "vc")])


def declare(L) -> None:
    """Signatures of the window heads' functions."""
    vp, sz, st = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    qk, win, dec = (ctypes.POINTER(c) for c in (MosaQkShape, MosaWindowShape, MosaDecodeShape))
    for name, args, res in (
            ("mosa_qk_norm_rope", [qk] + [vp] * 8, st),
            ("mosa_qk_norm_rope_workspace_bytes", [qk], sz),
            ("mosa_qk_norm_rope_backward", [qk] + [vp] * 11 + [vp, sz, vp], st),
            ("mosa_window_workspace_bytes", [win], sz),
            ("mosa_window_forward", [win] + [vp] * 6 + [vp, sz, vp], st),
            ("mosa_window_backward", [win] + [vp] * 10 + [vp, sz, vp], st),
            ("mosa_window_check_status", [vp, vp], st),
            ("mosa_window_decode_workspace_bytes", [dec], sz),
            ("mosa_window_decode", [dec] + [vp] * 9 + [vp, sz, vp], st)):
        f = getattr(L, name)
        f.argtypes, f.restype = args, res


def _at(t, name, dtype=None) -> int:
    """The device address of a strided tensor, checked."""
    if not isinstance(t, _b._torch_mod.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor (libmosa runs on the GPU only)")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _heads(t, name, like=None):
    """Strides of a tensor whose last dimension is contiguous, its shape ``like``'s."""
    if like is not None and t.shape != like:
        raise ValueError(f"{name} must have shape {tuple(like)}, got {tuple(t.shape)}")
    s = t.stride()
    if s[-1] != 1 and t.shape[-1] != 1:
        raise ValueError(f"{name}: the values of a head must be contiguous")
    return s[:-1]


def _new(t, out, name, shape=None, dtype=None):
    """out[name], or a new contiguous tensor of t's shape and dtype."""
    o = out.get(name) if out else None
    if o is None:
        torch = _b._torch_mod
        o = torch.empty(t.shape if shape is None else shape, dtype=dtype or t.dtype, device=t.device)
    return o


def _space(fn, ref, name, workspace, device):
    """The workspace's address and size, a new one where none is given."""
    if workspace is None:
        n = int(fn(ref))
        if n == 0:
            raise _b.MosaError(_b.MOSA_ERR_INVALID_ARG, name)
        torch = _b._torch_mod
        # zeroed: the status word of a window call's workspace is read before any call clears it
        workspace = torch.zeros(n, dtype=torch.uint8, device=device)
    return workspace


def _rank(t, name, n):
    if len(t.shape) != n:
        raise ValueError(f"{name} must have {n} dimensions, got {tuple(t.shape)}")


# ------------------------------------------------------ norm and rotation

@functools.lru_cache(maxsize=512)
def _qk_shape(sizes, theta, eps, *strides):
    s = MosaQkShape(*sizes, theta, eps, *[MosaStrides(*x) for x in strides])
    return s, ctypes.byref(s)


def _qk(q, k, gamma_q, gamma_k, positions, rotary, halves):
    torch = _b._torch()
    _rank(q, "q", 4)
    _rank(k, "k", 4)
    B, T, H, hp = q.shape
    Hkv = k.shape[2]
    if k.shape != (B, T, Hkv, hp):
        raise ValueError(f"k must be [B, T, Hkv, hp] with q's B, T and hp, got {tuple(k.shape)}")
    _b._same(q, ("k", k))
    ptrs = [None, None, None]
    for i, (n, g) in enumerate((("gamma_q", gamma_q), ("gamma_k", gamma_k))):
        if g is not None:
            _b._want(n, g, (hp,))
            ptrs[i] = _b._dev(g, n, q.dtype)
    if positions is not None:
        _b._want("positions", positions, (B, T))
        ptrs[2] = _b._dev(positions, "positions", torch.int32)
    sizes = (B, T, H, Hkv, hp, _b._dtype_code(q), hp // 2 if rotary is None else int(rotary),
             1 if halves else 0)
    return sizes, ptrs


def mosa_qk_norm_rope(q, k, gamma_q=None, gamma_k=None, positions=None, rotary=None,
                      theta: float = 10000.0, eps: float = 1e-6, halves: bool = False, out=None,
                      stream=None):
    """RMS norm per head of q [B,T,H,hp] and k [B,T,Hkv,hp], scaled by gamma [hp], then
    turned by the tokens' positions [B,T] int32 (0..T-1 by default): pairs of the first
    ``rotary`` dimensions (hp/2 by default) by t * theta^(-2p/rotary), neighbours or, with
    ``halves``, (p, p + rotary/2).  Returns (yq, yk); ``out`` may hold "q" and "k" to write
    to, q and k themselves among them."""
    sizes, (gq, gk, pos) = _qk(q, k, gamma_q, gamma_k, positions, rotary, halves)
    yq, yk = _new(q, out, "q"), _new(k, out, "k")
    sq, sk = _heads(q, "q"), _heads(k, "k")
    s, ref = _qk_shape(sizes, theta, eps, sq, sk, _heads(yq, "out q", q.shape),
                       _heads(yk, "out k", k.shape), (), ())
    dt = q.dtype
    rc = _b.load().mosa_qk_norm_rope(ref, _at(q, "q"), _at(k, "k"), gq, gk, pos,
                                     _at(yq, "out q", dt), _at(yk, "out k", dt), _b._stream(stream))
    if rc:
        _b._check(rc, "mosa_qk_norm_rope")
    return yq, yk


def mosa_qk_norm_rope_backward(q, k, gamma_q, gamma_k, dyq, dyk, positions=None, rotary=None,
                               theta: float = 10000.0, eps: float = 1e-6, halves: bool = False,
                               workspace=None, out=None, stream=None):
    """Gradients of mosa_qk_norm_rope from its inputs and the gradients of its outputs.
    Returns ({"dq", "dk", "dgamma_q", "dgamma_k"}, workspace); dgamma_* are fp32 [hp].
    ``out`` may hold any of them ("dq" and "dk" may be dyq and dyk)."""
    sizes, (gq, gk, pos) = _qk(q, k, gamma_q, gamma_k, positions, rotary, halves)
    _b._same(q, ("dyq", dyq), ("dyk", dyk))
    f32 = _b._torch_mod.float32
    g = {"dq": _new(q, out, "dq"), "dk": _new(k, out, "dk")}
    for n in ("dgamma_q", "dgamma_k"):
        g[n] = _new(q, out, n, (q.shape[3],), f32)
        _b._want(n, g[n], (q.shape[3],))
    s, ref = _qk_shape(sizes, theta, eps, _heads(q, "q"), _heads(k, "k"),
                       _heads(dyq, "dyq", q.shape), _heads(dyk, "dyk", k.shape),
                       _heads(g["dq"], "dq", q.shape), _heads(g["dk"], "dk", k.shape))
    L = _b.load()
    workspace = _space(L.mosa_qk_norm_rope_workspace_bytes, ref, "mosa_qk_norm_rope_backward",
                       workspace, q.device)
    dt = q.dtype
    rc = L.mosa_qk_norm_rope_backward(
        ref, _at(q, "q"), _at(k, "k"), gq, gk, pos, _at(dyq, "dyq"), _at(dyk, "dyk"),
        _at(g["dq"], "dq", dt), _at(g["dk"], "dk", dt), _b._dev(g["dgamma_q"], "dgamma_q", f32),
        _b._dev(g["dgamma_k"], "dgamma_k", f32), _b._dev(workspace, "workspace"),
        workspace.numel(), _b._stream(stream))
    if rc:
        _b._check(rc, "mosa_qk_norm_rope_backward")
    return g, workspace


# --------------------------------------------------------- window attention

@functools.lru_cache(maxsize=512)
def _window_shape(sizes, scale, *strides):
    s = MosaWindowShape(*sizes, scale, *[MosaStrides(*x) for x in strides])
    return s, ctypes.byref(s)


def _window(q, k, v, window, sinks, lens):
    torch = _b._torch()
    _rank(q, "q", 4)
    _rank(k, "k", 4)
    B, Tq, H, hp = q.shape
    Tk, Hkv = k.shape[1], k.shape[2]
    if k.shape != (B, Tk, Hkv, hp):
        raise ValueError(f"k must be [B, Tk, Hkv, hp] with q's B and hp, got {tuple(k.shape)}")
    _b._same(q, ("k", k), ("v", v))
    n = None
    if lens is not None:
        _b._want("lens", lens, (B,))
        n = _b._dev(lens, "lens", torch.int32)
    return (B, Tq, Tk, H, Hkv, hp, _b._dtype_code(q), int(window), int(sinks)), n


def mosa_window_forward(q, k, v, window: int, sinks: int = 0, lens=None, scale: float = 0.0,
                        workspace=None, out=None, stream=None, want_lse: bool = True):
    """Attention of q [B,Tq,H,hp], the last Tq of Tk tokens, over k and v [B,Tk,Hkv,hp]:
    each token sees those up to itself that are among the last ``window`` (0: all) or the
    first ``sinks``, below its sequence's length (lens [B] int32, Tk by default).
    scale = 0 is 1/sqrt(hp).  Returns (O, lse, workspace): O like q, lse [B,H,Tq] fp32, or
    None without ``want_lse`` (where no backward follows).  ``out`` may hold "O" and "lse"."""
    sizes, n = _window(q, k, v, window, sinks, lens)
    B, Tq, Tk, H = sizes[:4]
    f32 = _b._torch_mod.float32
    O = _new(q, out, "O")
    lse = _new(q, out, "lse", (B, H, Tq), f32) if want_lse else None
    _b._want("lse", lse, (B, H, Tq))
    s, ref = _window_shape(sizes, scale, _heads(q, "q"), _heads(k, "k"), _heads(v, "v", k.shape),
                           _heads(O, "O", q.shape))
    L = _b.load()
    workspace = _space(L.mosa_window_workspace_bytes, ref, "mosa_window_forward", workspace, q.device)
    rc = L.mosa_window_forward(ref, _at(q, "q"), _at(k, "k"), _at(v, "v"), n,
                               _at(O, "O", q.dtype),
                               None if lse is None else _b._dev(lse, "lse", f32),
                               _b._dev(workspace, "workspace"), workspace.numel(),
                               _b._stream(stream))
    if rc:
        _b._check(rc, "mosa_window_forward")
    return O, lse, workspace


def mosa_window_backward(q, k, v, O, lse, dO, workspace, window: int, sinks: int = 0, lens=None,
                         scale: float = 0.0, out=None, stream=None):
    """Gradients of mosa_window_forward, given its outputs and its workspace: a dict with dq, dk
    and dv like q, k and v, dk and dv summed over the query heads that share them.  ``out`` may
    hold any of them."""
    sizes, n = _window(q, k, v, window, sinks, lens)
    B, Tq, Tk, H = sizes[:4]
    _b._same(q, ("O", O), ("dO", dO))
    f32 = _b._torch_mod.float32
    _b._want("lse", lse, (B, H, Tq))
    g = {"dq": _new(q, out, "dq"), "dk": _new(k, out, "dk"), "dv": _new(v, out, "dv")}
    s, ref = _window_shape(sizes, scale, _heads(q, "q"), _heads(k, "k"), _heads(v, "v", k.shape),
                           _heads(O, "O", q.shape), _heads(dO, "dO", q.shape),
                           _heads(g["dq"], "dq", q.shape), _heads(g["dk"], "dk", k.shape),
                           _heads(g["dv"], "dv", k.shape))
    dt = q.dtype
    rc = _b.load().mosa_window_backward(
        ref, _at(q, "q"), _at(k, "k"), _at(v, "v"), n, _at(O, "O"), _b._dev(lse, "lse", f32),
        _at(dO, "dO"), _at(g["dq"], "dq", dt), _at(g["dk"], "dk", dt), _at(g["dv"], "dv", dt),
        _b._dev(workspace, "workspace"), workspace.numel(), _b._stream(stream))
    if rc:
        _b._check(rc, "mosa_window_backward")
    return g


def mosa_window_check_status(workspace, stream=None) -> int:
    """Synchronizes the stream, returns and clears the status code of a window workspace."""
    _b._torch()
    return int(_b.load().mosa_window_check_status(_b._dev(workspace, "workspace"),
                                                  _b._stream(stream)))


# ------------------------------------------------------------------- decode

@functools.lru_cache(maxsize=512)
def _decode_shape(sizes, scale, theta, eps, *strides):
    s = MosaDecodeShape(*sizes, scale, theta, eps, *[MosaStrides(*x) for x in strides])
    return s, ctypes.byref(s)


def _bh(t, name, like):
    """Strides (b, 0, h) of a tensor [B, heads, hp]."""
    s = _heads(t, name, like)
    return s[0], 0, s[1]


def mosa_window_decode(q, k, v, K_cache, V_cache, lens, window: int, sinks: int = 0, gamma_q=None,
                       gamma_k=None, norm: bool = True, rotary=None, theta: float = 10000.0,
                       eps: float = 1e-6, halves: bool = False, scale: float = 0.0, workspace=None,
                       out=None, stream=None):
    """One decoding step: the new tokens' q [B,H,hp] and k [B,Hkv,hp] are normalised (``norm``)
    and turned to their positions lens - 1 as in mosa_qk_norm_rope, k and v written to their
    slots of the ring caches [B,C,Hkv,hp] (token t < sinks in slot t, else sinks +
    (t - sinks) % (C - sinks)), and q attends over the visible tokens.  lens [B] int32 counts
    the new token; 0 skips a sequence.  Returns (O [B,H,hp], workspace)."""
    torch = _b._torch()
    for name, t, n in (("q", q, 3), ("k", k, 3), ("K_cache", K_cache, 4)):
        _rank(t, name, n)
    B, H, hp = q.shape
    Hkv, C = k.shape[1], K_cache.shape[1]
    kv, cache, dt = (B, Hkv, hp), (B, C, Hkv, hp), q.dtype
    _b._want("lens", lens, (B,))
    ptrs = [None, None]
    for i, (n, g) in enumerate((("gamma_q", gamma_q), ("gamma_k", gamma_k))):
        if g is not None:
            _b._want(n, g, (hp,))
            ptrs[i] = _b._dev(g, n, dt)
    O = _new(q, out, "O")
    s, ref = _decode_shape(
        (B, C, H, Hkv, hp, _b._dtype_code(q), int(window), int(sinks), 1 if norm else 0,
         hp // 2 if rotary is None else int(rotary), 1 if halves else 0), scale, theta, eps,
        _bh(q, "q", q.shape), _bh(k, "k", kv), _bh(v, "v", kv), _bh(O, "O", q.shape),
        _heads(K_cache, "K_cache", cache), _heads(V_cache, "V_cache", cache))
    L = _b.load()
    workspace = _space(L.mosa_window_decode_workspace_bytes, ref, "mosa_window_decode", workspace,
                       q.device)
    rc = L.mosa_window_decode(ref, _at(q, "q"), _at(k, "k", dt), _at(v, "v", dt), *ptrs,
                              _b._dev(lens, "lens", torch.int32), _at(K_cache, "K_cache", dt),
                              _at(V_cache, "V_cache", dt), _at(O, "O", dt),
                              _b._dev(workspace, "workspace"), workspace.numel(),
                              _b._stream(stream))
    if rc:
        _b._check(rc, "mosa_window_decode")
    return O, workspace
