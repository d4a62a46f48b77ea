"""ctypes binding of the window heads (include/mosa.h): norm and rotation of queries
and keys, sliding-window attention with sinks, and the decoding step over a ring
cache.  Argument marshalling only, as in ``_binding``; tensors are [B, T, heads, hp]
with any strides whose last is 1."""
from __future__ import annotations

import ctypes
import operator

from . import _binding as _b

_i32, _i64, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float

#: The workspace of a forward that no backward follows: the status word, at its alignment.
STATUS_BYTES = 256


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


# A call's host time is mostly this marshalling, so what depends on shapes, strides and types alone
# (the checks and the library's struct) is done once for each set of them and kept as a plan; a
# later call builds the key, looks it up and passes addresses, with as few Python calls as that takes
# (mosa_window_forward with its results' allocation 20.6 -> 15.1 us).
_plans: dict = {}


def _keep(key, plan):
    if len(_plans) >= 512:
        _plans.clear()
    _plans[key] = plan
    return plan


def _sig(t):
    """Shape, strides and type of an optional tensor, as part of a key."""
    return None if t is None else (t.shape, t.stride(), t.dtype)


def _half(rotary, hp):
    """The rotated dimensions: half a head by default."""
    return hp // 2 if rotary is None else _int(rotary, "rotary")


def _bad(*named):
    """Says which argument is not a tensor on the GPU."""
    for name, t in named:
        if t is not None and not isinstance(t, _b._torch().Tensor):
            raise TypeError(f"{name} must be a torch.Tensor")
    for name, t in named:
        if t is not None and not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor (libmosa runs on the GPU only)")
    raise TypeError("a tensor argument is missing")


def _heads(t, name, like=None, dtype=None):
    """Strides (but the last, 1) of a tensor of heads, its shape ``like`` and type checked."""
    if like is not None and t.shape != like:
        raise ValueError(f"{name} must have shape {tuple(like)}, got {tuple(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have the storage dtype {dtype}, got {t.dtype}")
    s = t.stride()
    if s[-1] != 1 and t.shape[-1] != 1:
        raise ValueError(f"{name}: the values of a head must be contiguous")
    return MosaStrides(*s[:-1])


def _packed(shape):
    """Strides of a new contiguous tensor of that shape."""
    return MosaStrides(shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3])


def _out(t, name, like, dtype):
    """Strides of a result: a given tensor's, or those of the one to be made."""
    return _packed(like) if t is None else _heads(t, name, like, dtype)


def _new(t):
    """A new contiguous tensor like t (empty_like takes 0.5 us less than empty)."""
    torch = _b._torch_mod
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _vector(t, name, shape, dtype):
    """A contiguous tensor of exactly that shape and type, or None."""
    if t is not None:
        _b._want(name, t, shape)
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _rank(t, name, n):
    if len(t.shape) != n:
        raise ValueError(f"{name} must have {n} dimensions, got {tuple(t.shape)}")


# What goes into a key is a plain number, taken from the argument at each call where that is none: an
# object that stands for one (a tensor, say) may hold another the next time.

def _int(x, name):
    """A Python or NumPy integer, or a tensor of one, that the library's 32-bit field holds."""
    x = operator.index(x)
    if not -2**31 <= x < 2**31:
        raise ValueError(f"{name} does not fit 32 bits: {x}")
    return x


def _float(x):
    """The value of a number, as the library's 32-bit field holds it if it is no Python float."""
    return x if type(x) is float else _f32(x).value


def _rotation(rotary, theta, eps, halves):
    """The rotation's and the norm's arguments as plain numbers (rotary None: half a head)."""
    return (None if rotary is None else _int(rotary, "rotary"), _float(theta), _float(eps), bool(halves))


def _on(stream):
    """The context in which a call for ``stream`` runs: with it the current one, so that what the call
    allocates (and zeroes) is that stream's too."""
    cuda = _b._torch().cuda
    return cuda.stream(stream if isinstance(stream, cuda.Stream) else cuda.ExternalStream(stream.cuda_stream))


def _space(workspace, need, device, status=False):
    """The given workspace, or a new one (empty where the library refuses the sizes, as it will say).  With
    ``status`` its first word is zeroed, which is read before any call clears it; the rest may hold anything
    (zeroing all of it was 68 MB a call at B4 T4096, 16 heads of 128)."""
    if workspace is not None:
        if not (workspace.is_cuda and workspace.dtype is _b._torch_mod.uint8 and workspace.is_contiguous()):
            _b._dev(workspace, "workspace", _b._torch_mod.uint8)   # says what is wrong
        return workspace
    workspace = _b._torch_mod.empty(need, dtype=_b._torch_mod.uint8, device=device)
    if status:
        workspace[:4].zero_()
    return workspace


# ------------------------------------------------------ norm and rotation

def _qk_plan(q, k, gamma_q, gamma_k, positions, rotary, theta, eps, halves, yq, yk, dq=None, dk=None,
             dgamma_q=None, dgamma_k=None, backward=False):
    torch = _b._torch_mod
    _rank(q, "q", 4)
    _rank(k, "k", 4)
    B, T, H, hp = q.shape
    Hkv = k.shape[2]
    if k.shape != (B, T, Hkv, hp):
        raise ValueError(f"k must be [B, T, Hkv, hp] with q's B, T and hp, got {tuple(k.shape)}")
    dt = q.dtype
    _vector(gamma_q, "gamma_q", (hp,), dt)
    _vector(gamma_k, "gamma_k", (hp,), dt)
    _vector(positions, "positions", (B, T), torch.int32)
    _vector(dgamma_q, "dgamma_q", (hp,), torch.float32)
    _vector(dgamma_k, "dgamma_k", (hp,), torch.float32)
    y = ("dyq", "dyk") if backward else ("out q", "out k")
    s = MosaQkShape(B, T, H, Hkv, hp, _b._dtype_code(q), _half(rotary, hp), 1 if halves else 0,
                    theta, eps, _heads(q, "q"), _heads(k, "k", None, dt), _out(yq, y[0], q.shape, dt),
                    _out(yk, y[1], k.shape, dt))
    need = 0
    if backward:
        s.dq, s.dk = _out(dq, "dq", q.shape, dt), _out(dk, "dk", k.shape, dt)
        need = int(_b.load().mosa_qk_norm_rope_workspace_bytes(ctypes.byref(s)))
    return ctypes.byref(s), need, s


def mosa_qk_norm_rope(q, k, gamma_q=None, gamma_k=None, positions=None, rotary=None,
                      theta: float = 10000.0, eps: float = 1e-6, halves: bool = False, out=None,
                      stream=None):
    """RMS norm per head of q [B,T,H,hp] and k [B,T,Hkv,hp], scaled by gamma [hp], then
    turned by the tokens' positions [B,T] int32 (0..T-1 by default): pairs of the first
    ``rotary`` dimensions (hp/2 by default) by t * theta^(-2p/rotary), neighbours or, with
    ``halves``, (p, p + rotary/2).  Returns (yq, yk); ``out`` may hold "q" and "k" to write
    to, q and k themselves among them."""
    if stream is not None:
        with _on(stream):
            return mosa_qk_norm_rope(q, k, gamma_q, gamma_k, positions, rotary, theta, eps, halves, out)
    torch = _b._torch()
    yq, yk = (out.get("q"), out.get("k")) if out else (None, None)
    if not (type(theta) is type(eps) is float and type(halves) is bool and (rotary is None or type(rotary) is int)):
        rotary, theta, eps, halves = _rotation(rotary, theta, eps, halves)
    try:
        key = (1, q.shape, q.stride(), q.dtype, k.shape, k.stride(), k.dtype, rotary, theta, eps, halves,
               _sig(gamma_q), _sig(gamma_k), _sig(positions), _sig(yq), _sig(yk))
    except AttributeError:
        _bad(("q", q), ("k", k), ("gamma_q", gamma_q), ("gamma_k", gamma_k), ("positions", positions),
             ("out q", yq), ("out k", yk))
    plan = _plans.get(key) or _keep(key, _qk_plan(q, k, gamma_q, gamma_k, positions, rotary, theta, eps,
                                                  halves, yq, yk))
    if yq is None:
        yq = _new(q)
    if yk is None:
        yk = _new(k)
    if not (q.is_cuda and k.is_cuda and yq.is_cuda and yk.is_cuda
            and (gamma_q is None or gamma_q.is_cuda) and (gamma_k is None or gamma_k.is_cuda)
            and (positions is None or positions.is_cuda)):
        _bad(("q", q), ("k", k), ("gamma_q", gamma_q), ("gamma_k", gamma_k), ("positions", positions),
             ("out q", yq), ("out k", yk))
    rc = _b.load().mosa_qk_norm_rope(
        plan[0], q.data_ptr(), k.data_ptr(), None if gamma_q is None else gamma_q.data_ptr(),
        None if gamma_k is None else gamma_k.data_ptr(),
        None if positions is None else positions.data_ptr(), yq.data_ptr(), yk.data_ptr(),
        _b._stream(None))
    if rc:
        _b._check(rc, "mosa_qk_norm_rope")
    return yq, yk


def mosa_qk_norm_rope_backward(q, k, gamma_q, gamma_k, dyq, dyk, positions=None, rotary=None,
                               theta: float = 10000.0, eps: float = 1e-6, halves: bool = False,
                               workspace=None, out=None, stream=None):
    """Gradients of mosa_qk_norm_rope from its inputs and the gradients of its outputs.
    Returns ({"dq", "dk", "dgamma_q", "dgamma_k"}, workspace); dgamma_* are fp32 [hp].
    ``out`` may hold any of them ("dq" and "dk" may be dyq and dyk)."""
    if stream is not None:
        with _on(stream):
            return mosa_qk_norm_rope_backward(q, k, gamma_q, gamma_k, dyq, dyk, positions, rotary, theta, eps, halves,
                                              workspace, out)
    torch = _b._torch()
    dq, dk, dgq, dgk = ((out.get("dq"), out.get("dk"), out.get("dgamma_q"), out.get("dgamma_k"))
                        if out else (None, None, None, None))
    if not (type(theta) is type(eps) is float and type(halves) is bool and (rotary is None or type(rotary) is int)):
        rotary, theta, eps, halves = _rotation(rotary, theta, eps, halves)
    try:
        key = (2, q.shape, q.stride(), q.dtype, k.shape, k.stride(), k.dtype, rotary, theta, eps, halves,
               _sig(gamma_q), _sig(gamma_k), _sig(positions), dyq.shape, dyq.stride(), dyq.dtype,
               dyk.shape, dyk.stride(), dyk.dtype, (_sig(dq), _sig(dk), _sig(dgq), _sig(dgk)) if out else None)
    except AttributeError:
        _bad(("q", q), ("k", k), ("gamma_q", gamma_q), ("gamma_k", gamma_k), ("dyq", dyq), ("dyk", dyk),
             ("positions", positions), ("dq", dq), ("dk", dk), ("dgamma_q", dgq), ("dgamma_k", dgk))
    plan = _plans.get(key) or _keep(key, _qk_plan(q, k, gamma_q, gamma_k, positions, rotary, theta, eps,
                                                  halves, dyq, dyk, dq, dk, dgq, dgk, True))
    dev, f32 = q.device, torch.float32
    if dq is None:
        dq = _new(q)
    if dk is None:
        dk = _new(k)
    if dgq is None:
        dgq = torch.empty(q.shape[3], dtype=f32, device=dev)
    if dgk is None:
        dgk = torch.empty(q.shape[3], dtype=f32, device=dev)
    if not (q.is_cuda and k.is_cuda and dyq.is_cuda and dyk.is_cuda and dq.is_cuda and dk.is_cuda
            and dgq.is_cuda and dgk.is_cuda and (gamma_q is None or gamma_q.is_cuda)
            and (gamma_k is None or gamma_k.is_cuda) and (positions is None or positions.is_cuda)):
        _bad(("q", q), ("k", k), ("gamma_q", gamma_q), ("gamma_k", gamma_k), ("dyq", dyq), ("dyk", dyk),
             ("positions", positions), ("dq", dq), ("dk", dk), ("dgamma_q", dgq), ("dgamma_k", dgk))
    workspace = _space(workspace, plan[1], dev)
    rc = _b.load().mosa_qk_norm_rope_backward(
        plan[0], q.data_ptr(), k.data_ptr(), None if gamma_q is None else gamma_q.data_ptr(),
        None if gamma_k is None else gamma_k.data_ptr(),
        None if positions is None else positions.data_ptr(), dyq.data_ptr(), dyk.data_ptr(),
        dq.data_ptr(), dk.data_ptr(), dgq.data_ptr(), dgk.data_ptr(), workspace.data_ptr(),
        workspace.numel(), _b._stream(None))
    if rc:
        _b._check(rc, "mosa_qk_norm_rope_backward")
    return {"dq": dq, "dk": dk, "dgamma_q": dgq, "dgamma_k": dgk}, workspace


# --------------------------------------------------------- window attention

def _window_plan(q, k, v, O, lse, lens, window, sinks, scale, dO=None, dq=None, dk=None, dv=None):
    torch = _b._torch_mod
    _rank(q, "q", 4)
    _rank(k, "k", 4)
    B, Tq, H, hp = q.shape
    Tk, Hkv = k.shape[1], k.shape[2]
    if k.shape != (B, Tk, Hkv, hp):
        raise ValueError(f"k must be [B, Tk, Hkv, hp] with q's B and hp, got {tuple(k.shape)}")
    dt = q.dtype
    _vector(lens, "lens", (B,), torch.int32)
    _vector(lse, "lse", (B, H, Tq), torch.float32)
    s = MosaWindowShape(B, Tq, Tk, H, Hkv, hp, _b._dtype_code(q), _int(window, "window"),
                        _int(sinks, "sinks"), scale, _heads(q, "q"), _heads(k, "k", None, dt),
                        _heads(v, "v", k.shape, dt), _out(O, "O", q.shape, dt))
    if dO is not None:
        s.go = _heads(dO, "dO", q.shape, dt)
        s.dq, s.dk, s.dv = (_out(dq, "dq", q.shape, dt), _out(dk, "dk", k.shape, dt),
                            _out(dv, "dv", k.shape, dt))
    return ctypes.byref(s), int(_b.load().mosa_window_workspace_bytes(ctypes.byref(s))), s


def mosa_window_forward(q, k, v, window: int, sinks: int = 0, lens=None, scale: float = 0.0,
                        workspace=None, out=None, stream=None, want_lse: bool = True):
    """Attention of q [B,Tq,H,hp], the last Tq of Tk tokens, over k and v [B,Tk,Hkv,hp]:
    each token sees those up to itself that are among the last ``window`` (0: all) or the
    first ``sinks``, below its sequence's length (lens [B] int32, Tk by default).
    scale = 0 is 1/sqrt(hp).  Returns (O, lse, workspace): O like q, lse [B,H,Tq] fp32, or
    None without ``want_lse`` (where no backward follows).  ``out`` may hold "O" and "lse"."""
    if stream is not None:
        with _on(stream):
            return mosa_window_forward(q, k, v, window, sinks, lens, scale, workspace, out, None, want_lse)
    torch = _b._torch()
    O, lse = (out.get("O"), out.get("lse")) if out else (None, None)
    if not (type(window) is type(sinks) is int and type(scale) is float):
        window, sinks, scale = _int(window, "window"), _int(sinks, "sinks"), _float(scale)
    try:
        qs = q.shape
        key = (3, qs, q.stride(), q.dtype, k.shape, k.stride(), k.dtype, v.shape, v.stride(), v.dtype,
               window, sinks, scale, _sig(lens), (_sig(O), _sig(lse)) if out else None)
    except AttributeError:
        _bad(("q", q), ("k", k), ("v", v), ("lens", lens), ("O", O), ("lse", lse))
    plan = _plans.get(key) or _keep(key, _window_plan(q, k, v, O, lse, lens, window, sinks, scale))
    dev = q.device
    if O is None:
        O = _new(q)
    if not want_lse:
        lse = None
    elif lse is None:
        lse = torch.empty((qs[0], qs[2], qs[1]), dtype=torch.float32, device=dev)
    if not (q.is_cuda and k.is_cuda and v.is_cuda and O.is_cuda and (lse is None or lse.is_cuda)
            and (lens is None or lens.is_cuda)):
        _bad(("q", q), ("k", k), ("v", v), ("lens", lens), ("O", O), ("lse", lse))
    workspace = _space(workspace, plan[1] if want_lse else min(plan[1], STATUS_BYTES), dev, True)
    rc = _b.load().mosa_window_forward(
        plan[0], q.data_ptr(), k.data_ptr(), v.data_ptr(), None if lens is None else lens.data_ptr(),
        O.data_ptr(), None if lse is None else lse.data_ptr(), workspace.data_ptr(),
        workspace.numel(), _b._stream(None))
    if rc:
        _b._check(rc, "mosa_window_forward")
    return O, lse, workspace


def mosa_window_backward(q, k, v, O, lse, dO, workspace, window: int, sinks: int = 0, lens=None,
                         scale: float = 0.0, out=None, stream=None):
    """Gradients of mosa_window_forward, given its outputs and its workspace: a dict with dq, dk
    and dv like q, k and v, dk and dv summed over the query heads that share them.  ``out`` may
    hold any of them."""
    if stream is not None:
        with _on(stream):
            return mosa_window_backward(q, k, v, O, lse, dO, workspace, window, sinks, lens, scale, out)
    torch = _b._torch()
    dq, dk, dv = (out.get("dq"), out.get("dk"), out.get("dv")) if out else (None, None, None)
    if not (type(window) is type(sinks) is int and type(scale) is float):
        window, sinks, scale = _int(window, "window"), _int(sinks, "sinks"), _float(scale)
    try:
        key = (4, q.shape, q.stride(), q.dtype, k.shape, k.stride(), k.dtype, v.shape, v.stride(), v.dtype,
               O.shape, O.stride(), O.dtype, lse.shape, lse.stride(), lse.dtype, dO.shape, dO.stride(),
               dO.dtype, window, sinks, scale, _sig(lens), (_sig(dq), _sig(dk), _sig(dv)) if out else None)
    except AttributeError:
        _bad(("q", q), ("k", k), ("v", v), ("O", O), ("lse", lse), ("dO", dO), ("lens", lens), ("dq", dq),
             ("dk", dk), ("dv", dv))
    plan = _plans.get(key) or _keep(key, _window_plan(q, k, v, O, lse, lens, window, sinks, scale, dO, dq,
                                                      dk, dv))
    dev = q.device
    if dq is None:
        dq = _new(q)
    if dk is None:
        dk = _new(k)
    if dv is None:
        dv = _new(k)
    if not (q.is_cuda and k.is_cuda and v.is_cuda and O.is_cuda and lse.is_cuda and dO.is_cuda
            and dq.is_cuda and dk.is_cuda and dv.is_cuda and (lens is None or lens.is_cuda)):
        _bad(("q", q), ("k", k), ("v", v), ("O", O), ("lse", lse), ("dO", dO), ("lens", lens), ("dq", dq),
             ("dk", dk), ("dv", dv))
    if workspace is None:
        raise TypeError("workspace must be the forward's")
    _space(workspace, 0, dev)
    rc = _b.load().mosa_window_backward(
        plan[0], q.data_ptr(), k.data_ptr(), v.data_ptr(), None if lens is None else lens.data_ptr(),
        O.data_ptr(), lse.data_ptr(), dO.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
        workspace.data_ptr(), workspace.numel(), _b._stream(None))
    if rc:
        _b._check(rc, "mosa_window_backward")
    return {"dq": dq, "dk": dk, "dv": dv}


def mosa_window_check_status(workspace, stream=None) -> int:
    """Synchronizes the stream, returns and clears the status code of a window workspace."""
    _b._torch()
    return int(_b.load().mosa_window_check_status(_b._dev(workspace, "workspace"),
                                                  _b._stream(stream)))


# ------------------------------------------------------------------- decode

def _bh(t, name, like, dtype):
    """Strides (b, -, h) of a tensor [B, heads, hp]."""
    if t is None:
        return MosaStrides(like[1] * like[2], 0, like[2])
    if t.shape != like:
        raise ValueError(f"{name} must have shape {tuple(like)}, got {tuple(t.shape)}")
    s = _heads(t[:, None], name, None, dtype)
    return MosaStrides(s.b, 0, s.h)


def _decode_plan(q, k, v, Kc, Vc, lens, O, gamma_q, gamma_k, window, sinks, norm, rotary, theta, eps,
                 halves, scale):
    for name, t, n in (("q", q, 3), ("k", k, 3), ("K_cache", Kc, 4)):
        _rank(t, name, n)
    B, H, hp = q.shape
    Hkv, C = k.shape[1], Kc.shape[1]
    kv, cache, dt = (B, Hkv, hp), (B, C, Hkv, hp), q.dtype
    _b._want("lens", lens, (B,))
    _vector(gamma_q, "gamma_q", (hp,), dt)
    _vector(gamma_k, "gamma_k", (hp,), dt)
    strides = (_bh(q, "q", q.shape, dt), _bh(k, "k", kv, dt), _bh(v, "v", kv, dt),
               _bh(O, "O", q.shape, dt), _heads(Kc, "K_cache", cache, dt),
               _heads(Vc, "V_cache", cache, dt))
    _vector(lens, "lens", (B,), _b._torch_mod.int32)
    s = MosaDecodeShape(B, C, H, Hkv, hp, _b._dtype_code(q), _int(window, "window"), _int(sinks, "sinks"),
                        1 if norm else 0, _half(rotary, hp), 1 if halves else 0, scale, theta, eps, *strides)
    return ctypes.byref(s), int(_b.load().mosa_window_decode_workspace_bytes(ctypes.byref(s))), s


def mosa_window_decode(q, k, v, K_cache, V_cache, lens, window: int, sinks: int = 0, gamma_q=None,
                       gamma_k=None, norm: bool = True, rotary=None, theta: float = 10000.0,
                       eps: float = 1e-6, halves: bool = False, scale: float = 0.0, workspace=None,
                       out=None, stream=None):
    """One decoding step: the new tokens' q [B,H,hp] and k [B,Hkv,hp] are normalised (``norm``)
    and turned to their positions lens - 1 as in mosa_qk_norm_rope, k and v written to their
    slots of the ring caches [B,C,Hkv,hp] (token t < sinks in slot t, else sinks +
    (t - sinks) % (C - sinks)), and q attends over the visible tokens.  lens [B] int32 counts
    the new token; 0 skips a sequence.  Returns (O [B,H,hp], workspace)."""
    if stream is not None:
        with _on(stream):
            return mosa_window_decode(q, k, v, K_cache, V_cache, lens, window, sinks, gamma_q, gamma_k, norm, rotary,
                                      theta, eps, halves, scale, workspace, out)
    torch = _b._torch()
    O = out.get("O") if out else None
    if not (type(window) is type(sinks) is int and type(scale) is float and type(norm) is bool):
        window, sinks, scale, norm = _int(window, "window"), _int(sinks, "sinks"), _float(scale), bool(norm)
    if not (type(theta) is type(eps) is float and type(halves) is bool and (rotary is None or type(rotary) is int)):
        rotary, theta, eps, halves = _rotation(rotary, theta, eps, halves)
    try:
        key = (5, q.shape, q.stride(), q.dtype, k.shape, k.stride(), k.dtype, v.shape, v.stride(), v.dtype,
               K_cache.shape, K_cache.stride(), K_cache.dtype, V_cache.shape, V_cache.stride(),
               V_cache.dtype, lens.shape, lens.stride(), lens.dtype, _sig(O), _sig(gamma_q),
               _sig(gamma_k), window, sinks, norm, rotary, theta, eps, halves, scale)
    except AttributeError:
        _bad(("q", q), ("k", k), ("v", v), ("K_cache", K_cache), ("V_cache", V_cache), ("lens", lens),
             ("O", O), ("gamma_q", gamma_q), ("gamma_k", gamma_k))
    plan = _plans.get(key) or _keep(key, _decode_plan(q, k, v, K_cache, V_cache, lens, O, gamma_q, gamma_k,
                                                      window, sinks, norm, rotary, theta, eps, halves,
                                                      scale))
    if O is None:
        O = _new(q)
    if not (q.is_cuda and k.is_cuda and v.is_cuda and K_cache.is_cuda and V_cache.is_cuda and lens.is_cuda
            and O.is_cuda and (gamma_q is None or gamma_q.is_cuda)
            and (gamma_k is None or gamma_k.is_cuda)):
        _bad(("q", q), ("k", k), ("v", v), ("K_cache", K_cache), ("V_cache", V_cache), ("lens", lens),
             ("O", O), ("gamma_q", gamma_q), ("gamma_k", gamma_k))
    workspace = _space(workspace, plan[1], q.device)
    rc = _b.load().mosa_window_decode(
        plan[0], q.data_ptr(), k.data_ptr(), v.data_ptr(),
        None if gamma_q is None else gamma_q.data_ptr(),
        None if gamma_k is None else gamma_k.data_ptr(), lens.data_ptr(), K_cache.data_ptr(),
        V_cache.data_ptr(), O.data_ptr(), workspace.data_ptr(), workspace.numel(), _b._stream(None))
    if rc:
        _b._check(rc, "mosa_window_decode")
    return O, workspace
