"""ctypes binding of the block operators (include/mosa.h): the residual step between two blocks,
dropout, and log probabilities of given tokens.  Argument marshalling only, as in
``_binding``; tensors are [B, T, n] with any strides whose last is 1."""
from __future__ import annotations

import ctypes

from . import _binding as _b
from ._window import MosaStrides, _bad, _float, _int, _keep, _new, _on, _plans, _rank, _sig, _space, _vector

_i32, _f32, _f64 = ctypes.c_int32, ctypes.c_float, ctypes.c_double

GATE_NONE, GATE_CHANNEL, GATE_TOKEN = 0, 1, 2


class MosaResidualShape(ctypes.Structure):
    """mosa_residual_shape: sizes, types, options and strides of mosa_residual_forward and its backward."""
    _fields_ = ([(n, _i32) for n in ("B", "T", "d", "dtype", "x_dtype", "y_dtype", "dh_dtype", "post_norm",
                                     "pre_norm", "gate", "sigmoid", "site")]
                + [("scale", _f32), ("eps", _f32), ("dropout", _f64)]
                + [(n, MosaStrides) for n in ("x", "y", "g", "xo", "h", "dxo", "dh", "dx", "dy", "dg")])


class MosaDropoutShape(ctypes.Structure):
    """mosa_dropout_shape: sizes and strides of mosa_dropout."""
    _fields_ = ([(n, _i32) for n in ("B", "T", "d", "dtype", "site")]
                + [("dropout", _f64), ("x", MosaStrides), ("y", MosaStrides)])


class MosaLogprobShape(ctypes.Structure):
    """mosa_logprob_shape: sizes and strides of mosa_token_logprobs and its backward."""
    _fields_ = ([(n, _i32) for n in ("B", "T", "V", "dtype", "target64", "top")]
                + [("scale", _f32), ("stats", _i32), ("z", MosaStrides), ("dz", MosaStrides)])


def declare(L) -> None:
    """Signatures of the block operators' functions."""
    vp, sz, st = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    res, drop, lp = (ctypes.POINTER(c) for c in (MosaResidualShape, MosaDropoutShape, MosaLogprobShape))
    for name, args, ret in (
            ("mosa_residual_forward", [res] + [vp] * 10, st),
            ("mosa_residual_workspace_bytes", [res], sz),
            ("mosa_residual_backward", [res] + [vp] * 14 + [vp, sz, vp], st),
            ("mosa_dropout", [drop] + [vp] * 4, st),
            ("mosa_token_logprobs_workspace_bytes", [lp], sz),
            ("mosa_token_logprobs", [lp] + [vp] * 7 + [vp, sz, vp], st),
            ("mosa_token_logprobs_backward", [lp] + [vp] * 11, st)):
        f = getattr(L, name)
        f.argtypes, f.restype = args, ret


# What depends on shapes, strides and types alone is done once and kept as a plan, as for the window heads.  Numbers in
# which a model's layers and steps differ (scale, eps, dropout, site) make no plans of their own: a plan keeps a struct for
# each set of them, which is written once and then only read.
# Calls make and look for everything on the current device and its current stream; one whose tensors lie on
# another device, or that names a stream, is made again in that one's place.

_structs = 0   # that plans keep, since they were last let go


def _numbered(plan, rng, **numbers):
    """A reference to the plan's struct with a call's numbers, kept under them."""
    global _structs
    if numbers.get("dropout", 0) > 0 and rng is None:
        raise ValueError("dropout needs rng, an int64 tensor of two numbers on the GPU")
    s = type(plan[2]).from_buffer_copy(plan[2])
    for name, value in numbers.items():
        setattr(s, name, _int(value, name) if name == "site" else value)
    if _structs >= 8192:   # (some megabytes: a site that counts steps, say)
        for p in list(_plans.values()):
            if type(p[0]) is dict:
                p[0].clear()
        _structs = 0
    _structs += 1
    plan[0][tuple(numbers.values())] = ref = ctypes.byref(s)
    return ref


def _there(t, stream, call, *args):
    """The call on ``stream``, or on the current stream of t's device."""
    cuda = _b._torch().cuda
    if stream is None:
        with cuda.device(t.get_device()):
            return call(*args)
    if not t.is_cuda:
        return call(*args)   # refuses it
    with _on(stream):
        if cuda.current_device() != t.get_device():
            raise ValueError("the stream must be one of the tensors' device")
        return call(*args)


def _all_on(dev, *ts):
    return all(t is None or t.get_device() == dev for t in ts)


def _elsewhere(dev, *named):
    """Says which tensor does not lie on device ``dev`` (a number; below 0: the CPU)."""
    for name, t in named:
        if t is not None and not t.is_cuda:
            _bad((name, t))
    for name, t in named:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"{name} must be on the device of the other tensors")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _rows(t, name, like=None, dtype=None):
    """Strides of a tensor [B, T, n], its shape ``like`` and type checked."""
    if like is not None and t.shape != like:
        raise ValueError(f"{name} must have shape {tuple(like)}, got {tuple(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    s = t.stride()
    if s[2] != 1 and t.shape[2] != 1:
        raise ValueError(f"{name}: the values of a token must be contiguous")
    return MosaStrides(s[0], s[1], 0)


def _result(t, name, like, dtype):
    """Strides of a result: a given tensor's, or those of the one to be made."""
    return MosaStrides(like[1] * like[2], like[2], 0) if t is None else _rows(t, name, like, dtype)


def _check_rng(rng):
    if rng is None:
        return
    if rng.shape != (2,) or rng.dtype != _b._torch_mod.int64 or not rng.is_contiguous():
        raise ValueError("rng must be a contiguous int64 tensor of two numbers")


# ------------------------------------------------------------ residual step

def _storage(dtype, gate, gamma_post, gamma_pre, x):
    """The storage type: given, or that of the first of gamma_pre, gamma_post, gate and x that is there."""
    if dtype is not None:
        return dtype
    for t in (gamma_pre, gamma_post, gate, x):
        if t is not None:
            return t.dtype


def _residual_plan(x, y, gate, gamma_post, gamma_pre, post_norm, pre_norm, sigmoid, rng, dtype, xo, h, stats, back=None):
    """Checks, and the library's struct without a call's numbers.  back: dx_out, dh and the results dx, dy, dgate,
    dgamma_post, dgamma_pre of a backward."""
    torch = _b._torch_mod
    for name, t in (("x", x), ("y", y)):
        _rank(t, name, 3)
    B, T, d = x.shape
    dtype = _storage(dtype, gate, gamma_post, gamma_pre, x)
    code = {torch.float32: _b.MOSA_F32, torch.bfloat16: _b.MOSA_BF16}
    if dtype not in code:
        raise TypeError(f"unsupported storage dtype {dtype} (float32 or bfloat16)")
    kind = GATE_NONE
    if gate is not None:
        kind = GATE_TOKEN if len(gate.shape) == 3 else GATE_CHANNEL
    s = MosaResidualShape(B, T, d, code[dtype], _b._dtype_code(x), _b._dtype_code(y), code[dtype],
                          1 if post_norm else 0, 1 if pre_norm else 0, kind, 1 if sigmoid else 0, 0, 1.0, 0.0, 0.0,
                          _rows(x, "x"), _rows(y, "y", x.shape))
    _vector(gamma_post, "gamma_post", (d,), dtype)
    _vector(gamma_pre, "gamma_pre", (d,), dtype)
    if kind == GATE_TOKEN:
        s.g = _rows(gate, "gate", x.shape, dtype)
    else:
        _vector(gate, "gate", (d,), dtype)
    _check_rng(rng)
    _vector(stats, "stats", (2, B, T), torch.float32)
    need = 0
    if back is None:
        s.xo = _result(xo, "out x", x.shape, x.dtype)
        s.h = _result(h, "out h", x.shape, dtype)
    else:
        dxo, dh, dx, dy, dg, dgpost, dgpre = back
        if dxo is not None:
            s.dxo = _rows(dxo, "dx_out", x.shape, x.dtype)
        if dh is not None:
            s.dh_dtype = _b._dtype_code(dh)
            s.dh = _rows(dh, "dh", x.shape)
        s.dx, s.dy = _result(dx, "dx", x.shape, x.dtype), _result(dy, "dy", x.shape, dtype)
        if kind == GATE_TOKEN:
            s.dg = _result(dg, "dgate", x.shape, dtype)
        else:
            _vector(dg, "dgate", (d,), torch.float32)
        _vector(dgpost, "dgamma_post", (d,), torch.float32)
        _vector(dgpre, "dgamma_pre", (d,), torch.float32)
        need = int(_b.load().mosa_residual_workspace_bytes(ctypes.byref(s)))
    return {}, need, s, (dtype, x.device, x.shape, (2, B, T))


def _options(post_norm, pre_norm, sigmoid, scale, eps, dropout, site):
    """Flags and numbers as plain ones."""
    return (bool(post_norm), bool(pre_norm), bool(sigmoid), _float(scale), _float(eps), float(dropout),
            _int(site, "site"))


def mosa_residual_forward(x, y, gate=None, gamma_post=None, gamma_pre=None, post_norm: bool = True,
                          pre_norm: bool = True, sigmoid: bool = False, scale: float = 1.0, eps: float = 1e-6,
                          dropout: float = 0.0, rng=None, site: int = 0, dtype=None, out=None, stream=None):
    """The step between two blocks, for the stream x and a block's output y, both [B,T,d]:
    n = RMS norm of y with gamma_post [d] (y itself without ``post_norm``); u = dropout of gate * n (gate: None,
    [d] or [B,T,d], through a sigmoid with ``sigmoid``); x_out = x + scale * u; h = RMS norm of x_out with
    gamma_pre (None without ``pre_norm``), the next block's input.  Returns (x_out, h, stats): x_out like
    x, h in the storage type (``dtype``, by default that of gamma_pre, gamma_post, gate or x), stats
    [2,B,T] fp32 for the backward.  x and y may each be fp32 or bf16; gammas and gate have the storage
    type.  ``rng`` [2] int64 on the GPU holds seed and offset, read when the call runs; ``site`` tells
    calls that share it apart.  ``out`` may hold "x" (x itself where no backward follows), "h" and "stats"."""
    try:
        dev = x.get_device()
        if stream is not None or (dev >= 0 and dev != _b._torch()._C._cuda_getDevice()):
            return _there(x, stream, mosa_residual_forward, x, y, gate, gamma_post, gamma_pre, post_norm, pre_norm,
                          sigmoid, scale, eps, dropout, rng, site, dtype, out)
        torch = _b._torch()
        xo, h, stats = (out.get("x"), out.get("h"), out.get("stats")) if out else (None, None, None)
        if not (type(scale) is type(eps) is type(dropout) is float and type(site) is int
                and type(post_norm) is type(pre_norm) is type(sigmoid) is bool):
            post_norm, pre_norm, sigmoid, scale, eps, dropout, site = _options(post_norm, pre_norm, sigmoid, scale, eps,
                                                                               dropout, site)
        key = (6, x.shape, x.stride(), x.dtype, y.shape, y.stride(), y.dtype,
               None if gate is None else (gate.shape, gate.stride(), gate.dtype),
               None if gamma_post is None else (gamma_post.shape, gamma_post.stride(), gamma_post.dtype),
               None if gamma_pre is None else (gamma_pre.shape, gamma_pre.stride(), gamma_pre.dtype),
               None if rng is None else (rng.shape, rng.stride(), rng.dtype), post_norm, pre_norm, sigmoid, dtype, dev,
               (_sig(xo), _sig(h), _sig(stats)) if out else None)
    except AttributeError:
        _bad(("x", x), ("y", y), ("gate", gate), ("gamma_post", gamma_post), ("gamma_pre", gamma_pre), ("rng", rng))
    plan = _plans.get(key) or _keep(key, _residual_plan(x, y, gate, gamma_post, gamma_pre, post_norm, pre_norm,
                                                        sigmoid, rng, dtype, xo, h, stats))
    ref = plan[0].get((scale, eps, dropout, site)) or _numbered(plan, rng, scale=scale, eps=eps, dropout=dropout,
                                                                site=site)
    if not (dev >= 0 and y.get_device() == dev and (gate is None or gate.get_device() == dev)
            and (gamma_post is None or gamma_post.get_device() == dev)
            and (gamma_pre is None or gamma_pre.get_device() == dev) and (rng is None or rng.get_device() == dev)
            and (out is None or _all_on(dev, xo, h, stats))):
        _elsewhere(dev, ("x", x), ("y", y), ("gate", gate), ("gamma_post", gamma_post), ("gamma_pre", gamma_pre),
                   ("rng", rng), ("out x", xo), ("out h", h), ("stats", stats))
    dt, device, shape, short = plan[3]
    if xo is None:
        xo = torch.empty_like(x) if x.is_contiguous() else torch.empty(shape, dtype=x.dtype, device=device)
    if not pre_norm:
        h = None
    elif h is None:
        h = torch.empty_like(xo) if dt is x.dtype and out is None else torch.empty(shape, dtype=dt, device=device)
    if stats is None:
        stats = torch.empty(short, dtype=torch.float32, device=device)
    rc = (_b._lib or _b.load()).mosa_residual_forward(
        ref, x.data_ptr(), y.data_ptr(), None if gate is None else gate.data_ptr(),
        None if gamma_post is None else gamma_post.data_ptr(), None if gamma_pre is None else gamma_pre.data_ptr(),
        None if rng is None else rng.data_ptr(), xo.data_ptr(), None if h is None else h.data_ptr(),
        stats.data_ptr(), torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        _b._check(rc, "mosa_residual_forward")
    return xo, h, stats


def mosa_residual_backward(x, y, stats, dx_out, dh, gate=None, gamma_post=None, gamma_pre=None,
                           post_norm: bool = True, pre_norm: bool = True, sigmoid: bool = False,
                           scale: float = 1.0, eps: float = 1e-6, dropout: float = 0.0, rng=None, site: int = 0,
                           dtype=None, workspace=None, out=None, stream=None):
    """Gradients of mosa_residual_forward from its inputs and stats and the gradients dx_out (like x) and
    dh (fp32 or bf16) of its results, either of which may be None.  Returns ({"dx", "dy", "dgate",
    "dgamma_post", "dgamma_pre"}, workspace): dx like x, dy in the storage type, dgate [d] fp32 or [B,T,d]
    in the storage type, dgamma_* [d] fp32; without the ones that the call has no input for (a norm
    without gamma has a gamma of ones).  ``rng`` must hold what it held in the forward.  ``out`` may hold any of
    them ("dx" may be dx_out)."""
    try:
        dev = x.get_device()
        if stream is not None or (dev >= 0 and dev != _b._torch()._C._cuda_getDevice()):
            return _there(x, stream, mosa_residual_backward, x, y, stats, dx_out, dh, gate, gamma_post, gamma_pre,
                          post_norm, pre_norm, sigmoid, scale, eps, dropout, rng, site, dtype, workspace, out)
        torch = _b._torch()
        f32 = torch.float32
        dx, dy, dg, dgpost, dgpre = ((out.get("dx"), out.get("dy"), out.get("dgate"), out.get("dgamma_post"),
                                      out.get("dgamma_pre")) if out else (None,) * 5)
        if not (type(scale) is type(eps) is type(dropout) is float and type(site) is int
                and type(post_norm) is type(pre_norm) is type(sigmoid) is bool):
            post_norm, pre_norm, sigmoid, scale, eps, dropout, site = _options(post_norm, pre_norm, sigmoid, scale, eps,
                                                                               dropout, site)
        if not pre_norm:
            dh = None
        key = (7, x.shape, x.stride(), x.dtype, y.shape, y.stride(), y.dtype,
               None if gate is None else (gate.shape, gate.stride(), gate.dtype),
               None if gamma_post is None else (gamma_post.shape, gamma_post.stride(), gamma_post.dtype),
               None if gamma_pre is None else (gamma_pre.shape, gamma_pre.stride(), gamma_pre.dtype),
               None if rng is None else (rng.shape, rng.stride(), rng.dtype), post_norm, pre_norm, sigmoid, dtype, dev,
               stats.shape, stats.stride(), stats.dtype,
               None if dx_out is None else (dx_out.shape, dx_out.stride(), dx_out.dtype),
               None if dh is None else (dh.shape, dh.stride(), dh.dtype),
               (_sig(dx), _sig(dy), _sig(dg), _sig(dgpost), _sig(dgpre)) if out else None)
    except AttributeError:
        _bad(("x", x), ("y", y), ("stats", stats), ("dx_out", dx_out), ("dh", dh), ("gate", gate),
             ("gamma_post", gamma_post), ("gamma_pre", gamma_pre), ("rng", rng))
    plan = _plans.get(key) or _keep(key, _residual_plan(x, y, gate, gamma_post, gamma_pre, post_norm, pre_norm,
                                                        sigmoid, rng, dtype, None, None, stats,
                                                        (dx_out, dh, dx, dy, dg, dgpost, dgpre)))
    ref = plan[0].get((scale, eps, dropout, site)) or _numbered(plan, rng, scale=scale, eps=eps, dropout=dropout,
                                                                site=site)
    if not (dev >= 0 and y.get_device() == dev and stats.get_device() == dev
            and (dx_out is None or dx_out.get_device() == dev) and (dh is None or dh.get_device() == dev)
            and (gate is None or gate.get_device() == dev) and (gamma_post is None or gamma_post.get_device() == dev)
            and (gamma_pre is None or gamma_pre.get_device() == dev) and (rng is None or rng.get_device() == dev)
            and (workspace is None or workspace.get_device() == dev)
            and (out is None or _all_on(dev, dx, dy, dg, dgpost, dgpre))):
        _elsewhere(dev, ("x", x), ("y", y), ("stats", stats), ("dx_out", dx_out), ("dh", dh), ("gate", gate),
                   ("gamma_post", gamma_post), ("gamma_pre", gamma_pre), ("rng", rng), ("workspace", workspace),
                   ("dx", dx), ("dy", dy), ("dgate", dg), ("dgamma_post", dgpost), ("dgamma_pre", dgpre))
    dt, device, shape, _ = plan[3]
    if dx is None:
        dx = torch.empty_like(x) if x.is_contiguous() else torch.empty(shape, dtype=x.dtype, device=device)
    if dy is None:
        dy = torch.empty(shape, dtype=dt, device=device)
    g = {"dx": dx, "dy": dy}
    width = shape[2]
    if gate is None:
        dg = None
    else:
        if dg is None:
            dg = torch.empty(gate.shape, dtype=dt if len(gate.shape) == 3 else f32, device=device)
        g["dgate"] = dg
    if not post_norm:
        dgpost = None
    else:
        g["dgamma_post"] = dgpost = torch.empty(width, dtype=f32, device=device) if dgpost is None else dgpost
    if not pre_norm:
        dgpre = None
    else:
        g["dgamma_pre"] = dgpre = torch.empty(width, dtype=f32, device=device) if dgpre is None else dgpre
    workspace = _space(workspace, plan[1], device)
    rc = (_b._lib or _b.load()).mosa_residual_backward(
        ref, x.data_ptr(), y.data_ptr(), None if gate is None else gate.data_ptr(),
        None if gamma_post is None else gamma_post.data_ptr(), None if gamma_pre is None else gamma_pre.data_ptr(),
        None if rng is None else rng.data_ptr(), stats.data_ptr(), None if dx_out is None else dx_out.data_ptr(),
        None if dh is None else dh.data_ptr(), dx.data_ptr(), dy.data_ptr(), None if dg is None else dg.data_ptr(),
        None if dgpost is None else dgpost.data_ptr(), None if dgpre is None else dgpre.data_ptr(),
        workspace.data_ptr(), workspace.numel(), torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        _b._check(rc, "mosa_residual_backward")
    return g, workspace


# ------------------------------------------------------------------ dropout

def _dropout_plan(x, rng, y):
    _rank(x, "x", 3)
    _check_rng(rng)
    s = MosaDropoutShape(*x.shape, _b._dtype_code(x), 0, 0.0, _rows(x, "x"), _result(y, "out y", x.shape, x.dtype))
    return {}, 0, s


def mosa_dropout(x, p: float, rng, site: int = 0, out=None, stream=None):
    """x [B,T,d] with each value dropped (0) with probability p, the others times 1/(1-p).  ``rng`` [2]
    int64 on the GPU holds seed and offset, read when the call runs; ``site`` tells calls that share
    it apart.  The same call on the gradient is the backward.  ``out`` may hold "y", x itself among them."""
    y = None
    try:
        dev = x.get_device()
        if stream is not None or (dev >= 0 and dev != _b._torch()._C._cuda_getDevice()):
            return _there(x, stream, mosa_dropout, x, p, rng, site, out)
        torch = _b._torch()
        y = out.get("y") if out else None
        if not (type(p) is float and type(site) is int):
            p, site = float(p), _int(site, "site")
        key = (8, x.shape, x.stride(), x.dtype, None if rng is None else (rng.shape, rng.stride(), rng.dtype),
               None if y is None else _sig(y))
    except AttributeError:
        _bad(("x", x), ("rng", rng), ("out y", y))
    plan = _plans.get(key) or _keep(key, _dropout_plan(x, rng, y))
    ref = plan[0].get((p, site)) or _numbered(plan, rng, dropout=p, site=site)
    if not (dev >= 0 and (rng is None or rng.get_device() == dev) and (y is None or y.get_device() == dev)):
        _elsewhere(dev, ("x", x), ("rng", rng), ("out y", y))
    if y is None:
        y = torch.empty_like(x) if x.is_contiguous() else _new(x)
    rc = (_b._lib or _b.load()).mosa_dropout(ref, x.data_ptr(), None if rng is None else rng.data_ptr(), y.data_ptr(),
                                             torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        _b._check(rc, "mosa_dropout")
    return y


# -------------------------------------------------------- log probabilities

def _logprob_plan(logits, targets, top, results, stats=None, keeps=False, back=None):
    """results: (name, tensor, columns or 0, type) of [B,T] or [B,T,columns] tensors to be checked; stats [3,B,T],
    which the call ``keeps`` or reads."""
    torch = _b._torch_mod
    _rank(logits, "logits", 3)
    B, T, V = logits.shape
    if targets is not None:
        _b._want("targets", targets, (B, T))
        if targets.dtype not in (torch.int32, torch.int64):
            raise TypeError(f"targets must be int32 or int64, got {targets.dtype}")
        if not targets.is_contiguous():
            raise ValueError("targets must be contiguous")
    for name, t, n, dtype in results:
        _vector(t, name, (B, T, n) if n else (B, T), dtype)
    _vector(stats, "stats", (3, B, T), torch.float32)
    s = MosaLogprobShape(B, T, V, _b._dtype_code(logits),
                         1 if targets is not None and targets.dtype == torch.int64 else 0,
                         _int(top, "top"), 1.0, 1 if keeps else 0, _rows(logits, "logits"))
    if back is not None:
        s.dz = _result(back[0], "dlogits", logits.shape, logits.dtype)
        return {}, 0, s
    return ({}, int(_b.load().mosa_token_logprobs_workspace_bytes(ctypes.byref(s))), s,
            (logits.device, (B, T), (B, T, top), (3, B, T)))


def mosa_token_logprobs(logits, targets=None, top: int = 0, scale: float = 1.0, workspace=None, out=None,
                        stream=None, stats: bool = False):
    """Log probabilities under softmax(scale * logits), logits [B,T,V] (scale: 1 / temperature).  Returns
    ({"logp", "entropy", "lse", "top", "top_logp"}, workspace): logp [B,T] of the targets [B,T] (int32 or int64;
    below 0: none, logp 0), entropy and lse [B,T], and with ``top`` > 0 (up to 32) the indices [B,T,top] int32
    of the largest entries in falling order, ties by the lower index, and their log probabilities;
    all fp32 but the indices.  Entries of -inf (or -2^90 and less) are ruled out.  With ``stats``, also "stats" [3,B,T]
    for the backward: lse (r["lse"] is that plane), the largest entry and the sum of powers relative to it, whose gradient does
    not lose digits where logits are large.  ``out`` may hold any of them."""
    try:
        dev = logits.get_device()
        if stream is not None or (dev >= 0 and dev != _b._torch()._C._cuda_getDevice()):
            return _there(logits, stream, mosa_token_logprobs, logits, targets, top, scale, workspace, out, None, stats)
        torch = _b._torch()
        f32 = torch.float32
        logp, ent, lse, idx, tlp = ((out.get("logp"), out.get("entropy"), out.get("lse"), out.get("top"),
                                     out.get("top_logp")) if out else (None,) * 5)
        if not (type(top) is int and type(scale) is float):
            top, scale = _int(top, "top"), _float(scale)
        if top == 0:
            idx = tlp = None
        sums = None
        if stats:
            stats = True
            sums = out.get("stats") if out else None
            if lse is not None and (sums is None or lse.data_ptr() != sums.data_ptr()):
                raise ValueError("with stats, lse is the first of its planes: out may hold stats alone")
        key = (9, logits.shape, logits.stride(), logits.dtype,
               None if targets is None else (targets.shape, targets.stride(), targets.dtype), top, dev,
               (_sig(logp), _sig(ent), _sig(lse), _sig(idx), _sig(tlp), _sig(sums)) if out else None,
               True if stats else False)
    except AttributeError:
        _bad(("logits", logits), ("targets", targets))
    plan = _plans.get(key) or _keep(key, _logprob_plan(
        logits, targets, top, [("logp", logp, 0, f32), ("entropy", ent, 0, f32), ("lse", lse, 0, f32),
                               ("top", idx, top, torch.int32), ("top_logp", tlp, top, f32)], sums, stats))
    ref = plan[0].get((scale,)) or _numbered(plan, None, scale=scale)
    if not (dev >= 0 and (targets is None or targets.get_device() == dev)
            and (workspace is None or workspace.get_device() == dev)
            and (out is None or _all_on(dev, logp, ent, lse, idx, tlp, sums))):
        _elsewhere(dev, ("logits", logits), ("targets", targets), ("workspace", workspace), ("logp", logp),
                   ("entropy", ent), ("lse", lse), ("top", idx), ("top_logp", tlp), ("stats", sums))
    device, lead, tops, planes = plan[3]
    r = {}
    if targets is None:
        logp = None
    else:
        r["logp"] = logp = torch.empty(lead, dtype=f32, device=device) if logp is None else logp
    r["entropy"] = ent = torch.empty(lead, dtype=f32, device=device) if ent is None else ent
    if stats:
        r["stats"] = sums = torch.empty(planes, dtype=f32, device=device) if sums is None else sums
        lse = sums[0] if lse is None else lse
    r["lse"] = lse = torch.empty(lead, dtype=f32, device=device) if lse is None else lse
    if top > 0:
        r["top"] = idx = torch.empty(tops, dtype=torch.int32, device=device) if idx is None else idx
        r["top_logp"] = tlp = torch.empty(tops, dtype=f32, device=device) if tlp is None else tlp
    workspace = _space(workspace, plan[1], device)
    rc = (_b._lib or _b.load()).mosa_token_logprobs(
        ref, logits.data_ptr(), None if targets is None else targets.data_ptr(),
        None if logp is None else logp.data_ptr(), ent.data_ptr(), lse.data_ptr(), _ptr(idx), _ptr(tlp),
        workspace.data_ptr(), workspace.numel(), torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        _b._check(rc, "mosa_token_logprobs")
    return r, workspace


def mosa_token_logprobs_backward(logits, targets, lse, entropy=None, dlogp=None, dentropy=None, dlse=None, top=None,
                                 dtop_logp=None, scale: float = 1.0, out=None, stream=None):
    """Gradient of the logits (like them) from mosa_token_logprobs' lse [B,T] or stats [3,B,T] and entropy and the gradients
    dlogp, dentropy, dlse [B,T] and dtop_logp [B,T,top] fp32 of its results, each None where there is none; ``top``:
    the indices that it returned, read with dtop_logp.  From lse alone the row's probabilities are off by |lse| 2^-24
    relative (its rounding), from stats by an amount that does not grow with the logits.  ``out`` may hold "dlogits", logits
    itself among them."""
    dz = None
    try:
        dev = logits.get_device()
        if stream is not None or (dev >= 0 and dev != _b._torch()._C._cuda_getDevice()):
            return _there(logits, stream, mosa_token_logprobs_backward, logits, targets, lse, entropy, dlogp, dentropy,
                          dlse, top, dtop_logp, scale, out)
        torch = _b._torch()
        f32 = torch.float32
        dz = out.get("dlogits") if out else None
        if dtop_logp is None:
            top = None
        if type(scale) is not float:
            scale = _float(scale)
        key = (10, logits.shape, logits.stride(), logits.dtype, _sig(targets), lse.shape, lse.stride(), lse.dtype,
               _sig(entropy), _sig(dlogp), _sig(dentropy), _sig(dlse), _sig(top), _sig(dtop_logp), _sig(dz))
    except AttributeError:
        _bad(("logits", logits), ("lse", lse), ("targets", targets), ("entropy", entropy), ("dlogp", dlogp),
             ("dentropy", dentropy), ("dlse", dlse), ("top", top), ("dtop_logp", dtop_logp), ("dlogits", dz))
    plan = _plans.get(key)
    if plan is None:
        n = 0
        if dtop_logp is not None:
            if top is None:
                raise TypeError("dtop_logp needs top, the indices of the forward")
            _rank(top, "top", 3)
            n = top.shape[2]
            if n == 0:
                raise ValueError("top must hold at least one index of each row")
        if dlogp is not None and targets is None:
            raise TypeError("dlogp needs targets")
        if dentropy is not None and entropy is None:
            raise TypeError("dentropy needs entropy, the forward's")
        kept = len(lse.shape) == 3
        plan = _keep(key, _logprob_plan(
            logits, targets, n,
            [("lse", None if kept else lse, 0, f32), ("entropy", entropy, 0, f32), ("dlogp", dlogp, 0, f32),
             ("dentropy", dentropy, 0, f32), ("dlse", dlse, 0, f32), ("top", top, n, torch.int32),
             ("dtop_logp", dtop_logp, n, f32)],
            lse if kept else None, kept, (dz,)))
    ref = plan[0].get((scale,)) or _numbered(plan, None, scale=scale)
    if not (dev >= 0 and lse.get_device() == dev
            and _all_on(dev, targets, entropy, dlogp, dentropy, dlse, top, dtop_logp, dz)):
        _elsewhere(dev, ("logits", logits), ("targets", targets), ("lse", lse), ("entropy", entropy), ("dlogp", dlogp),
                   ("dentropy", dentropy), ("dlse", dlse), ("top", top), ("dtop_logp", dtop_logp), ("dlogits", dz))
    if dz is None:
        dz = _new(logits)
    rc = (_b._lib or _b.load()).mosa_token_logprobs_backward(
        ref, logits.data_ptr(), _ptr(targets), lse.data_ptr(), _ptr(entropy), _ptr(top), _ptr(dlogp), _ptr(dentropy),
        _ptr(dlse), _ptr(dtop_logp), dz.data_ptr(), torch._C._cuda_getCurrentRawStream(dev))
    if rc:
        _b._check(rc, "mosa_token_logprobs_backward")
    return dz
