"""The block operators' C ABI and binding without a GPU: what they refuse, before anything is launched and
before any CUDA call; and the random words' definition."""
import ctypes

import numpy as np
import pytest
import torch

from _block_ref import philox, philox_words
from paper_2505_00315_gb300 import _binding as B
from paper_2505_00315_gb300 import _block as K

FAKE = ctypes.c_void_p(0x100000)   # never dereferenced: validation fails first
OFF = ctypes.c_void_p(0x100001)    # not at a multiple of any element's size
INV, UNS, WS = B.MOSA_ERR_INVALID_ARG, B.MOSA_ERR_UNSUPPORTED, B.MOSA_ERR_WORKSPACE
S = K.MosaStrides
NAN, INF = float("nan"), float("inf")


def dense(T, n):
    return S(T * n, n, 0)


def residual(**kw):
    f = dict(B=2, T=10, d=64, dtype=B.MOSA_BF16, x_dtype=B.MOSA_BF16, y_dtype=B.MOSA_F32, dh_dtype=B.MOSA_F32,
             post_norm=1, pre_norm=1, gate=K.GATE_TOKEN, sigmoid=1, site=0, scale=1.0, eps=1e-6, dropout=0.1)
    f.update({k: v for k, v in kw.items() if k in f})
    s = K.MosaResidualShape(**f)
    for n in ("x", "y", "g", "xo", "h", "dxo", "dh", "dx", "dy", "dg"):
        setattr(s, n, kw.get("s_" + n, dense(f["T"], f["d"])))
    return s


def res_fwd(s, ptrs=None):
    return B.load().mosa_residual_forward(ctypes.byref(s), *(ptrs or [FAKE] * 9), None)


def res_bwd(s, ptrs=None, ws=FAKE, n=1 << 40):
    return B.load().mosa_residual_backward(ctypes.byref(s), *(ptrs or [FAKE] * 14), ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), INV), (dict(T=0), INV), (dict(d=-1), INV), (dict(dtype=5), INV), (dict(x_dtype=2), INV),
    (dict(y_dtype=-1), INV), (dict(post_norm=2), INV), (dict(pre_norm=-1), INV), (dict(gate=3), INV),
    (dict(gate=-1), INV), (dict(sigmoid=2), INV), (dict(scale=INF), INV), (dict(scale=NAN), INV),
    (dict(eps=-1.0), INV), (dict(eps=NAN), INV), (dict(eps=INF), INV), (dict(dropout=-0.1), INV),
    (dict(dropout=1.1), INV), (dict(dropout=NAN), INV), (dict(d=8200), UNS), (dict(B=1 << 16, T=1 << 15), UNS),
    (dict(s_x=S(-1, 64, 0)), INV), (dict(s_y=S(640, -64, 0)), INV), (dict(s_g=S(1 << 61, 64, 0)), INV),
])
def test_residual_refuses(kw, code):
    s = residual(**kw)
    assert res_fwd(s) == code and res_bwd(s) == code
    assert B.load().mosa_residual_workspace_bytes(ctypes.byref(s)) == 0


def test_residual_refuses_outputs_that_meet_themselves():
    for n in ("s_xo", "s_h"):
        assert res_fwd(residual(**{n: S(640, 32, 0)})) == INV
        assert res_fwd(residual(**{n: S(0, 64, 0)})) == INV
    for n in ("s_dx", "s_dy", "s_dg"):
        assert res_bwd(residual(**{n: S(640, 32, 0)})) == INV
        assert res_bwd(residual(**{n: S(64, 64, 0)})) == INV
    assert res_bwd(residual(dh_dtype=7)) == INV


def test_residual_refuses_pointers_and_workspaces():
    L = B.load()
    for i in (0, 1, 2, 5, 6, 7):       # x, y, gate, rng, x_out, h
        for bad in (None, OFF):
            p = [FAKE] * 9
            p[i] = bad
            assert res_fwd(residual(), p) == INV, i
    for i in (3, 4, 8):                # gammas and stats may be NULL, not misplaced
        p = [FAKE] * 9
        p[i] = OFF
        assert res_fwd(residual(), p) == INV, i
    for i in (0, 1, 2, 5, 6, 9, 10):   # x, y, gate, rng, stats, dx, dy
        for bad in (None, OFF):
            p = [FAKE] * 14
            p[i] = bad
            assert res_bwd(residual(), p) == INV, i
    for i in (3, 4, 7, 8, 11, 12, 13):
        p = [FAKE] * 14
        p[i] = OFF
        assert res_bwd(residual(), p) == INV, i
    p = [FAKE] * 9
    p[5] = ctypes.c_void_p(0x100004)   # rng holds 64-bit numbers
    assert res_fwd(residual(), p) == INV
    need = L.mosa_residual_workspace_bytes(ctypes.byref(residual()))
    assert need > 0
    assert res_bwd(residual(), ws=None) == WS
    assert res_bwd(residual(), ws=ctypes.c_void_p(0x100010)) == WS
    assert res_bwd(residual(), n=need - 1) == WS
    assert L.mosa_residual_forward(None, *[FAKE] * 9, None) == INV


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), INV), (dict(T=-1), INV), (dict(d=0), INV), (dict(dtype=2), INV), (dict(dropout=1.5), INV),
    (dict(dropout=NAN), INV), (dict(B=1 << 16, T=1 << 15), UNS), (dict(d=2**31 - 1), UNS), (dict(T=1 << 20, d=1 << 20), UNS),
    (dict(x=S(-1, 64, 0)), INV), (dict(y=S(0, 64, 0)), INV),
    (dict(y=S(640, 63, 0)), INV),
])
def test_dropout_refuses(kw, code):
    f = dict(B=2, T=10, d=64, dtype=B.MOSA_BF16, site=0, dropout=0.5, x=dense(10, 64), y=dense(10, 64))
    assert B.load().mosa_dropout(ctypes.byref(K.MosaDropoutShape(**{**f, **kw})), FAKE, FAKE, FAKE, None) == code


def test_dropout_refuses_pointers():
    s = K.MosaDropoutShape(2, 10, 64, B.MOSA_F32, 0, 0.5, dense(10, 64), dense(10, 64))
    for p in ((None, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, None), (OFF, FAKE, FAKE), (FAKE, OFF, FAKE),
              (FAKE, FAKE, OFF)):
        assert B.load().mosa_dropout(ctypes.byref(s), *p, None) == INV
    assert B.load().mosa_dropout(None, FAKE, FAKE, FAKE, None) == INV


def logprob(**kw):
    f = dict(B=2, T=3, V=100, dtype=B.MOSA_BF16, target64=1, top=5, scale=1.0, z=dense(3, 100), dz=dense(3, 100))
    return K.MosaLogprobShape(**{**f, **kw})


def lp_fwd(s, ptrs=None, ws=FAKE, n=1 << 40):
    return B.load().mosa_token_logprobs(ctypes.byref(s), *(ptrs or [FAKE] * 7), ws, n, None)


def lp_bwd(s, ptrs=None):
    return B.load().mosa_token_logprobs_backward(ctypes.byref(s), *(ptrs or [FAKE] * 10), None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), INV), (dict(T=0), INV), (dict(V=0), INV), (dict(dtype=3), INV), (dict(target64=2), INV),
    (dict(top=-1), INV), (dict(V=4, top=5), INV), (dict(top=33), UNS), (dict(scale=0.0), INV), (dict(scale=-1.0), INV),
    (dict(scale=NAN), INV), (dict(scale=INF), INV), (dict(scale=1e-7), UNS), (dict(scale=2e6), UNS),
    (dict(V=2**31 - 1), UNS), (dict(B=1 << 16, T=1 << 15), UNS), (dict(z=S(-1, 100, 0)), INV),
])
def test_logprobs_refuse(kw, code):
    s = logprob(**kw)
    assert lp_fwd(s) == code and lp_bwd(s) == code
    assert B.load().mosa_token_logprobs_workspace_bytes(ctypes.byref(s)) == 0


def test_logprobs_refuse_pointers_and_workspaces():
    L = B.load()
    for i in (0, 5, 6):            # logits, top, top_logp
        for bad in (None, OFF):
            p = [FAKE] * 7
            p[i] = bad
            assert lp_fwd(logprob(), p) == INV, i
    for i in (1, 2, 3, 4):
        p = [FAKE] * 7
        p[i] = OFF
        assert lp_fwd(logprob(), p) == INV, i
    p = [FAKE] * 7
    p[1] = None                    # logp without targets
    assert lp_fwd(logprob(), p) == INV
    p[1] = ctypes.c_void_p(0x100004)
    assert lp_fwd(logprob(), p) == INV
    for i in (0, 2, 4, 8, 9):      # logits, lse, top, dtop_logp, dlogits
        for bad in (None, OFF):
            p = [FAKE] * 10
            p[i] = bad
            assert lp_bwd(logprob(), p) == INV, i
    for i, needs in ((1, 5), (3, 6)):   # dlogp needs targets, dentropy needs entropy
        p = [FAKE] * 10
        p[i] = None
        assert lp_bwd(logprob(), p) == INV, needs
    assert lp_bwd(logprob(dz=S(300, 99, 0))) == INV
    need = L.mosa_token_logprobs_workspace_bytes(ctypes.byref(logprob()))
    assert need > 0 and lp_fwd(logprob(), ws=None) == WS and lp_fwd(logprob(), n=need - 1) == WS
    assert lp_fwd(logprob(), ws=ctypes.c_void_p(0x100080)) == WS


def test_binding_refuses():
    """Shapes, types and devices, before the library is called."""
    x, v = torch.zeros(2, 8, 64), torch.zeros(64)
    rng = torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA tensor"):
        K.mosa_residual_forward(x, x)
    with pytest.raises(TypeError, match="torch.Tensor"):
        K.mosa_residual_forward(x.numpy(), x)
    with pytest.raises(ValueError, match="dimensions"):
        K.mosa_residual_forward(x[0], x)
    with pytest.raises(ValueError, match="must have shape"):
        K.mosa_residual_forward(x, x[:, :4])
    with pytest.raises(TypeError, match="unsupported"):
        K.mosa_residual_forward(x.half(), x)
    with pytest.raises(TypeError, match="gamma_post"):
        K.mosa_residual_forward(x, x, gamma_post=v.bfloat16(), gamma_pre=v)
    with pytest.raises(ValueError, match="gate"):
        K.mosa_residual_forward(x, x, gate=v[:8])
    with pytest.raises(ValueError, match="contiguous"):
        K.mosa_residual_forward(x.transpose(1, 2).contiguous().transpose(1, 2), x)
    with pytest.raises(ValueError, match="rng"):
        K.mosa_residual_forward(x, x, dropout=0.1)
    with pytest.raises(ValueError, match="rng"):
        K.mosa_residual_forward(x, x, dropout=0.1, rng=rng.int())
    with pytest.raises(ValueError, match="32 bits"):
        K.mosa_residual_forward(x, x, site=2**31)
    with pytest.raises(ValueError, match="stats"):
        K.mosa_residual_backward(x, x, torch.zeros(2, 8, 2), x, x)
    with pytest.raises(ValueError, match="dh must have shape"):
        K.mosa_residual_backward(x, x, torch.zeros(2, 2, 8), x, x[:1])
    with pytest.raises(TypeError, match="dx_out"):
        K.mosa_residual_backward(x, x, torch.zeros(2, 2, 8), x.bfloat16(), x)
    with pytest.raises(ValueError, match="CUDA tensor"):
        K.mosa_dropout(x, 0.1, rng)
    with pytest.raises(ValueError, match="rng"):
        K.mosa_dropout(x, 0.1, None)
    with pytest.raises(ValueError, match="CUDA tensor"):
        K.mosa_token_logprobs(x)
    with pytest.raises(ValueError, match="targets"):
        K.mosa_token_logprobs(x, torch.zeros(2, 7, dtype=torch.int64))
    with pytest.raises(TypeError, match="targets"):
        K.mosa_token_logprobs(x, torch.zeros(2, 8))
    with pytest.raises(ValueError, match="top must have shape"):
        K.mosa_token_logprobs(x, top=3, out={"top": torch.zeros(2, 8, 4, dtype=torch.int32)})
    with pytest.raises(TypeError, match="dlogp needs targets"):
        K.mosa_token_logprobs_backward(x, None, x[..., 0].contiguous(), dlogp=x[..., 0].contiguous())
    with pytest.raises(TypeError, match="dtop_logp needs top"):
        K.mosa_token_logprobs_backward(x, None, x[..., 0].contiguous(), dtop_logp=x[..., :2].contiguous())
    with pytest.raises(TypeError, match="dentropy needs entropy"):
        K.mosa_token_logprobs_backward(x, None, x[..., 0].contiguous(), dentropy=x[..., 0].contiguous())


@pytest.mark.parametrize("bad", [None, [1.0], 3])
def test_binding_names_what_is_no_tensor(bad):
    x, rng = torch.zeros(2, 8, 64), torch.zeros(2, dtype=torch.int64)
    row = x[..., 0].contiguous()
    for call in (lambda: K.mosa_residual_forward(bad, x), lambda: K.mosa_residual_backward(bad, x, x, x, x),
                 lambda: K.mosa_dropout(bad, 0.5, rng), lambda: K.mosa_token_logprobs(bad),
                 lambda: K.mosa_token_logprobs_backward(bad, None, row)):
        with pytest.raises((TypeError, ValueError), match="must be a|missing"):
            call()


def test_random_words_are_the_published_ones():
    """Philox 4x32 with seven rounds: the known answers that its authors publish with their library."""
    for counter, key, words in (
            ((0, 0, 0, 0), 0, (0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48)),
            ((0xFFFFFFFF,) * 4, 2**64 - 1, (0x5207DDC2, 0x45165E59, 0x4D8EE751, 0x8C52F662))):
        x = [np.array([c], np.uint64) for c in counter]
        assert tuple(int(w[0]) for w in philox_words(x, key)) == words


def test_random_words_are_even():
    """Each bit of a column's word is 1 half of the time, over rows and over sites: 4096 words, within
    five standard deviations (0.5 +- 5 / 128)."""
    w = philox(12345, 7, 4096, 3)
    v = np.stack([philox(12345, s, 1, 1)[0] for s in range(4096)])
    for x in (w, v):
        ones = ((x[..., None] >> np.arange(32, dtype=np.uint64)) & np.uint64(1)).mean(0)
        assert np.all(np.abs(ones - 0.5) < 5 / 128)
