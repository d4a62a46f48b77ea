"""Outputs whose elements share places are refused: two CTAs would write to one."""
import ctypes
import random

import pytest

from paper_2505_00315_gb300 import _binding as B
from paper_2505_00315_gb300 import _window as W
from test_window_abi import INV, S, decode, norm_bwd, norm_fwd, qk, win_bwd, win_dec, win_fwd, window


@pytest.mark.parametrize("st", [S(2560, 64, 64), S(2560, 128, 64), S(256, 256, 64), S(640, 64, 640),
                                S(100, 256, 64), S(2560, 250, 64)])
def test_overlaps_are_refused(st):
    """Tokens as far apart as heads, sequences as far as tokens, rows that share some values."""
    assert win_fwd(window(s_o=st)) == INV
    assert win_bwd(window(s_dq=st)) == INV
    assert norm_fwd(qk(s_yq=st)) == INV
    assert norm_bwd(qk(s_dq=st)) == INV
    assert win_dec(decode(H=4, Hkv=4, s_kc=st)) == INV


def overlaps(B_, T, H, st, hp):
    seen = set()
    for b in range(B_):
        for t in range(T):
            for h in range(H):
                at = b * st.b * (B_ > 1) + t * st.t * (T > 1) + h * st.h * (H > 1)
                for e in range(hp):
                    if at + e in seen:
                        return True
                    seen.add(at + e)
    return False


def test_against_every_element():
    """Layouts of all kinds, taken or refused as their elements say."""
    rng, found = random.Random(3), [0, 0]
    for _ in range(1500):
        B_, T, H, hp = rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 4), 16
        st = S(*(rng.choice((0, 8, 16, 17, 24, 32, 40, 48, 64, 80, 112, 128, 200)) for _ in range(3)))
        bad = overlaps(B_, T, H, st, hp)
        s = window(B=B_, Tq=T, Tk=T, H=H, Hkv=H, hp=hp, s_o=st)
        need = B.load().mosa_window_workspace_bytes(ctypes.byref(s))
        assert (need == 0) == bad, (B_, T, H, st.b, st.t, st.h)
        found[bad] += 1
    assert min(found) > 200


def test_large_layouts_are_taken():
    """Orders of the dimensions, padded rows, a slice of heads, every other token; sizes of 1 at any stride."""
    for B_, T, H, st in ((8, 4096, 32, S(4096 * 40 * 128, 40 * 128, 128)), (8, 4096, 32, S(32 * 4096 * 128, 128, 4096 * 128)),
                         (48, 4100, 8, S(128, 48 * 8 * 128, 48 * 128)), (1, 300, 2, S(0, 9_000_000, 128)),
                         (65535, 3, 1, S(128 * 6, 256, 0)), (1, 1, 1, S(0, 0, 0)), (65535, 2, 65535, S(2 * 65535 * 128, 128, 256))):
        s = qk(B=B_, T=T, H=H, Hkv=H, hp=128, **{n: st for n in ("s_q", "s_k", "s_yq", "s_yk", "s_dq", "s_dk")})
        assert B.load().mosa_qk_norm_rope_workspace_bytes(ctypes.byref(s)) > 0, (B_, T, H)
