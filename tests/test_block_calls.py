"""The block operators' binding and C ABI without a GPU: what reaches the library, and what is refused before it."""
import ctypes


import test_block_abi as abi
from paper_2505_00315_gb300 import _binding as B
from paper_2505_00315_gb300 import _block as K


def test_stats_is_a_truth_value():
    for bad in (2, -1):
        s = abi.logprob(stats=bad)
        assert abi.lp_fwd(s) == abi.INV and abi.lp_bwd(s) == abi.INV
        assert B.load().mosa_token_logprobs_workspace_bytes(ctypes.byref(s)) == 0
    p = [abi.FAKE] * 7
    p[4] = abi.OFF                  # lse, or stats
    assert abi.lp_fwd(abi.logprob(stats=1), p) == abi.INV


def test_stats_takes_no_other_place():
    """The struct is as long as before: the new field lies where alignment left room."""
    assert ctypes.sizeof(K.MosaLogprobShape) == 7 * 4 + 4 + 6 * 8
    assert K.MosaLogprobShape.z.offset == 32
