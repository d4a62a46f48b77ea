"""The window kernels' device waits run out: the call says so, and the next one is as ever."""
import pytest
import torch

import paper_2505_00315_gb300 as mosa
from test_gpu_window import inputs, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hp,T,window,sinks", [(64, 1500, 0, 0), (128, 1500, 700, 4), (64, 1500, 60, 2)])
def test_waits_that_run_out_are_reported_and_leave_nothing_behind(hp, T, window, sinks, monkeypatch):
    """A limit of 1 ns, which the first loads outlast: every CTA gives up, lets its copies and products in
    flight finish, frees its tensor memory and ends.  The same workspace then gives the same bits."""
    q, k, v, dO = inputs(2, T, T, 8, 4, hp, "bf16", seed=51)
    want = run(q, k, v, dO, window, sinks)
    O, lse, ws = mosa.mosa_window_forward(q, k, v, window, sinks)
    torch.cuda.synchronize()
    monkeypatch.setenv("MOSA_TEST_WINDOW_WAIT_NS", "1")
    mosa.mosa_window_forward(q, k, v, window, sinks, workspace=ws)
    assert mosa.mosa_window_check_status(ws) == 4        # MOSA_ERR_DEVICE_TIMEOUT
    mosa.mosa_window_backward(q, k, v, O, lse, dO, ws, window, sinks)
    assert mosa.mosa_window_check_status(ws) == 4
    monkeypatch.delenv("MOSA_TEST_WINDOW_WAIT_NS")
    O, lse, _ = mosa.mosa_window_forward(q, k, v, window, sinks, workspace=ws)
    g = mosa.mosa_window_backward(q, k, v, O, lse, dO, ws, window, sinks)
    assert mosa.mosa_window_check_status(ws) == 0
    for name, x in {"O": O, "lse": lse, **g}.items():
        assert torch.equal(x, want[name]), name
