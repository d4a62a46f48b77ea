"""The window calls' workspaces: what they hold before a call has no effect, and a forward that no
backward follows needs a status word only."""
import pytest
import torch

import paper_2505_00315_gb300 as mosa
from test_gpu_window import inputs, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("force", ["0", "1"])
@pytest.mark.parametrize("hp,T,window,sinks", [(64, 700, 100, 4), (128, 700, 64, 130), (32, 90, 0, 0)])
def test_whatever_a_workspace_held(hp, T, window, sinks, force, monkeypatch):
    """NaNs everywhere but in the status word, sequences that end early among the tiles: the same bits."""
    monkeypatch.setenv("MOSA_FORCE_SIMT", force)
    q, k, v, dO = inputs(3, T, T, 4, 2, hp, "bf16", seed=hp)
    lens = torch.tensor([T, T // 3, 0], device="cuda", dtype=torch.int32)
    want = run(q, k, v, dO, window, sinks, lens)
    _, _, ws = mosa.mosa_window_forward(q, k, v, window, sinks, lens=lens)
    ws.fill_(0xFF)
    ws[:4].zero_()
    O, lse, _ = mosa.mosa_window_forward(q, k, v, window, sinks, lens=lens, workspace=ws)
    g = mosa.mosa_window_backward(q, k, v, O, lse, dO, ws, window, sinks, lens=lens)
    assert mosa.mosa_window_check_status(ws) == 0
    for name, x in {"O": O, "lse": lse, **g}.items():
        assert torch.equal(x, want[name]), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_forward_alone_takes_a_status_word(dtype):
    q, k, v, _ = inputs(2, 500, 500, 4, 2, 64, dtype, seed=3)
    want = mosa.mosa_window_forward(q, k, v, 100, 4)[0]
    O, lse, ws = mosa.mosa_window_forward(q, k, v, 100, 4, want_lse=False)
    assert ws.numel() == 256 and lse is None and torch.equal(O, want)
    assert mosa.mosa_window_check_status(ws) == 0
    with pytest.raises(RuntimeError, match="workspace"):
        mosa.mosa_window_forward(q, k, v, 100, 4, workspace=ws)   # with lse it keeps more


def test_the_status_word_is_read_and_cleared():
    """A wait that gave up sets 2 in it."""
    q, k, v, _ = inputs(1, 200, 200, 2, 1, 64, "bf16", seed=4)
    _, _, ws = mosa.mosa_window_forward(q, k, v, 100, 4)
    assert mosa.mosa_window_check_status(ws) == 0
    ws[:4].view(torch.int32).fill_(2)
    assert mosa.mosa_window_check_status(ws) == 4    # MOSA_ERR_DEVICE_TIMEOUT
    assert mosa.mosa_window_check_status(ws) == 0
