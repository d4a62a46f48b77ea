"""Window heads called for a stream that is not the current one."""
import pytest
import torch

import paper_2505_00315_gb300 as mosa
from test_gpu_window import inputs, norm_inputs, run

pytestmark = pytest.mark.gpu


def test_a_call_for_a_stream_is_not_held_up_by_the_current_one():
    """The current stream is busy while another one's calls make their results and workspaces: what
    they leave in the workspace is still there when the current stream is done."""
    q, k, v, dO = inputs(2, 500, 500, 4, 2, 64, "bf16", seed=15)
    want = run(q, k, v, dO, 100, 4)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    O, lse, ws = mosa.mosa_window_forward(q, k, v, 100, 4, stream=s)
    s.synchronize()
    assert not torch.cuda.current_stream().query()     # (0.1 s: still asleep)
    torch.cuda.synchronize()
    g = mosa.mosa_window_backward(q, k, v, O, lse, dO, ws, 100, 4, stream=s)
    s.synchronize()
    assert mosa.mosa_window_check_status(ws, stream=s) == 0
    for name, x in {"O": O, "lse": lse, **g}.items():
        assert torch.equal(x, want[name]), name


def test_norms_and_decoding_for_a_stream():
    q, k, gq, gk, dyq, dyk, pos = norm_inputs(2, 300, 8, 2, 64, "bf16", seed=6)
    lens = torch.tensor([64, 100], device="cuda", dtype=torch.int32)

    def calls(stream):
        cache = [torch.zeros(2, 64, 2, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
        torch.cuda.synchronize()
        y = mosa.mosa_qk_norm_rope(q, k, gq, gk, positions=pos, stream=stream)
        g, _ = mosa.mosa_qk_norm_rope_backward(q, k, gq, gk, dyq, dyk, positions=pos, stream=stream)
        o, _ = mosa.mosa_window_decode(q[:, 0], k[:, 0], k[:, 1], *cache, lens, 60, 4, gamma_q=gq,
                                       gamma_k=gk, stream=stream)
        torch.cuda.synchronize()
        return [*y, *g.values(), o, *cache]

    for a, b in zip(calls(torch.cuda.Stream()), calls(None)):
        assert torch.equal(a, b)
