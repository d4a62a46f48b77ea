"""The window heads as a model uses them: the example trains, with and without MoSA heads beside
them, and continues its language token by token."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("window_lm", os.path.join(ROOT, "examples",
                                                                            "window_lm.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.gpu
def test_model_trains_and_generates():
    first, last, right, far = example().main(steps=150, quiet=True)
    assert first > 3.0 and last < 0.5 * first
    # whole text and token by token differ by the roundings of two layers' activations to bf16
    # (some 2^-9 each): 5 %
    assert far < 0.05
    assert right > 0.5


@pytest.mark.gpu
def test_model_trains_beside_mosa_heads():
    first, last, _, _ = example().main(steps=60, n_mosa=4, quiet=True)
    assert first > 3.0 and last < first - 0.2
