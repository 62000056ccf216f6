"""The training operators as they are used together: the example trains, with 32- and with 8-bit states."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_gated_block", os.path.join(ROOT, "examples", "train_gated_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_example_trains_alike_with_32_and_8_bit_states():
    """The loss of a random start falls by half at least, and 8-bit states lose no more than a tenth of that fall."""
    train = _example().train
    full, eight = train(steps=60), train(steps=60, state_bits=8)
    assert full[0] == eight[0]
    assert full[-1] < 0.5 * full[0]
    assert full[0] - eight[-1] > 0.9 * (full[0] - full[-1])


def test_example_runs_one_layer_one_worker():
    losses = _example().train(steps=3, workers=1, layers=1, d=64, f=136, tokens=33)
    assert len(losses) == 3 and losses[-1] < losses[0]
