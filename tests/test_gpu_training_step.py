"""The 4-bit products, both exchanges and the orthogonalised update together, as examples/train_four_bit.py uses them."""
import importlib.util
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu


def test_the_example_learns():
    path = Path(__file__).resolve().parent.parent / "examples" / "train_four_bit.py"
    spec = importlib.util.spec_from_file_location("train_four_bit", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses = m.train(steps=40)
    assert all(v == v for v in losses)
    # the loss falls while aggregating in 4-bit blocks and keeps falling in the compressed domain
    assert losses[m.COLLECT - 1] < 0.9 * losses[0]
    assert sum(losses[-5:]) / 5 < 0.6 * losses[0]
    assert m.train(steps=3) == losses[:3]        # the same bits every time
