"""examples/learn_ids.py end to end on a small data set: both losses fall, and
the model assigns new points as kernel K-means does."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_learn_ids():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.fail("GPU test on a machine without a GPU")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "learn_ids.py")
    spec = importlib.util.spec_from_file_location("learn_ids", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    out = example.run(points=3000, new=400, clusters=10, dims=64, steps=40)
    for losses, agree in out.values():
        assert losses[-1] < losses[0]
    assert out["ids"][1] >= 0.95 and out["distances"][1] >= 0.95
