"""The training-side operators and the compressed aggregation together, as
examples/compressed_step.py runs them: every sum is recovered, and it learns."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_compressed_steps_learn():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location(
        "compressed_step", os.path.join(ROOT, "examples", "compressed_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.main(steps=12, workers=3)
    assert all(math.isfinite(v) for v in losses)
    # it starts at about the entropy of the classes and has to fall by a tenth of it
    assert losses[-1] < losses[0] - 0.1 * math.log(example.CLASSES)
