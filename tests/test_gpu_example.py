"""The language-model example: the operators and the averaging step together."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dtype,keep,drop", [("f32", "values", 0.0), ("f32", "int8", 0.1), ("bf16", "int8", 0.1)])
def test_workers_learn_over_a_lossy_network(dtype, keep, drop):
    if not torch.cuda.is_available():
        pytest.fail("this test needs a CUDA device")
    import train_language_model

    losses = train_language_model.train(steps=120, workers=4, drop=drop, vocab=200, width=64, blocks=2, tokens=512, dtype=dtype, keep=keep)
    assert torch.isfinite(losses).all()
    # log 200 = 5.3 at the start; the successor of every word is learnt to a good part
    assert losses[:3].mean() > 4.5 and losses[-10:].mean() < 0.7 * losses[:3].mean()

