"""The context operators together, as the example runs them: training lowers the objective, a served word gets the vector
that the whole text gives it."""
import os
import sys

import pytest
import torch

from paper_1606_08495_amd import w2v

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.gpu
def test_training_lowers_the_objective_and_a_cache_serves_it():
    import context_vectors as cv
    model = cv.ContextModel()
    losses = []
    for h in range(25):
        tokens, off = cv.texts(h)
        losses.append(float(model.step(tokens, off, w2v.minibatch_seed(7, h), 0.05)))
    assert losses[-1] < 0.9 * losses[0], losses
    words = [100, 103, 107, 101, 109, 110, 104, 102]
    one = model.serve(words)
    model.see["right"] = 0                                      # the whole text, causal
    off = torch.tensor([0, len(words)], dtype=torch.int64, device="cuda")
    whole = model.forward(w2v.as_index_tensor(words), off)[-1][0]
    assert torch.allclose(one[0], whole[-1], atol=1e-4)
    model.shard.destroy()
