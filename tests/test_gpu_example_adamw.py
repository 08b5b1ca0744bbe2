"""The training example with AdamW for its vectors: one step of them against the definition in 64 bits, and the scores of tokens."""
import os
import sys

import pytest

from paper_2309_06497_amd import binding as B

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


def model_and_batch(vectors):
    import train_residual_mlp as ex
    return ex, ex.ResidualMLP(512, 128, 2, seed=1, vectors=vectors), ex.batch(512, 1024, 0)


def test_first_step_of_the_vectors():
    """m = 0.1 g and v = 0.001 g^2 at the first step: every vector moves by the sign of its gradient times lr / (1 + epsilon / |g|), whatever the norm limits.  Half a dozen float32
    roundings of a move of lr and one of a weight of 1: 1e-6 of lr and 2^-23."""
    import torch
    ex, model, (tokens, targets) = model_and_batch("adamw")
    before = [v.double().clone() for v in model.vectors]
    _, matrices, vectors = model.loss_and_gradients(tokens, targets)
    norm = torch.sqrt(sum(g.double().square().sum() for g in matrices + vectors))
    model.step(tokens, targets, 0.02, 0)
    for v, w, g in zip(model.vectors, before, vectors):
        g = g.double() * min(1.0, 1.0 / float(norm))
        want = -0.002 * g / (g.abs() + 1e-8)
        assert float((v.double() - w - want).abs().max()) <= 1e-6 * 0.002 + 2.0 ** -23
    for t in range(1, 4):
        assert torch.isfinite(model.step(*ex.batch(512, 1024, t), 0.02, t))


@pytest.mark.parametrize("vectors", ["shampoo", "adamw"])
def test_scores(vectors):
    """Against the loss of the same tokens, which shampoo_linear_cross_entropy makes from the same activations: the logits here are rounded to bf16 first, half a step of 2^-8 of values
    of a few units: 0.02 of each, a tenth of that in the mean over 1024"""
    import torch
    _, model, (tokens, targets) = model_and_batch(vectors)
    r = model.scores(tokens, targets)
    loss, _, _ = model.loss_and_gradients(tokens, targets)
    assert abs(float(r.log_probs.mean()) + float(loss)) < 0.02
    assert r.top_tokens.shape == (1024, 2) and (r.top_log_probs[:, 0] >= r.top_log_probs[:, 1]).all() and (r.top_log_probs[:, 0] >= r.log_probs).all()
    assert isinstance(r, B.LogProbs) and (r.entropy > 0).all()
