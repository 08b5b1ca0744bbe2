"""The training example: its gradients against automatic differentiation of the same model, and that it learns."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


def model_and_batch():
    import train_residual_mlp as ex
    return ex, ex.ResidualMLP(512, 128, 2, seed=1), ex.batch(512, 1024, 0)


def test_gradients_of_the_example():
    """Against float64 differentiation.  What separates the two: activations in bf16 (2^-8 an element at most, half a dozen of them one
    behind the other) and in 8 bits (half a step is 1/127 of a group's largest, about 1/60 of a typical element): errors of
    some percent of a gradient's norm.  A term that is left out shows as tens of percent."""
    import torch
    ex, model, (tokens, targets) = model_and_batch()
    loss, matrices, vectors = model.loss_and_gradients(tokens, targets)
    m = [w.double().requires_grad_() for w in model.matrices]
    v = [w.double().requires_grad_() for w in model.vectors]
    norm = lambda x, w: x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-5) * w
    r = model.embed[tokens].double()
    h = r
    for i in range(model.layers):
        gate, w_post, w_pre = v[3 * i:3 * i + 3]
        f = torch.nn.functional.gelu(h @ m[2 * i]) @ m[2 * i + 1]
        r = r + model.SCALE * gate * norm(f, w_post)
        h = norm(r, w_pre)
    value = torch.nn.functional.cross_entropy(h @ m[-1].t(), targets)
    want = torch.autograd.grad(value, m + v)
    assert abs(float(loss) - float(value.detach())) <= 0.02 * float(value.detach())
    for got, w in zip(matrices + vectors, want):
        assert float(torch.linalg.vector_norm(got.double() - w) / torch.linalg.vector_norm(w)) <= 0.08


def test_the_example_learns():
    import torch
    ex, model, _ = model_and_batch()
    losses = [float(model.step(*ex.batch(512, 1024, t), 0.02, t)) for t in range(40)]
    assert all(l == l for l in losses)
    assert losses[-1] < losses[0] - 1.0, losses
    assert model.opt.status()["failed_roots"] == 0
