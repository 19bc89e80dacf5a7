"""The training step of examples/train_step.py: its gradients against PyTorch's own, and that it learns."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    spec = importlib.util.spec_from_file_location("train_step", os.path.join(ROOT, "examples", "train_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradients_of_the_step(example):
    """In binary32 throughout, PyTorch's differ from the step's by the bfloat16 roundings of hidden states and weight (2^-8 each,
    the same values on both sides here), of d and of the results: under 2 % of each gradient's norm."""
    import torch
    model = example.Model(seed=3)
    tokens, targets = example.batch(0)
    loss, grads = model.gradients(tokens, targets)
    embedding, mix = (p.detach().clone().requires_grad_() for p in (model.embedding, model.mix))
    head = model.head.to(torch.bfloat16).float().requires_grad_()
    hidden = torch.tanh(embedding[tokens] @ mix).to(torch.bfloat16).float()
    want = torch.nn.functional.cross_entropy(hidden @ head.t(), targets, ignore_index=example.IGNORE)
    want.backward()
    assert abs(float(loss) - float(want)) < 1e-4 * float(want)
    for got, ref in zip(grads, (embedding.grad, mix.grad, head.grad)):
        assert float((got.float() - ref).norm()) < 0.02 * float(ref.norm())


def test_the_step_learns_from_clipped_compressed_gradients(example):
    losses = example.main(steps=60)
    assert losses[0] > 7.0 and losses[-1] < 0.7 * losses[0]


def test_the_step_clips_the_exchanged_gradient(example):
    """What the update takes has the limit's norm: clipping comes after the exchange, which changes norms (rounding to 8 bits adds to them),
    and its factor follows from what every rank holds.  Limit / norm, the norm itself and the products are each rounded to binary32."""
    import torch
    model = example.Model(seed=3)
    for max_norm in (0.05, 1e9):
        before = [p.detach().clone() for p in model.layers]
        model.step(*example.batch(0), seed=1, rate=1.0, max_norm=max_norm)
        size, norm = float(model.fused.double().norm()), float(model.norm)
        assert norm > 0.05
        assert abs(size - min(max_norm, norm)) <= 2.0**-22 * size
        for p, b, lo, hi in zip(model.layers, before, model.plan.offsets[:-1], model.plan.offsets[1:]):
            assert torch.equal(p.detach(), b - model.fused[lo:hi].view_as(b))
