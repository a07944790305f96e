"""The example that uses the layer operators together: an 8-bit head on FF
activities learns, repeats bit for bit, answers single samples as in a batch,
and its gradients follow the loss."""

import importlib.util
import os

import numpy as np
import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    torch_cuda()
    lib_ready()
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "eight_bit_head.py")
    spec = importlib.util.spec_from_file_location("eight_bit_head", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_learns_serves_and_repeats(example):
    said = []
    kw = dict(samples=2048, batch=256, steps=40, widths=(300, 250), hidden=96, groups=10, report=said.append)
    losses, accuracy, same = example.run(**kw)
    # chance: log 10 and 0.1; the task's classes can be read off their supports
    assert np.isfinite(losses).all() and losses[-8:].mean() < 0.5 * np.log(10.0)
    assert accuracy > 0.7
    # a sample alone takes the path for few rows, whose sums have another order: at most an argmax near a tie may differ
    assert same >= 15
    again, accuracy2, same2 = example.run(**kw)
    assert np.array_equal(losses, again) and accuracy == accuracy2 and same == same2 and said[0] == said[1]


def test_its_gradients_follow_the_loss(example):
    """The loss of the same batch and masks falls along the gradient by about
    the gradient's square times the step.  e4m3 operands leave each product
    with rounding of 2^-4 per term at most, independent between terms, so a
    gradient of thousands of values keeps its direction: the measured fall is
    asked for within a factor of two."""
    import torch
    torch.manual_seed(0)
    head = example.EightBitHead(192, 64, 8, p=0.25, seed=3)
    h = torch.relu(torch.randn(512, 192, device="cuda")).bfloat16()
    y = torch.randint(0, 10, (512,), device="cuda")
    loss, grads = head.gradients(h, y)
    norm2 = sum(float((g.double() ** 2).sum()) for g in grads)
    step = 0.02 / norm2 ** 0.5
    for p, g in zip(head.parameters, grads):
        p -= step * g
    after, _ = head.gradients(h, y)
    fall, expected = float(loss) - float(after), step * norm2
    assert 0.5 * expected < fall < 2.0 * expected
    head.check()
