"""Samples without a label in the deep head's training step: they count for the
entropy bonus alone."""

import pytest

from .gpu_common import lib_ready, torch_cuda
from .test_gpu_deep_head import batch, example  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def test_without_a_bonus_no_norm_and_no_bias_sees_them(example):  # noqa: F811
    """Their rows of the logits' gradient are zeros, so the rows on the way back are, and the sums over rows of the gammas'
    and the bias's gradients have the same bits whatever these samples are.  (The weights' products quantize the batch's
    activations in blocks of 128 samples, whose scales these share.)"""
    import torch
    n = 2
    head = example.DeepHead(192, 128, 160, n, seed=1, bonus=0.0)
    h, y = batch(torch, 64)
    y[::2] = -1
    _, grads = head.gradients(h, y)
    h2 = h.clone()
    h2[::2] = torch.relu(torch.randn(32, 192, generator=torch.Generator().manual_seed(9))).cuda().bfloat16()
    _, again = head.gradients(h2, y)
    gammas = slice(2 * n + 2, 3 * n + 3)
    assert [g.shape for g in grads[gammas]] == [(128,)] * (n + 1)
    for a, b in zip(grads[gammas] + grads[-1:], again[gammas] + again[-1:]):
        assert torch.equal(a, b) and bool((a != 0).any())
    y[:] = -1
    loss, none = head.gradients(h, y)
    assert float(loss) == 0.0 and all(bool((g == 0).all()) for g in none)
    head.check()


def test_with_a_bonus_they_add_its_part(example):  # noqa: F811
    """The logits do not depend on the labels, so the bias's gradient (the column sums of dx = g (1[label] - p) - g' p (ln p +
    H), g = -1 / 64 for a labelled sample and 0 for another, g' = -bonus / 64) is the sum of that without a bonus and that
    without labels.  An element is two products and a sum of d = x - m and of g + g' (H - ln s): 8 roundings and 2^-21 of an
    approximate exponential, of parts that are below (1 + bonus (|d| + H + ln s)) / 64 with |d| below 30 here; a column adds
    64 of them.  Three such sums are compared."""
    import torch
    bonus = 0.5
    h, y = batch(torch, 64)
    some = y.clone()
    some[::2] = -1
    none = torch.full_like(y, -1)

    def bias_gradient(bonus, labels):
        head = example.DeepHead(192, 128, 160, 1, seed=1, bonus=bonus)
        _, grads = head.gradients(h, labels)
        head.check()
        return grads[-1].double()

    joined, labels_alone, bonus_alone = bias_gradient(bonus, some), bias_gradient(0.0, some), bias_gradient(bonus, none)
    tol = 3 * (64 + 8 + 8) * U * (1 + bonus * 36)
    assert bool(((joined - labels_alone - bonus_alone).abs() <= tol).all())
    assert float(bonus_alone.abs().max()) > 4 * tol
    # the unlabelled half alone: with the bonus, other samples there give another gradient
    h2 = h.clone()
    h2[::2] = torch.relu(torch.randn(32, 192, generator=torch.Generator().manual_seed(9))).cuda().bfloat16()
    head = example.DeepHead(192, 128, 160, 1, seed=1, bonus=bonus)
    _, other = head.gradients(h2, some)
    assert float((other[-1].double() - joined).abs().max()) > 4 * tol
