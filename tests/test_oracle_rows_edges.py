"""The float64 oracle of the operators on rows of logits at the ends of its range, against logarithms and closed forms.
CPU only."""
import math

import numpy as np
import pytest
import torch

import oracle


@pytest.mark.parametrize("kind", ["tail", "reverse"])
@pytest.mark.parametrize("gap", [1.0, 90.0, 900.0])
def test_a_class_outside_far_below_the_list(rng, gap, kind):
    """Below float64's range the mass outside still has a logarithm: by differentiation of logarithms."""
    n, V, k = 3, 30, 4
    x = rng.standard_normal((n, V))
    x[:, :k] += gap
    x[:, V - 2:] = -np.inf
    ids, values = np.tile(np.arange(k), (n, 1)), np.log(np.full((n, k), 0.2))
    loss, grad = oracle.distill_loss(x, ids, values, kind=kind)
    t = torch.from_numpy(x).requires_grad_()
    lq = torch.log_softmax(t, 1)
    v, out = torch.from_numpy(values), torch.logsumexp(lq[:, k:], 1)
    if kind == "tail":
        ref = (torch.exp(v) * (v - lq[:, :k])).sum(1) + 0.2 * (math.log(0.2) - out)
    else:
        ref = (torch.exp(lq[:, :k]) * (lq[:, :k] - v)).sum(1) + torch.exp(out) * (out - math.log(0.2))
    (g,) = torch.autograd.grad(ref.sum(), t)
    assert np.allclose(loss, ref.detach().numpy(), rtol=1e-13, atol=1e-13)
    assert np.allclose(grad, g.numpy(), rtol=1e-12, atol=1e-13)


@pytest.mark.parametrize("kind", ["topk", "tail", "reverse"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_teachers_values_that_are_no_numbers(rng, bad, kind):
    x = rng.standard_normal((2, 9))
    x[1, 4] = -np.inf
    loss, _ = oracle.distill_loss(x, np.array([[1, 4], [1, 4]]), np.array([[-1.0, bad], [-1.0, bad]]), kind=kind)
    assert not np.isfinite(loss).any()


def test_ratios_that_are_no_finite_numbers(rng):
    """A token that cannot occur has r = 0 whatever the old policy gave it; an advantage of 0 has no surrogate."""
    x = rng.standard_normal((4, 9))
    x[0, 4] = x[1, 4] = -np.inf
    old, adv = np.array([-np.inf, -1.0, -np.inf, -np.inf]), np.array([1.0, 1.0, 0.0, 2.0])
    loss, _, _, grad = oracle.policy_loss(x, np.full(4, 4), old, adv)
    assert loss.tolist() == [0.0, 0.0, 0.0, -1.2 * 2.0] and not grad.any()
