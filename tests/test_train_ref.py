"""The 64-bit definitions that the GPU tests compare with, pinned on the CPU:
gradients against differences, constructed cases worked by hand."""
import math

import numpy as np
import pytest

import train_ref as ref


@pytest.mark.parametrize("V,inv_t,h", [(2, 1.0, 0.0), (7, 0.7, 0.3), (40, 1.6, -0.2)])
def test_logp_gradient_is_the_difference_quotient(V, inv_t, h):
    rng = np.random.default_rng(V)
    x, t, g = rng.normal(size=V) * 2, V // 2, 0.8

    def loss(y):
        (logp, _, ent), _ = ref.token_logp(y, t, inv_t)
        return g * logp + h * ent

    (_, lse, ent), _ = ref.token_logp(x, t, inv_t)
    grad, _ = ref.token_logp_grad(x, t, inv_t, lse, ent, g, h, "f32")
    step = 1e-5
    for j in range(V):
        e = np.zeros(V)
        e[j] = step
        # a central difference is off by step^2 / 6 of the third derivative and
        # by the 64-bit rounding over the step
        assert abs((loss(x + e) - loss(x - e)) / (2 * step) - grad[j]) < 1e-8
    assert abs(grad.sum()) < 1e-14  # a shift of all logits changes nothing


def test_logp_by_hand():
    (logp, lse, h), _ = ref.token_logp(np.zeros(8), 3, 1.0)
    assert (logp, lse, h) == (-math.log(8), math.log(8), math.log(8))
    (logp, lse, h), _ = ref.token_logp(np.array([-np.inf, 0.0, -np.inf]), 1, 1.0)
    assert (logp, lse, h) == (0.0, 0.0, 0.0)
    assert ref.token_logp(np.zeros(8), -1, 1.0)[0] == (0.0, 0.0, 0.0)
    assert ref.token_logp(np.full(4, -np.inf), 1, 1.0)[0] == (-np.inf, -np.inf, 0.0)


@pytest.mark.parametrize("reduction", [0, 1, 2])
@pytest.mark.parametrize("with_ref", [True, False])
def test_policy_gradient_is_the_difference_quotient(reduction, with_ref):
    rng = np.random.default_rng(3 + reduction)
    N, start = 24, np.array([0, 5, 5, 6, 20, 24])
    logp = -np.abs(rng.normal(size=N))
    old = logp + 0.3 * rng.normal(size=N)
    r = logp + 0.4 * rng.normal(size=N) if with_ref else None
    adv = rng.normal(size=5)
    mask = rng.integers(0, 2, N)
    args = (old, r, adv, False, mask, start, reduction, 0.7, 0.2, 0.3, 0.5)
    terms, _, grad, _ = ref.policy(logp, *args)
    assert abs(terms[0] - terms[1] - 0.5 * terms[2]) < 1e-14
    step = 1e-6
    for i in range(N):
        e = np.zeros(N)
        e[i] = step
        diff = (ref.policy(logp + e, *args)[0][0] - ref.policy(logp - e, *args)[0][0]) / (2 * step)
        assert abs(diff - grad[i]) < 1e-8
    assert not grad[mask == 0].any()


def test_policy_weights_by_hand():
    # on-policy tokens: every ratio is 1, so the policy term is minus the mean
    # advantage: over 6 tokens, or over the two sequences that have any
    lp = np.full(8, -1.0)
    start, mask = np.array([0, 4, 4, 8]), np.array([1, 1, 1, 1, 1, 1, 0, 0])
    adv = np.array([3.0, 9.0, -6.0])
    assert abs(ref.policy(lp, lp, None, adv, False, mask, start, 0, 1.0, 0.2, 0.2, 0.0)[0][0] - 0.0) < 1e-15
    assert abs(ref.policy(lp, lp, None, adv, False, mask, start, 1, 1.0, 0.2, 0.2, 0.0)[0][0] - 1.5) < 1e-15
    assert not ref.policy(lp, lp, lp, adv, False, np.zeros(8), start, 1, 1.0, 0.2, 0.2, 1.0)[0].any()


def test_norms_by_hand():
    per, total, wrong = ref.norms([np.array([3.0, 4.0]), np.zeros(0), np.array([12.0])])
    assert per == [5.0, 0.0, 12.0] and total == 13.0 and wrong == [0, 0, 0]
    assert ref.norms([np.array([np.inf, np.nan, 1.0])])[2] == [2]
