"""The plain implementations that the GPU tests of the logits operators compare
with, checked by themselves (CPU): the draw in whole numbers against the one in
64 bits, and the divergence's gradient against differences of its loss."""
import numpy as np
import pytest

from tests import rows_ref as R


@pytest.mark.parametrize("T,k,p,q", [(1.0, 0, 1.0, 0.0), (0.7, 5, 1.0, 0.0), (1.3, 0, 0.8, 0.0), (1.0, 20, 0.9, 0.05)])
def test_draw_follows_the_kept_probabilities(T, k, p, q):
    rng = np.random.default_rng(5)
    l = (2 * rng.standard_normal(97)).astype(np.float32)
    e = np.exp2(R.exponents(l, T)).astype(np.float32)
    prob = R.probabilities(l, T)
    order = np.argsort(-prob, kind="stable")
    n = len(l) if k == 0 else k
    mass = np.cumsum(prob[order])
    keep = (np.arange(len(l)) < n) & (mass - prob[order] < p * mass[n - 1]) & (prob[order] >= q * prob[order[0]])
    want = np.zeros(len(l))
    want[order] = prob[order] * keep
    want /= want.sum()
    us = (np.arange(4096) + 0.5) / 4096
    got = np.bincount([R.draw(l, e, float(np.float32(u)), T, k, p, q)[0] for u in us], minlength=len(l)) / 4096
    assert np.abs(got - want).max() <= 1 / 4096 + 1e-6  # a token's run of equally spaced numbers, to one at an end
    tok, conf = R.draw(l, e, 0.5, T, k, p, q)
    assert abs(conf - prob[tok]) <= 1e-5 * prob[tok]


def test_draw_of_rows_without_a_choice():
    e = np.zeros(3, np.float32)
    for row in ([-np.inf] * 3, [np.nan] * 3, [1.0, np.inf, 0.0]):
        with np.errstate(all="ignore"):
            assert R.draw(np.array(row, np.float32), e, 0.5, 1.0, 0, 1.0, 0.0) == (-1, 0.0)


@pytest.mark.parametrize("tau,with_rest", [(1.0, True), (2.0, False), (0.5, True)])
def test_divergence_gradient_against_differences(tau, with_rest):
    rng = np.random.default_rng(8)
    l = rng.standard_normal(23) * 2
    ids = np.array([4, 17, 4, -1, 9])  # one listed twice, one absent
    t = rng.standard_normal(5)
    lse = np.log(np.exp(t[ids >= 0] / tau).sum()) + 0.3 if with_rest else None
    loss, grad, _, _ = R.distill(l, ids, t, tau, lse)
    assert loss > 0 or not with_rest
    h = 1e-5
    for j in range(len(l)):
        a, b = l.copy(), l.copy()
        a[j] += h
        b[j] -= h
        d = (R.distill(a, ids, t, tau, lse)[0] - R.distill(b, ids, t, tau, lse)[0]) / (2 * h)
        assert abs(d - grad[j]) <= 1e-8  # h^2 times the third derivative, plus 2^-52 / h
    assert abs(grad.sum()) <= 1e-12


def test_divergence_is_zero_at_the_teacher():
    l = np.log(np.array([0.5, 0.2, 0.2, 0.1]))
    loss, grad, lse, lse_rest = R.distill(l, [0, 1], l[:2], 1.0, 0.0)
    assert abs(loss) < 1e-14 and np.abs(grad).max() < 1e-14 and abs(lse) < 1e-14 and abs(lse_rest - np.log(0.3)) < 1e-14
