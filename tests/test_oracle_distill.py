"""The oracle of the distillation operators against differences and hand-computed cases."""
import numpy as np
import pytest

from oracle import distill


def _difference(f, x, at, h=1e-6):
    up, down = x.copy(), x.copy()
    up.reshape(-1)[at] += h
    down.reshape(-1)[at] -= h
    return (f(up) - f(down)) / (2 * h)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("rest", [None, -1.0, 3.0])
@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_distill_gradient_is_the_difference(reverse, rest, tau):
    if reverse and rest is None:
        return
    rng = np.random.default_rng(3)
    s = rng.normal(size=23) * 2
    token = np.array([4, 0, -1, 22, 9])
    logit = rng.normal(size=5) * 2
    loss, g = distill.distill_row(s, token, logit, rest, tau, reverse)
    assert loss > 0
    for j in range(23):
        d = _difference(lambda x: distill.distill_row(x, token, logit, rest, tau, reverse)[0], s, j)
        assert abs(d - g[j]) < 1e-8  # differences of h = 1e-6: h^2 and 1e-16 / h


def test_distill_of_the_students_own_list_is_zero():
    rng = np.random.default_rng(4)
    s = rng.normal(size=(1, 50))
    logit, token, rest = distill.top_logits(s, 7, 1.7)
    for reverse in (False, True):
        loss, g = distill.distill_row(s[0], token[0], logit[0], rest[0], 1.7, reverse)
        assert abs(loss) < 1e-14 and np.max(np.abs(g)) < 1e-15


def test_top_logits_order_and_rest():
    logit, token, rest = distill.top_logits(np.array([[1.0, 3.0, -0.0, 3.0, 0.0]]), 3)
    assert token.tolist() == [[1, 3, 0]] and logit.tolist() == [[3.0, 3.0, 1.0]]
    assert abs(rest[0] - np.log(2.0)) < 1e-15
    assert distill.top_logits(np.ones((1, 4)), 4)[2][0] == -np.inf


def test_a_list_of_one_token_is_cross_entropy():
    rng = np.random.default_rng(5)
    s = rng.normal(size=11)
    loss, g = distill.distill_row(s, np.array([3]), np.array([-7.0]), None)
    p = np.exp(s) / np.exp(s).sum()
    assert abs(loss + np.log(p[3])) < 1e-14
    p[3] -= 1
    assert np.max(np.abs(g - p)) < 1e-15


def test_linear_ce_gradients_are_the_differences():
    rng = np.random.default_rng(6)
    x, w = rng.normal(size=(4, 8)), rng.normal(size=(9, 8))
    token, weight, valid = np.array([2, 8, 0, 99]), np.array([1.0, -0.5, 2.0, 1.0]), np.array([1, 1, 0, 1])
    loss, logp, dx, dw = distill.linear_ce(x, w, token, weight, valid, 0.25)
    assert loss[2] == 0 and np.isnan(loss[3]) and np.all(np.isnan(dx[3])) and np.all(dx[2] == 0)
    total = lambda a, b: 0.25 * np.nansum(distill.linear_ce(a, b, token, weight, valid)[0])  # noqa: E731
    for at in range(0, 24, 5):
        assert abs(_difference(lambda a: total(a, w), x, at) - dx.reshape(-1)[at]) < 1e-8
    for at in range(0, 72, 7):
        assert abs(_difference(lambda b: total(x, b), w, at) - dw.reshape(-1)[at]) < 1e-8


def test_a_list_over_tokens_below_the_least_number():
    """The student gives the unlisted tokens e^-900 of the row: the forward gradient is finite and sums to 0."""
    s = np.zeros(40)
    s[:2] = 900.0
    loss, g = distill.distill_row(s, np.array([0, 1]), np.array([1.0, 1.0]), 0.0)
    assert np.isfinite(loss) and loss > 100
    assert abs(g.sum()) < 1e-12 and g[5] < -1e-3  # (logarithms near 900 are rounded by 2^-44 each)
