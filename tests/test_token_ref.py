"""The 64-bit statements of the post-training operators against differences and
closed forms (no GPU)."""
import numpy as np
import pytest

import token_ref as ref

H = 1e-5


def _data(n=6, V=11, seed=0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, V)) * 2
    y = rng.integers(0, V, n)
    y[1] = -1
    return rng, x, y


def _differences(f, x):
    d = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = H
        d[i] = (f(x + e) - f(x - e)) / (2 * H)
    return d


def test_logp_gradient_against_differences():
    rng, x, y = _data()
    g, s = rng.standard_normal(len(y)), 1.3
    want = _differences(lambda v: (g * ref.token_logp(v, y, s)).sum(), x)
    np.testing.assert_allclose(ref.gradient(x, y, g, s), want, atol=1e-8)


@pytest.mark.parametrize("kl", [0.0, 0.1])
def test_policy_gradient_against_differences(kl):
    rng, x, y = _data(seed=1)
    n, s = len(y), 0.7
    logp = ref.token_logp(x, y, s)
    old, rf = logp + rng.standard_normal(n) * 0.3, logp + rng.standard_normal(n) * 0.3
    adv, w = rng.standard_normal(n), np.array([0.2, 0.3, 0.0, 0.5, 0.1, 0.4])

    def f(v):
        return ref.policy(ref.token_logp(v, y, s), y, old, adv, w, rf, 0.2, 0.28, kl)

    want = _differences(lambda v: f(v)[0], x)
    np.testing.assert_allclose(ref.gradient(x, y, f(x)[2], s), want, atol=1e-8)


def test_preference_gradient_against_differences():
    rng, x, y = _data(n=9, seed=2)
    off = np.array([0, 2, 5, 5, 9])      # the second pair's preferred sequence is empty
    w, s = np.array([0.4, 1.1]), 1.0
    rf = ref.token_logp(x, y, s) + rng.standard_normal(9) * 0.3
    none = np.zeros(9, bool)

    def f(v):
        return ref.preference(ref.token_logp(v, y, s), y, off, rf, w, 0.5, 0.1, none)

    want = _differences(lambda v: f(v)[0], x)
    np.testing.assert_allclose(ref.gradient(x, y, f(x)[3], s), want, atol=1e-8)


def test_closed_forms():
    x = np.zeros((1, 8))
    np.testing.assert_allclose(ref.token_logp(x, np.array([3]), 2.0), -np.log(8))
    # equal log ratios: margin 0, loss log 2, slope -beta/2
    loss, each, _, coef = ref.preference(np.full(2, -1.0), np.array([0, 0]), np.array([0, 1, 2]), np.zeros(2),
                                         np.ones(1), 0.3, 0.0, np.zeros(2, bool))
    np.testing.assert_allclose([loss, each[0]], np.log(2))
    np.testing.assert_allclose(coef, [-0.15, 0.15])
    # the old policy itself: ratio 1, loss -A, slope -A
    lp = np.array([-2.0])
    loss, _, slope = ref.policy(lp, np.array([0]), lp, np.array([1.5]), np.ones(1), lp, 0.2, 0.2, 0.5)
    np.testing.assert_allclose([loss, slope[0]], -1.5)


def test_dropout_bits_are_even():
    b = ref.dropout_bits(5, 0, 0, 0, 40_000)
    counts = np.bincount(b >> 12, minlength=16)
    chi2 = ((counts - 2500) ** 2 / 2500).sum()
    assert chi2 < 45          # 15 degrees of freedom: passed by all but 1e-4 of seeds
    other = ref.dropout_bits(5, 0, 1, 0, 40_000)
    assert abs(np.corrcoef(b, other)[0, 1]) < 0.02
