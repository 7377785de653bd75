"""The 64-bit formulas that the kernels of the losses are compared with, against central differences of their own
totals: a gradient written down wrong would show here, without a GPU.

Step h = 1e-5: the difference's error is h^2/6 times a third derivative (of order 1, times the weights) plus 2^-52/h times
the total's size, some 1e-10; 1e-7 of the gradient's scale is asked for."""
import numpy as np
import pytest

import losses_reference as ref


def _differences(total, z, h=1e-5):
    g = np.zeros(z.shape)
    for i in np.ndindex(*z.shape):
        if not np.isfinite(z[i]):
            continue
        up, down = z.copy(), z.copy()
        up[i] += h
        down[i] -= h
        g[i] = (total(up) - total(down)) / (2 * h)
    return g


def _near(got, want):
    assert np.abs(got - want).max() <= 1e-7 * max(1.0, np.abs(want).max()), np.abs(got - want).max()


@pytest.mark.parametrize("s", [1.0, 0.5])
def test_token_gradient(s):
    rng = np.random.default_rng(1)
    z = rng.normal(size=(4, 7)) * 2
    z[1, 2] = -np.inf
    y = np.array([3, 0, -100, 6])
    d, e = rng.normal(size=4), rng.normal(size=4)

    def total(x):
        logp, _, H = ref.token_logprob(x, y, s)
        return np.sum(d * logp + e * H)

    _near(ref.token_grad(z, y, s, d, e), _differences(total, z))


@pytest.mark.parametrize("kl_kind", ["k1", "k2", "k3"])
def test_policy_gradient(kl_kind):
    rng = np.random.default_rng(2)
    z = rng.normal(size=(12, 5))
    y = rng.integers(0, 5, 12)
    y[3] = -1
    logp = ref.token_logprob(z, y, 0.8)[0]
    x = rng.normal(size=12) * 0.3                  # (some ratios are clipped; none is near an edge)
    x[np.abs(np.exp(x) - 1.2) < 0.01] += 0.05
    x[np.abs(np.exp(x) - 0.7) < 0.01] += 0.05
    old, r = logp - x, logp - rng.normal(size=12) * 0.4
    adv, w = rng.normal(size=12), rng.random(12)
    w[5] = 0

    def run(q):
        return ref.policy(q, y, old, adv, r, w, 0.8, 0.3, 0.2, 0.1, kl_kind, 0.05, 3.0)

    _near(run(z)[4], _differences(lambda q: run(q)[0], z))


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("s", [1.0, 0.5])
def test_distill_gradient(rest, s):
    rng = np.random.default_rng(3)
    z = rng.normal(size=(5, 9))
    index = np.array([[1, 4, 8], [0, 0, 2], [5, -1, 3], [-1, -1, -1], [7, 2, 1]])
    a = rng.normal(size=(5, 3)) + 1
    scaled = np.where(index >= 0, a * s, -np.inf)
    lse = np.logaddexp.reduce(scaled, axis=1) + 0.4 if rest else None
    if rest:
        lse[3] = 1.0
    w = rng.random(5) + 0.1

    def run(q):
        return ref.distill(q, index, a, lse, w, s, 2.0)

    _near(run(z)[2], _differences(lambda q: run(q)[0], z))


@pytest.mark.parametrize("kind", ["sigmoid", "hinge", "ipo"])
@pytest.mark.parametrize("normalised", [False, True])
def test_preference_gradient(kind, normalised):
    rng = np.random.default_rng(4)
    off = np.array([1, 5, 5, 9, 12, 15, 20])        # three pairs; one chosen answer is empty
    logp, r = -rng.random(22), -rng.random(22)
    mask = rng.random(22) < 0.8
    w = rng.random(3)

    def run(x):
        return ref.preference(x, r, off, mask, w, 0.7, kind, 0.1 if kind == "sigmoid" else 0.0, 0.2, normalised, 1.5)

    _near(run(logp)[3], _differences(lambda x: run(x)[0], logp))
